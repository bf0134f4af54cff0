// Layer norm over the last axis and its gradients, for the norms in front of a transformer block's
// projections: affine, or modulated by one scale and shift per sample (adaptive layer norm).
//
//   mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),  n = (x - mean) rstd,  y = n w + b
//   g = dy w:   dx = rstd (g - sum g / C - n sum(g n) / C),   dw = sum_rows dy n,   db = sum_rows dy
//
// Both directions are bound by HBM: every element is read once (twice as many streams backward) and written
// once.  A row stays in registers between its statistics and its output; sums are fp32, the variance is taken
// around the mean that has already been summed (no difference of large squares).
#include <cuda_bf16.h>

#include <algorithm>

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace hilberta {
namespace {

constexpr int MAX_COLS = 16384;

// VEC elements at p, as floats: one 16-byte load (VEC * sizeof(T) = 16, or 32 in two), or one element.
template <class T, int VEC>
struct Vec {
    static constexpr int BYTES = VEC * (int)sizeof(T);
    static constexpr int WORDS = BYTES / 4 ? BYTES / 4 : 1;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (BYTES >= 16) {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) {
                const uint4 v = *(reinterpret_cast<const uint4 *>(p) + i);
                w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
            }
        } else if constexpr (BYTES == 4) {
            w[0] = *reinterpret_cast<const uint32_t *>(p);
        } else {
            w[0] = *reinterpret_cast<const uint16_t *>(p);
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0u;
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float((i & 1) ? (w[i >> 1] & 0xffff0000u) : (w[i >> 1] << 16));
    }
    __device__ __forceinline__ void set(const float *f) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[i] = __float_as_uint(f[i]);
        } else if constexpr (VEC == 1) {
            w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(f[0]));
        } else {
#pragma unroll
            for (int i = 0; i < VEC / 2; ++i) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
    }
    __device__ __forceinline__ void store(T *p) const {
        if constexpr (BYTES >= 16) {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i)
                *(reinterpret_cast<uint4 *>(p) + i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        } else if constexpr (BYTES == 4) {
            *reinterpret_cast<uint32_t *>(p) = w[0];
        } else {
            *reinterpret_cast<uint16_t *>(p) = (uint16_t)w[0];
        }
    }
};

struct ForwardParams {
    const void *x, *weight, *bias;
    void *y;
    float *mean, *rstd;
    long long rows, rows_per_group, stride_x, stride_y, stride_w;
    int cols;
    float eps, offset;   // offset is added to the weight
};

// sum over LANES consecutive lanes of a warp, in all of them
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// LANES <= 32: that many lanes of a warp have a row; more: one row for the CTA of LANES threads.
// NV vectors of VEC elements per thread, strided by LANES, so that neighbouring lanes take neighbouring ones.
template <class T, class W, int VEC, int LANES, int NV>
__global__ void __launch_bounds__(LANES > 32 ? LANES : 128)
layer_norm_kernel(const ForwardParams prm) {
    constexpr int THREADS = LANES > 32 ? LANES : 128;
    constexpr int ROWS = THREADS / LANES;
    __shared__ float part[2][LANES > 32 ? LANES / 32 : 1];
    const int lane = threadIdx.x % LANES, cols = prm.cols;
    const long long row = (long long)blockIdx.x * ROWS + threadIdx.x / LANES;
    const bool in = row < prm.rows;
    allow_next();
    wait_for_previous();
    auto row_sum = [&](float v, int k) {
        v = lanes_sum<LANES < 32 ? LANES : 32>(v);
        if constexpr (LANES > 32) {
            if (threadIdx.x % 32 == 0) part[k][threadIdx.x / 32] = v;
            __syncthreads();
            v = 0.f;
#pragma unroll
            for (int i = 0; i < LANES / 32; ++i) v += part[k][i];
        }
        return v;
    };
    const T *x = (const T *)prm.x + row * prm.stride_x;
    Vec<T, VEC> v[NV];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * LANES + lane) * VEC;
        if (in && c < cols) v[i].load(x + c);
        else v[i].zero();
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum += v[i].get(e);
    const float mean = row_sum(sum, 0) / (float)cols;
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * LANES + lane) * VEC;
        if (c < cols) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float d = v[i].get(e) - mean;
                sq = fmaf(d, d, sq);
            }
        }
    }
    const float rstd = 1.f / sqrtf(row_sum(sq, 1) / (float)cols + prm.eps);
    if (!in) return;
    if (lane == 0) {
        if (prm.mean) prm.mean[row] = mean;
        if (prm.rstd) prm.rstd[row] = rstd;
    }
    const long long group = prm.rows_per_group >= prm.rows ? 0 : row / prm.rows_per_group;
    const W *w = prm.weight ? (const W *)prm.weight + group * prm.stride_w : nullptr;
    const W *b = prm.bias ? (const W *)prm.bias + group * prm.stride_w : nullptr;
    T *y = (T *)prm.y + row * prm.stride_y;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * LANES + lane) * VEC;
        if (c >= cols) continue;
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = (v[i].get(e) - mean) * rstd;
        if (w) {
            Vec<W, VEC> t;
            t.load(w + c);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] *= t.get(e) + prm.offset;
        }
        if (b) {
            Vec<W, VEC> t;
            t.load(b + c);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] += t.get(e);
        }
        Vec<T, VEC> o;
        o.set(f);
        o.store(y + c);
    }
}

struct BackwardParams {
    const void *dy, *x, *weight;
    const float *mean, *rstd;
    void *dx, *dweight, *dbias;
    float *partial;   // [groups, ctas, 2, cols] sums of each CTA, nullptr with one CTA a group
    long long rows, rows_per_group, stride_dy, stride_x, stride_dx, stride_w, stride_dw;
    int cols;
    float offset;
    int stages, pitch;   // of the ring in shared memory
};

// weights as the gradients use them: w [+ 1], 1 without any
template <class W, int VEC>
__device__ __forceinline__ void load_weights(float *w, const W *p, bool given, float offset) {
    Vec<W, VEC> v;
    v.zero();
    if (given) v.load(p);
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = given ? v.get(e) + offset : 1.f;
}

// this CTA's sum over its rows of dy n (which = 0) or dy (1) for one column: a partial sum, or the result
template <class W>
__device__ __forceinline__ void write_sum(const BackwardParams &prm, int which, int c, float sum) {
    if (prm.partial) {
        prm.partial[(((long long)blockIdx.y * gridDim.x + blockIdx.x) * 2 + which) * prm.cols + c] = sum;
    } else if (void *to = which ? prm.dbias : prm.dweight) {
        Vec<W, 1> o;
        o.set(&sum);
        o.store((W *)to + blockIdx.y * prm.stride_dw + c);
    }
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

// Sums over columns need every element of a row, sums over rows one column of all: a thread keeps its columns for all
// rows that its CTA sees (2 NV VEC fp32 sums in registers), and the two sums of a row cross the team that shares the row.

// Rows of few vectors: a team of LANES <= 32 lanes has a row (one vector each, R rows at a time for loads in flight),
// shuffles do the row sums and no barrier is needed until the teams' sums over rows are added up.
template <class T, class W, int VEC, int LANES, int R>
__global__ void __launch_bounds__(256)
layer_norm_bwd_lanes_kernel(const BackwardParams prm) {
    constexpr int TEAMS = 256 / LANES;
    __shared__ float part[2][TEAMS][LANES * VEC + 1];
    const int cols = prm.cols, lane = threadIdx.x % LANES, team = threadIdx.x / LANES, c = lane * VEC;
    const long long row_begin = (long long)blockIdx.y * prm.rows_per_group;
    const long long row_end = min(row_begin + prm.rows_per_group, prm.rows);
    const float inv_cols = 1.f / (float)cols;
    const bool in = c < cols;
    float dw[VEC] = {}, db[VEC] = {}, w[VEC];
    allow_next();
    wait_for_previous();
    load_weights<W, VEC>(w, (const W *)prm.weight + blockIdx.y * prm.stride_w + c, prm.weight && in, prm.offset);
    // a warp's teams stay together: the bound is that of the warp's first team
    const long long step = (long long)gridDim.x * TEAMS * R;
    for (long long r0 = row_begin + ((long long)blockIdx.x * TEAMS + team) * R; __any_sync(0xffffffffu, r0 < row_end); r0 += step) {
        Vec<T, VEC> x[R], dy[R];
        float mean[R], rstd[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool live = r0 + r < row_end;
            x[r].zero();
            dy[r].zero();
            mean[r] = live ? prm.mean[r0 + r] : 0.f;
            rstd[r] = live ? prm.rstd[r0 + r] : 0.f;
            if (live && in) {
                x[r].load((const T *)prm.x + (r0 + r) * prm.stride_x + c);
                dy[r].load((const T *)prm.dy + (r0 + r) * prm.stride_dy + c);
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float n[VEC], g[VEC], a = 0.f, b = 0.f;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float d = dy[r].get(e);
                n[e] = (x[r].get(e) - mean[r]) * rstd[r];
                g[e] = d * w[e];
                if (in) {
                    a += g[e];
                    b = fmaf(g[e], n[e], b);
                    dw[e] = fmaf(d, n[e], dw[e]);
                    db[e] += d;
                }
            }
            a = lanes_sum<LANES>(a) * inv_cols;
            b = lanes_sum<LANES>(b) * inv_cols;
            if (prm.dx && in && r0 + r < row_end) {
                Vec<T, VEC> o;
                float f[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] = rstd[r] * (g[e] - a - n[e] * b);
                o.set(f);
                o.store((T *)prm.dx + (r0 + r) * prm.stride_dx + c);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        part[0][team][c + e] = dw[e];
        part[1][team][c + e] = db[e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * cols; i += 256) {
        const int which = i / cols, col = i % cols;
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < TEAMS; ++t) sum += part[which][t][col];
        write_sum<W>(prm, which, col, sum);
    }
}

// Longer rows: the CTA is the team.  R rows at a time come through a ring of shared memory, filled STAGES - 1 rounds
// ahead by bulk copies (a register's worth of loads ahead left HBM idle at the barrier that the two row sums need), and
// are read from there twice, for the sums and for dx.  A row that does not start on a 16-byte boundary is copied from the
// boundary before to the one behind: the granules are those of its own first and last elements.
constexpr int MAX_STAGES = 4;
template <class T, class W, int VEC, int NV, int R>
__global__ void __launch_bounds__(512)
layer_norm_bwd_kernel(const BackwardParams prm) {
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ __align__(16) float part[2][16][2 * R];
    __shared__ uint64_t full[MAX_STAGES];
    const int cols = prm.cols, warps = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32, stages = prm.stages;
    const long long row_begin = (long long)blockIdx.y * prm.rows_per_group;
    const long long row_end = min(row_begin + prm.rows_per_group, prm.rows);
    const long long first = row_begin + (long long)blockIdx.x * R, step = (long long)gridDim.x * R;
    const int rounds = first < row_end ? (int)((row_end - first + step - 1) / step) : 0;
    const float inv_cols = 1.f / (float)cols;
    const int pitch = prm.pitch;   // bytes of a row in the ring
    float dw[NV * VEC] = {}, db[NV * VEC] = {};
    float w[NV * VEC];
    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) ptx::mbar_init(ptx::smem_u32(&full[i]), 1);
        ptx::mbar_fence_init();
    }
    allow_next();
    wait_for_previous();
    __syncthreads();
    // x and dy of round i into its stage
    auto fill = [&](int i) {
        const int s = i % stages;
        const uint32_t bar = ptx::smem_u32(&full[s]), to = ptx::smem_u32(ring) + (uint32_t)(s * 2 * R * pitch);
        const long long r0 = first + i * step;
        const int live = (int)min((long long)R, row_end - r0);
        const T *src[2] = {(const T *)prm.x + r0 * prm.stride_x, (const T *)prm.dy + r0 * prm.stride_dy};
        const long long stride[2] = {prm.stride_x, prm.stride_dy};
        uint32_t bytes = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k)
            for (int r = 0; r < live; ++r) {
                const uintptr_t at = (uintptr_t)(src[k] + r * stride[k]), from = at & ~(uintptr_t)15;
                bytes += (uint32_t)((at + (size_t)cols * sizeof(T) + 15 & ~(uintptr_t)15) - from);
            }
        ptx::mbar_expect_tx(bar, bytes);
#pragma unroll
        for (int k = 0; k < 2; ++k)
            for (int r = 0; r < live; ++r) {
                const uintptr_t at = (uintptr_t)(src[k] + r * stride[k]), from = at & ~(uintptr_t)15;
                bulk_load(to + (uint32_t)((k * R + r) * pitch), (const void *)from,
                          (uint32_t)((at + (size_t)cols * sizeof(T) + 15 & ~(uintptr_t)15) - from), bar);
            }
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < stages && i < rounds; ++i) fill(i);
    bool in[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * (int)blockDim.x + (int)threadIdx.x) * VEC;
        in[i] = c < cols;
        load_weights<W, VEC>(w + i * VEC, (const W *)prm.weight + blockIdx.y * prm.stride_w + c, prm.weight && in[i], prm.offset);
    }
    float mean_ahead[R], rstd_ahead[R];   // of the next round
    auto statistics = [&](long long r0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean_ahead[r] = r0 + r < row_end ? prm.mean[r0 + r] : 0.f;
            rstd_ahead[r] = r0 + r < row_end ? prm.rstd[r0 + r] : 0.f;
        }
    };
    statistics(first);
    for (int i = 0; i < rounds; ++i) {
        const int s = i % stages, k = i & 1;
        const long long r0 = first + i * step;
        const int live = (int)min((long long)R, row_end - r0);
        float mean[R], rstd[R], sum[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean[r] = mean_ahead[r];
            rstd[r] = rstd_ahead[r];
        }
        statistics(r0 + step);
        const T *xs[R], *ds[R];   // the rows in the ring
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint8_t *base = ring + (size_t)s * 2 * R * pitch;
            // VEC = 1: the offset within the granule
            xs[r] = (const T *)(base + r * pitch + (VEC == 1 ? ((uintptr_t)((const T *)prm.x + (r0 + r) * prm.stride_x) & 15) : 0));
            ds[r] = (const T *)(base + (R + r) * pitch + (VEC == 1 ? ((uintptr_t)((const T *)prm.dy + (r0 + r) * prm.stride_dy) & 15) : 0));
        }
        if (!ptx::mbar_wait(ptx::smem_u32(&full[s]), (i / stages) & 1)) return;   // never: the copy's bytes have been asked for
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float a = 0.f, b = 0.f;
            if (r < live) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    if (!in[v]) continue;
                    const int c = (v * (int)blockDim.x + (int)threadIdx.x) * VEC;
                    Vec<T, VEC> x, dy;
                    x.load(xs[r] + c);
                    dy.load(ds[r] + c);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float d = dy.get(e), n = (x.get(e) - mean[r]) * rstd[r], g = d * w[v * VEC + e];
                        a += g;
                        b = fmaf(g, n, b);
                        dw[v * VEC + e] = fmaf(d, n, dw[v * VEC + e]);
                        db[v * VEC + e] += d;
                    }
                }
            }
            sum[2 * r] = a;
            sum[2 * r + 1] = b;
        }
        // lane j of each eight (R = 4) is left with sum j over the warp: each step hands half of the sums over
        float total[2 * R];
        {
            int width = 2 * R;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                if (width > 1) {
                    width /= 2;
                    const bool up = (lane & o) != 0;
#pragma unroll
                    for (int j = 0; j < R; ++j) {
                        if (j >= width) continue;
                        const float keep = up ? sum[j + width] : sum[j], give = up ? sum[j] : sum[j + width];
                        sum[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                    }
                } else {
                    sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], o);
                }
            }
            // part[k] was last read two rounds ago, before the barrier of the round between
            constexpr int SHARE = 32 / (2 * R);
            if (lane % SHARE == 0) part[k][warp][lane / SHARE] = sum[0];
        }
        __syncthreads();
        // every thread is done with the round before: its stage takes the rows of the round that comes after those under way
        if (threadIdx.x == 0 && i > 0 && i - 1 + stages < rounds) fill(i - 1 + stages);
        if (prm.dx) {
#pragma unroll
            for (int j = 0; j < 2 * R; ++j) total[j] = 0.f;
            for (int q = 0; q < warps; ++q)
#pragma unroll
                for (int j = 0; j < 2 * R; j += 2) {
                    const float2 t = *reinterpret_cast<const float2 *>(&part[k][q][j]);
                    total[j] += t.x;
                    total[j + 1] += t.y;
                }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (r >= live) continue;
                const float a = total[2 * r] * inv_cols, b = total[2 * r + 1] * inv_cols;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    if (!in[v]) continue;
                    const int c = (v * (int)blockDim.x + (int)threadIdx.x) * VEC;
                    Vec<T, VEC> x, dy, o;
                    x.load(xs[r] + c);
                    dy.load(ds[r] + c);
                    float f[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float n = (x.get(e) - mean[r]) * rstd[r];
                        f[e] = rstd[r] * (dy.get(e) * w[v * VEC + e] - a - n * b);
                    }
                    o.set(f);
                    o.store((T *)prm.dx + (r0 + r) * prm.stride_dx + c);
                }
            }
        }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * (int)blockDim.x + (int)threadIdx.x) * VEC;
        if (!in[v]) continue;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            write_sum<W>(prm, 0, c + e, dw[v * VEC + e]);
            write_sum<W>(prm, 1, c + e, db[v * VEC + e]);
        }
    }
}

// dw, db of a group: the sums of its CTAs added up in a fixed order.  32 columns a block; SUMS rows of threads
// share the CTAs out.
constexpr int SUMS = 16;
template <class W>
__global__ void __launch_bounds__(32 * SUMS)
layer_norm_sums_kernel(const float *partial, void *dweight, void *dbias, int cols, int ctas, long long stride_dw) {
    __shared__ float part[SUMS][33];
    const int lane = threadIdx.x % 32, slot = threadIdx.x / 32, which = blockIdx.z;
    const int c = blockIdx.x * 32 + lane;
    allow_next();
    wait_for_previous();
    void *to = which ? dbias : dweight;
    if (!to) return;
    float sum = 0.f;
    if (c < cols) {
        const float *p = partial + ((long long)blockIdx.y * ctas * 2 + which) * cols + c;
#pragma unroll 8
        for (int i = slot; i < ctas; i += SUMS) sum += p[(long long)i * 2 * cols];
    }
    part[slot][lane] = sum;
    __syncthreads();
    if (slot == 0 && c < cols) {
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < SUMS; ++i) sum += part[i][lane];
        Vec<W, 1> o;
        o.set(&sum);
        o.store((W *)to + blockIdx.y * stride_dw + c);
    }
}

// The rows x cols elements at a (row stride sa) and at b: apart, or the very same rows?
bool rows_overlap(const void *a, long long sa, const void *b, long long sb, long long rows, int cols, size_t esz) {
    if (!a || !b || (a == b && sa == sb)) return false;
    const char *a0 = (const char *)a, *b0 = (const char *)b;
    const long long la = ((rows - 1) * sa + cols) * (long long)esz, lb = ((rows - 1) * sb + cols) * (long long)esz;
    return a0 < b0 + lb && b0 < a0 + la;
}

struct Shape {
    long long rows, rows_per_group, groups;
    int cols, dtype, weight_dtype;
    size_t esz, wsz;
};

int check_shape(Shape &s, long long rows, int cols, long long rows_per_group, int dtype, int weight_dtype) {
    if (rows < 0 || cols < 1 || rows_per_group < 0) return HILBERTA_ERR_INVALID;
    if ((dtype != HILBERTA_BF16 && dtype != HILBERTA_FP32) || (weight_dtype != dtype && weight_dtype != HILBERTA_FP32))
        return dtype == HILBERTA_FP8_E4M3 || (dtype == HILBERTA_FP32 && weight_dtype == HILBERTA_BF16) ? HILBERTA_ERR_UNSUPPORTED
                                                                                                       : HILBERTA_ERR_INVALID;
    if (cols > MAX_COLS || rows > (1ll << 40)) return HILBERTA_ERR_UNSUPPORTED;
    s.rows = rows;
    s.rows_per_group = rows_per_group ? rows_per_group : std::max(rows, 1ll);
    s.groups = rows ? (rows + s.rows_per_group - 1) / s.rows_per_group : 0;
    s.cols = cols;
    s.dtype = dtype;
    s.weight_dtype = weight_dtype;
    s.esz = dtype == HILBERTA_BF16 ? 2 : 4;
    s.wsz = weight_dtype == HILBERTA_BF16 ? 2 : 4;
    return HILBERTA_OK;
}

bool aligned16(const void *p, long long stride, size_t esz) {
    return ((uintptr_t)p & 15) == 0 && (stride * (long long)esz) % 16 == 0;
}

template <class F>
int by_types(const Shape &s, F f) {
    if (s.dtype == HILBERTA_FP32) return f(float{}, float{});
    if (s.weight_dtype == HILBERTA_BF16) return f(__nv_bfloat16{}, __nv_bfloat16{});
    return f(__nv_bfloat16{}, float{});
}

template <class T, class W, int VEC, int LANES, int NV>
int launch_forward(const ForwardParams &prm, bool overlap, cudaStream_t stream) {
    constexpr int THREADS = LANES > 32 ? LANES : 128, ROWS = THREADS / LANES;
    const long long blocks = (prm.rows + ROWS - 1) / ROWS;
    if (blocks > 0x7fffffffll) return HILBERTA_ERR_UNSUPPORTED;
    HB_CUDA(launch_overlapping(layer_norm_kernel<T, W, VEC, LANES, NV>, (unsigned)blocks, THREADS, 0, 1, stream, overlap, prm));
    HB_LAUNCHED();
    return HILBERTA_OK;
}

// Lanes and vectors per lane by the number of vectors in a row.
template <class T, class W, int VEC>
int forward_by_cols(const ForwardParams &prm, bool overlap, cudaStream_t stream) {
    const int n = (prm.cols + VEC - 1) / VEC;
    if constexpr (VEC > 1) {
        constexpr int U = 8 / VEC;   // fp32 vectors hold half as many values
        if (n <= 8) return launch_forward<T, W, VEC, 8, 1>(prm, overlap, stream);
        if (n <= 32) return launch_forward<T, W, VEC, 32, 1>(prm, overlap, stream);
        if (n <= 64) return launch_forward<T, W, VEC, 32, 2>(prm, overlap, stream);
        if (n <= 128) return launch_forward<T, W, VEC, 32, 4>(prm, overlap, stream);
        if (n <= 192 * U) return launch_forward<T, W, VEC, 32, 6 * U>(prm, overlap, stream);
        if (n <= 512 * U) return launch_forward<T, W, VEC, 128, 4 * U>(prm, overlap, stream);
        if (n <= 1024 * U) return launch_forward<T, W, VEC, 256, 4 * U>(prm, overlap, stream);
        return launch_forward<T, W, VEC, 512, 4 * U>(prm, overlap, stream);
    } else {
        if (n <= 64) return launch_forward<T, W, 1, 32, 2>(prm, overlap, stream);
        if (n <= 256) return launch_forward<T, W, 1, 32, 8>(prm, overlap, stream);
        if (n <= 1024) return launch_forward<T, W, 1, 128, 8>(prm, overlap, stream);
        if (n <= 4096) return launch_forward<T, W, 1, 256, 16>(prm, overlap, stream);
        return launch_forward<T, W, 1, 512, 32>(prm, overlap, stream);
    }
}

// The backward grid.  lanes > 0: that many lanes have a row; else CTAs of `threads` threads with nv vectors each, r rows
// at a time and a ring of `stages` rounds of them.
struct BackwardGrid {
    int lanes, threads, nv, r, stages, pitch;
    long long ctas;   // of a group
};

constexpr int RING_BYTES = 220 << 10;   // shared memory of an SM for the rings of its CTAs

BackwardGrid backward_grid(const Shape &s, int vec, int sms) {
    BackwardGrid g{};
    const int n = (s.cols + vec - 1) / vec;
    long long resident, most;   // CTAs that run at once; those that have rows
    if (n <= 32) {
        g.lanes = n <= 8 ? 8 : 32;
        g.threads = 256;
        g.r = 4;
        resident = (long long)sms * 4;
        most = (s.rows_per_group + g.r * (256 / g.lanes) - 1) / (g.r * (256 / g.lanes));
    } else {
        const int most_nv = 32 / vec;
        for (g.nv = 1; g.nv < most_nv && n > 256 * g.nv; g.nv *= 2) {
        }
        g.threads = std::min(512, ((n + g.nv - 1) / g.nv + 31) / 32 * 32);
        const int per_sm = std::max(1, std::min(4, 640 / g.threads));
        // in rows that are not aligned a granule more
        g.pitch = (int)((s.cols * s.esz + 15) / 16 * 16) + (vec == 1 ? 16 : 0);
        const int budget = RING_BYTES / per_sm - 2048;   // what the kernel has besides, and the system
        g.r = g.nv * vec <= 8 ? 4 : g.nv * vec <= 16 ? 2 : 1;
        while (g.r > 1 && 3 * 2 * g.r * g.pitch > budget) g.r /= 2;
        g.stages = std::max(1, std::min(MAX_STAGES, budget / (2 * g.r * g.pitch)));
        resident = (long long)sms * per_sm;
        most = (s.rows_per_group + g.r - 1) / g.r;
    }
    g.ctas = std::max(1ll, std::min(most, resident / std::max(1ll, s.groups)));
    return g;
}

template <class T, class W, int VEC, int NV, int R>
int launch_backward(const BackwardParams &prm, const BackwardGrid &g, long long groups, bool overlap, cudaStream_t stream) {
    const int smem = g.stages * 2 * g.r * g.pitch;
    // the shared-memory opt-in is an attribute of the kernel on one device
    static std::atomic<uint64_t> done{0};
    int dev = -1;
    HB_CUDA(cudaGetDevice(&dev));
    if (!(done.load() >> dev & 1)) {
        HB_CUDA(cudaFuncSetAttribute(layer_norm_bwd_kernel<T, W, VEC, NV, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, RING_BYTES));
        done.fetch_or(1ull << dev);
    }
    HB_CUDA(launch_overlapping(layer_norm_bwd_kernel<T, W, VEC, NV, R>, dim3((unsigned)g.ctas, (unsigned)groups), g.threads, (size_t)smem, 1,
                               stream, overlap, prm));
    HB_LAUNCHED();
    return HILBERTA_OK;
}

template <class T, class W, int VEC, int LANES>
int launch_lanes(const BackwardParams &prm, const BackwardGrid &g, long long groups, bool overlap, cudaStream_t stream) {
    HB_CUDA(launch_overlapping(layer_norm_bwd_lanes_kernel<T, W, VEC, LANES, 4>, dim3((unsigned)g.ctas, (unsigned)groups), 256, 0, 1, stream,
                               overlap, prm));
    HB_LAUNCHED();
    return HILBERTA_OK;
}

template <class T, class W, int VEC, int NV>
int backward_by_rows(const BackwardParams &prm, const BackwardGrid &g, long long groups, bool overlap, cudaStream_t stream) {
    if constexpr (NV * VEC <= 8)
        if (g.r == 4) return launch_backward<T, W, VEC, NV, 4>(prm, g, groups, overlap, stream);
    if constexpr (NV * VEC <= 16)
        if (g.r == 2) return launch_backward<T, W, VEC, NV, 2>(prm, g, groups, overlap, stream);
    return launch_backward<T, W, VEC, NV, 1>(prm, g, groups, overlap, stream);
}

template <class T, class W, int VEC>
int backward_by_cols(const BackwardParams &prm, const BackwardGrid &g, long long groups, bool overlap, cudaStream_t stream) {
    if (g.lanes == 8) return launch_lanes<T, W, VEC, 8>(prm, g, groups, overlap, stream);
    if (g.lanes == 32) return launch_lanes<T, W, VEC, 32>(prm, g, groups, overlap, stream);
    switch (g.nv) {
        case 1: return backward_by_rows<T, W, VEC, 1>(prm, g, groups, overlap, stream);
        case 2: return backward_by_rows<T, W, VEC, 2>(prm, g, groups, overlap, stream);
        case 4: return backward_by_rows<T, W, VEC, 4>(prm, g, groups, overlap, stream);
    }
    if constexpr (VEC <= 4)
        if (g.nv == 8) return backward_by_rows<T, W, VEC, 8>(prm, g, groups, overlap, stream);
    if constexpr (VEC == 1) {
        if (g.nv == 16) return backward_by_rows<T, W, VEC, 16>(prm, g, groups, overlap, stream);
        if (g.nv == 32) return backward_by_rows<T, W, VEC, 32>(prm, g, groups, overlap, stream);
    }
    return HILBERTA_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace hilberta

using namespace hilberta;

extern "C" int hilberta_layer_norm(const void *x, const void *weight, const void *bias, void *y, float *mean, float *rstd,
                                   int64_t rows, int cols, int64_t rows_per_group, int64_t stride_x, int64_t stride_y,
                                   int64_t stride_w, int dtype, int weight_dtype, int unit_offset, float eps, void *stream) {
    Shape s;
    const int rc = check_shape(s, rows, cols, rows_per_group, dtype, weight_dtype);
    if (rc != HILBERTA_OK) return rc;
    if ((rows > 0 && (!x || !y)) || stride_x < 0 || stride_y < cols || !(eps >= 0.f)) return HILBERTA_ERR_INVALID;
    if (((uintptr_t)x | (uintptr_t)y) & (s.esz - 1) || ((uintptr_t)weight | (uintptr_t)bias) & (s.wsz - 1) ||
        ((uintptr_t)mean | (uintptr_t)rstd) & 3)
        return HILBERTA_ERR_INVALID;
    if (s.groups > 1 && (weight || bias) && stride_w < 0) return HILBERTA_ERR_INVALID;
    if (rows_overlap(x, stride_x, y, stride_y, rows, cols, s.esz)) return HILBERTA_ERR_INVALID;
    int dev = -1;
    HB_CUDA(cudaGetDevice(&dev));
    if (!sm100_count(dev)) return HILBERTA_ERR_ARCH;
    if (rows == 0) return HILBERTA_OK;
    ForwardParams prm{x, weight, bias, y, mean, rstd, rows, s.rows_per_group, stride_x, stride_y, s.groups > 1 ? stride_w : 0, cols, eps,
                      unit_offset ? 1.f : 0.f};
    const int vec = (int)(16 / s.esz);
    const bool vectors = cols % vec == 0 && aligned16(x, stride_x, s.esz) && aligned16(y, stride_y, s.esz) &&
                         aligned16(weight, prm.stride_w, s.wsz) && aligned16(bias, prm.stride_w, s.wsz);
    const bool overlap = rows * (long long)cols * (long long)s.esz <= kOverlapBytes;
    return by_types(s, [&](auto t, auto w) {
        using T = decltype(t);
        using W = decltype(w);
        if (vectors) return forward_by_cols<T, W, 16 / (int)sizeof(T)>(prm, overlap, (cudaStream_t)stream);
        return forward_by_cols<T, W, 1>(prm, overlap, (cudaStream_t)stream);
    });
}

extern "C" size_t hilberta_layer_norm_workspace(int64_t rows, int cols, int64_t rows_per_group) {
    Shape s;
    if (check_shape(s, rows, cols, rows_per_group, HILBERTA_FP32, HILBERTA_FP32) != HILBERTA_OK) return 0;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    const int sms = sm100_count(dev);
    size_t most = 0;
    for (size_t esz : {2, 4})   // whatever the type and the alignment
        for (int vec : {1, (int)(16 / esz)}) {
            s.esz = esz;
            const BackwardGrid g = backward_grid(s, vec, sms);
            if (g.ctas > 1) most = std::max(most, (size_t)(g.ctas * s.groups) * 2 * (size_t)cols * sizeof(float));
        }
    return most;
}

extern "C" int hilberta_layer_norm_backward(const void *dy, const void *x, const void *weight, const float *mean,
                                            const float *rstd, void *dx, void *dweight, void *dbias, void *workspace,
                                            size_t workspace_bytes, int64_t rows, int cols, int64_t rows_per_group,
                                            int64_t stride_dy, int64_t stride_x, int64_t stride_dx, int64_t stride_w,
                                            int64_t stride_dw, int dtype, int weight_dtype, int unit_offset, void *stream) {
    Shape s;
    const int rc = check_shape(s, rows, cols, rows_per_group, dtype, weight_dtype);
    if (rc != HILBERTA_OK) return rc;
    if (rows > 0 && (!dy || !x || !mean || !rstd || (!dx && !dweight && !dbias))) return HILBERTA_ERR_INVALID;
    if (stride_dy < 0 || stride_x < 0 || (dx && stride_dx < cols)) return HILBERTA_ERR_INVALID;
    if (s.groups > 1 && ((weight && stride_w < 0) || ((dweight || dbias) && stride_dw < cols))) return HILBERTA_ERR_INVALID;
    if (((uintptr_t)dy | (uintptr_t)x | (uintptr_t)dx) & (s.esz - 1) ||
        ((uintptr_t)weight | (uintptr_t)dweight | (uintptr_t)dbias) & (s.wsz - 1) || ((uintptr_t)mean | (uintptr_t)rstd | (uintptr_t)workspace) & 3)
        return HILBERTA_ERR_INVALID;
    if (rows_overlap(dx, stride_dx, x, stride_x, rows, cols, s.esz) || rows_overlap(dx, stride_dx, dy, stride_dy, rows, cols, s.esz))
        return HILBERTA_ERR_INVALID;
    if (s.groups > 65535) return HILBERTA_ERR_UNSUPPORTED;
    int dev = -1;
    HB_CUDA(cudaGetDevice(&dev));
    const int sms = sm100_count(dev);
    if (!sms) return HILBERTA_ERR_ARCH;
    cudaStream_t st = (cudaStream_t)stream;
    if (rows == 0) {
        // no row: one group without rows, whose sums are zero
        if (dweight) HB_CUDA(cudaMemsetAsync(dweight, 0, (size_t)cols * s.wsz, st));
        if (dbias) HB_CUDA(cudaMemsetAsync(dbias, 0, (size_t)cols * s.wsz, st));
        return HILBERTA_OK;
    }
    const bool one = s.groups == 1;
    BackwardParams prm{dy, x, weight, mean, rstd, dx, dweight, dbias, nullptr, rows, s.rows_per_group, stride_dy, stride_x, stride_dx,
                       one ? 0 : stride_w, one ? 0 : stride_dw, cols, unit_offset ? 1.f : 0.f, 0, 0};
    const int vec = (int)(16 / s.esz);
    const bool vectors = cols % vec == 0 && aligned16(dy, stride_dy, s.esz) && aligned16(x, stride_x, s.esz) && aligned16(dx, stride_dx, s.esz) &&
                         aligned16(weight, prm.stride_w, s.wsz) && aligned16(dweight, prm.stride_dw, s.wsz) &&
                         aligned16(dbias, prm.stride_dw, s.wsz);
    BackwardGrid g = backward_grid(s, vectors ? vec : 1, sms);
    prm.stages = g.stages;
    prm.pitch = g.pitch;
    const bool sums = (dweight || dbias) && g.ctas > 1;
    if (sums) {
        if (!workspace || workspace_bytes < (size_t)(g.ctas * s.groups) * 2 * (size_t)cols * sizeof(float)) return HILBERTA_ERR_BUFFER;
        prm.partial = (float *)workspace;
    }
    const bool overlap = rows * (long long)cols * (long long)s.esz <= kOverlapBytes;
    return by_types(s, [&](auto t, auto w) {
        using T = decltype(t);
        using W = decltype(w);
        const int rc2 = vectors ? backward_by_cols<T, W, 16 / (int)sizeof(T)>(prm, g, s.groups, overlap, st)
                                : backward_by_cols<T, W, 1>(prm, g, s.groups, overlap, st);
        if (rc2 != HILBERTA_OK || !sums) return rc2;
        HB_CUDA(launch_overlapping(layer_norm_sums_kernel<W>, dim3((unsigned)((cols + 31) / 32), (unsigned)s.groups, 2), 32 * SUMS, 0, 1, st,
                                   true, (const float *)prm.partial, prm.dweight, prm.dbias, cols, (int)g.ctas, (long long)prm.stride_dw));
        HB_LAUNCHED();
        return HILBERTA_OK;
    });
}
