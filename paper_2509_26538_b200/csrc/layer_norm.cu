// Layer norm over the last axis and its gradients, for the norms in front of a transformer block's
// projections: affine, or modulated by one scale and shift per sample (adaptive layer norm).
//
//   mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),  n = (x - mean) rstd,  y = n w + b
//   g = dy w:   dx = rstd (g - sum g / C - n sum(g n) / C),   dw = sum_rows dy n,   db = sum_rows dy
//
// Both directions are bound by HBM: every element is read once (twice as many streams backward) and written
// once.  A row stays in registers between its statistics and its output; sums are fp32, the variance is taken
// around the mean that has already been summed (no difference of large squares).
// Measured (B200, us; share of the copy bandwidth).  Forward: 33792 x 1536 bf16, modulated 40 (79 %), 40000 x 1024 bf16 29 (85 %),
// 12000 x 4096 fp32 63 (95 %): what is left in bf16 is unpacking and packing on the integer pipe, half busy.  Backward: 40000 x
// 1024 bf16 46 (82 %), 36864 x 1152 bf16 52 (75 %), 12000 x 4096 fp32 97 (93 %), 3000 x 16000 bf16 96 (46 %: a row at a time, 15
// warps and one barrier a row), of which 5 ... 7 add the CTAs' sums up; rows that are not aligned, or whose columns are no multiple of
// a vector (of eight backward, whatever the type), take elements one by one (30000 x 1001 bf16 forward 47, backward 66: 39 and 42 %).
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace hilberta {
namespace {

constexpr int MAX_COLS = 16384;

__device__ int g_status[64];   // [0]: code of the first wait that gave up

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
        } else if constexpr (BYTES == 8) {
            const uint2 v = *reinterpret_cast<const uint2 *>(p);
            w[0] = v.x, w[1] = v.y;
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
    // elements 2 i and 2 i + 1; of a single element the second is zero
    __device__ __forceinline__ float2 pair(int i) const {
        if constexpr (VEC == 1) return make_float2(get(0), 0.f);
        else return make_float2(get(2 * i), get(2 * i + 1));
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
        } else if constexpr (BYTES == 8) {
            *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        } else if constexpr (BYTES == 4) {
            *reinterpret_cast<uint32_t *>(p) = w[0];
        } else {
            *reinterpret_cast<uint16_t *>(p) = (uint16_t)w[0];
        }
    }
};

// Two elements at a time: Blackwell's packed fp32 instructions, which halve the arithmetic of these kernels (a single
// element has the other half idle).
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
template <int VEC>
constexpr int PAIRS = (VEC + 1) / 2;

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
    // Vectors of one element go through the arithmetic two by two.
    constexpr int STEP = VEC > 1 ? 1 : 2, P = VEC > 1 ? VEC / 2 : 1;   // vectors and pairs at a time
    static_assert(NV % STEP == 0, "single elements come in pairs");
    auto col = [&](int i) { return (i * LANES + lane) * VEC; };
    Vec<T, VEC> v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (in && col(i) < cols) v[i].load(x + col(i));
        else v[i].zero();
    }
    // unpacked once: in bf16 that is what the integer pipe, the busiest one, spends its time on
    float2 d[NV / STEP * P], acc[2] = {both(0.f), both(0.f)};   // two chains
#pragma unroll
    for (int i = 0; i < NV; i += STEP)
#pragma unroll
        for (int e = 0; e < P; ++e) {
            float2 &at = d[i / STEP * P + e];
            at = VEC > 1 ? v[i].pair(e) : make_float2(v[i].get(0), v[(i + 1) % NV].get(0));
            acc[(i + e) & 1] = __fadd2_rn(acc[(i + e) & 1], at);
        }
    acc[0] = __fadd2_rn(acc[0], acc[1]);
    const float mean = row_sum(acc[0].x + acc[0].y, 0) / (float)cols;
    const float2 shift = both(-mean);
    acc[0] = acc[1] = both(0.f);
#pragma unroll
    for (int i = 0; i < NV; i += STEP) {
        if (col(i) < cols) {
#pragma unroll
            for (int e = 0; e < P; ++e) {
                float2 &at = d[i / STEP * P + e];
                at = __fadd2_rn(at, shift);
                if (VEC == 1 && col(i + 1) >= cols) at.y = 0.f;
                acc[(i + e) & 1] = __ffma2_rn(at, at, acc[(i + e) & 1]);
            }
        }
    }
    acc[0] = __fadd2_rn(acc[0], acc[1]);
    const float rstd = 1.f / sqrtf(row_sum(acc[0].x + acc[0].y, 1) / (float)cols + prm.eps);
    if (!in) return;
    if (lane == 0) {
        if (prm.mean) prm.mean[row] = mean;
        if (prm.rstd) prm.rstd[row] = rstd;
    }
    const long long group = prm.rows_per_group >= prm.rows ? 0 : row / prm.rows_per_group;
    const W *w = prm.weight ? (const W *)prm.weight + group * prm.stride_w : nullptr;
    const W *b = prm.bias ? (const W *)prm.bias + group * prm.stride_w : nullptr;
    T *y = (T *)prm.y + row * prm.stride_y;
    const float2 scale = both(rstd), offset = both(prm.offset);
    auto weights = [&](float2 *to, const W *from, int i) {
        Vec<W, VEC> t;
        t.load(from + col(i));
#pragma unroll
        for (int e = 0; e < P; ++e) to[e] = t.pair(e);
        if (VEC == 1 && col(i + 1) < cols) {
            t.load(from + col(i + 1));
            to[0].y = t.get(0);
        }
    };
#pragma unroll
    for (int i = 0; i < NV; i += STEP) {
        if (col(i) >= cols) continue;
        float2 f[P], t[P];
#pragma unroll
        for (int e = 0; e < P; ++e) f[e] = __fmul2_rn(d[i / STEP * P + e], scale);
        if (w) {
            weights(t, w, i);
#pragma unroll
            for (int e = 0; e < P; ++e) f[e] = __fmul2_rn(f[e], __fadd2_rn(t[e], offset));
        }
        if (b) {
            weights(t, b, i);
#pragma unroll
            for (int e = 0; e < P; ++e) f[e] = __fadd2_rn(f[e], t[e]);
        }
        float out[2 * P];
#pragma unroll
        for (int e = 0; e < P; ++e) out[2 * e] = f[e].x, out[2 * e + 1] = f[e].y;
        Vec<T, VEC> o;
        o.set(out);
        o.store(y + col(i));
        if (VEC == 1 && col(i + 1) < cols) {
            o.set(out + 1);
            o.store(y + col(i + 1));
        }
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
    int team_warps;      // warps that share a row
    int stages, pitch;   // of the ring in shared memory
};

// weights as the gradients use them: w [+ 1], 1 without any
template <class W, int VEC>
__device__ __forceinline__ void load_weights(float2 *w, const W *p, bool given, float offset) {
    Vec<W, VEC> v;
    v.zero();
    if (given) v.load(p);
#pragma unroll
    for (int e = 0; e < PAIRS<VEC>; ++e) w[e] = given ? __fadd2_rn(v.pair(e), both(offset)) : both(1.f);
}

// (x - mean) rstd: the difference first: with a mean far from zero, x rstd - mean rstd would lose what they share.
__device__ __forceinline__ float2 normalised(float2 x, float mean, float2 scale) { return __fmul2_rn(__fadd2_rn(x, both(-mean)), scale); }

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

// The ring's bounded wait.  One that gives up leaves its code in the status, and the CTA's other waits give up soon after it.
// TRIES: it counts tries and has no clock, whose registers cost the kernel of two 16-byte bf16 vectors a thread and one row at a
// time 7 ... 9 % (5120 and 6656 columns; 1 % so); the others are up to 10 % faster with the clock (10000 ... 14000 columns).
template <bool TRIES>
__device__ __forceinline__ bool ring_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, int code) {
    if constexpr (!TRIES) return ptx::wait_or_abort(bar, parity, abort_flag, g_status, code);
    if (ptx::mbar_try_wait(bar, parity)) return true;
#pragma unroll 1
    for (int i = 0; *abort_flag == 0 && i < (1 << 22); ++i)
        if (ptx::mbar_try_wait(bar, parity)) return true;
    *abort_flag = 1;
    atomicCAS(g_status, 0, code);
    return false;
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
    constexpr int P = PAIRS<VEC>;
    float2 dw[P] = {}, db[P] = {}, w[P];
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
            const float2 scale = both(rstd[r]);
            float2 n[P], g[P], a2 = both(0.f), b2 = both(0.f);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const float2 d = dy[r].pair(e);
                n[e] = normalised(x[r].pair(e), mean[r], scale);
                g[e] = __fmul2_rn(d, w[e]);
                if (in) {
                    a2 = __fadd2_rn(a2, g[e]);
                    b2 = __ffma2_rn(g[e], n[e], b2);
                    dw[e] = __ffma2_rn(d, n[e], dw[e]);
                    db[e] = __fadd2_rn(db[e], d);
                }
            }
            const float a = -rstd[r] * (lanes_sum<LANES>(a2.x + a2.y) * inv_cols), b = -rstd[r] * (lanes_sum<LANES>(b2.x + b2.y) * inv_cols);
            if (prm.dx && in && r0 + r < row_end) {
                Vec<T, VEC> o;
                float f[2 * P];
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const float2 d = __ffma2_rn(g[e], scale, __ffma2_rn(n[e], both(b), both(a)));
                    f[2 * e] = d.x;
                    f[2 * e + 1] = d.y;
                }
                o.set(f);
                o.store((T *)prm.dx + (r0 + r) * prm.stride_dx + c);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < P; ++e) {
        part[0][team][c + 2 * e] = dw[e].x;
        part[1][team][c + 2 * e] = db[e].x;
        if (VEC > 1) {
            part[0][team][c + 2 * e + 1] = dw[e].y;
            part[1][team][c + 2 * e + 1] = db[e].y;
        }
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

// Longer rows: a team of `warps` warps has a row, a CTA several teams, R rows each at a time.  They come through a ring of
// shared memory that a warp of its own fills with bulk copies, rounds ahead (a register's worth of loads ahead left HBM
// idle at the barrier that the two row sums need; filling from a computing warp cost more than the warp), and are read
// from there twice, for the sums and for dx.  Rows that lie one
// behind the other are one copy.  A row that does not start on a 16-byte boundary is copied from the boundary before to the
// one behind: the granules are those of its own first and last elements.  Columns behind the row's end count as zeros.
constexpr int MAX_STAGES = 4, MAX_ROWS = 16, MAX_WARPS = 16;
template <class T, class W, int VEC, int NV, int R>
__global__ void __launch_bounds__(NV * VEC <= 16 ? 32 * (MAX_WARPS + 1) : 32 * MAX_WARPS)
layer_norm_bwd_kernel(const BackwardParams prm) {
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ __align__(16) float part[2][MAX_WARPS][2 * R];
    __shared__ __align__(16) float2 stats[MAX_STAGES][MAX_ROWS];   // -mean, rstd of a stage's rows
    __shared__ uint64_t full[MAX_STAGES], empty[MAX_STAGES];
    __shared__ int abort_flag;
    constexpr int P = NV * VEC / 2;           // pairs of a thread
    constexpr bool TRIES = VEC == 8 && NV == 2 && R == 1;
    constexpr bool KEEP_W = NV * VEC <= 16;   // weights in registers, else behind the ring
    const int cols = prm.cols, all = (int)blockDim.x / 32 - 1, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int warps = prm.team_warps, teams = all / warps, rows = teams * R;   // rows of a round
    const int stages = prm.stages, pitch = prm.pitch;                          // pitch: bytes of a row in the ring
    const long long row_begin = (long long)blockIdx.y * prm.rows_per_group;
    const long long row_end = min(row_begin + prm.rows_per_group, prm.rows);
    const long long first = row_begin + (long long)blockIdx.x * rows, step = (long long)gridDim.x * rows;
    const int rounds = first < row_end ? (int)((row_end - first + step - 1) / step) : 0;
    const uint32_t full0 = ptx::smem_u32(full), empty0 = ptx::smem_u32(empty);
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int i = 0; i < stages; ++i) {
            ptx::mbar_init(full0 + 8 * i, 1);
            ptx::mbar_init(empty0 + 8 * i, all);
        }
        ptx::mbar_fence_init();
    }
    allow_next();
    wait_for_previous();
    __syncthreads();
    if (warp == all) {
        // ------------------------------------------------ fills the ring: x, dy and the statistics of each round's rows
        // lane r < rows is for row r of x, lane rows + r for row r of dy; where a tensor's rows lie one behind the other
        // its first lane copies them all
        const bool of_x = lane < rows;
        const int r = of_x ? lane : lane - rows;
        const long long stride = of_x ? prm.stride_x : prm.stride_dy;
        const bool dense = VEC > 1 && stride == cols;
        const T *src = (const T *)(of_x ? prm.x : prm.dy) + (first + r) * stride;
        for (int i = 0; i < rounds; ++i, src += step * stride) {
            const int s = i % stages;
            const long long r0 = first + i * step;
            const int live = (int)min((long long)rows, row_end - r0);
            const bool mine = r < live;
            const float value = mine ? (of_x ? prm.mean : prm.rstd)[r0 + r] : 0.f;
            if (!__all_sync(0xffffffffu, ring_wait<TRIES>(empty0 + 8 * s, ((i / stages) & 1) ^ 1, &abort_flag, 0x700))) break;
            if (r < rows) (of_x ? stats[s][r].x : stats[s][r].y) = of_x ? -value : value;
            const uintptr_t at = (uintptr_t)src, from = at & ~(uintptr_t)15;
            uint32_t bytes = mine ? (uint32_t)(((at + (size_t)cols * sizeof(T) + 15) & ~(uintptr_t)15) - from) : 0u;
            if (dense) bytes = r == 0 ? bytes * live : 0u;
            const uint32_t sum = __reduce_add_sync(0xffffffffu, bytes);
            __syncwarp();   // all lanes' statistics come before lane 0's arrival
            if (lane == 0) ptx::mbar_expect_tx(full0 + 8 * s, sum);
            __syncwarp();
            if (bytes) bulk_load(ptx::smem_u32(ring) + (uint32_t)((s * 2 * rows + lane) * pitch), (const void *)from, bytes, full0 + 8 * s);
        }
    }
    const int team = warp / warps, threads = 32 * warps, tid = (warp - team * warps) * 32 + lane;
    const W *weight = prm.weight ? (const W *)prm.weight + blockIdx.y * prm.stride_w : nullptr;
    W *const kept = reinterpret_cast<W *>(ring + prm.stages * 2 * rows * pitch);
    const float inv_cols = 1.f / (float)cols;
    float2 dw[P] = {}, db[P] = {}, w[KEEP_W ? P : (VEC > 1 ? VEC / 2 : 1)];
    // This thread's vector v: its column, and whether there is one.  A warp's vectors lie side by side, at distances that the
    // compiler knows (up to 36 registers otherwise, whose spills come back from L2: 3000 x 10001 bf16 250 us, 83 so; 12000 x
    // 4096 fp32 102 and 97; 30000 x 1001 bf16 79 and 66), but the team's where few vectors are of 8 bytes or single fp32 elements
    // (36864 x 1152 bf16 79 us with a warp's side by side, 52 so; 3 x 1777 x 777 fp32 20 and 17.7).
    constexpr bool NEAR = !KEEP_W || VEC * sizeof(T) >= 16 || VEC * sizeof(T) == 2;
    const int apart = NEAR ? 32 * VEC : threads * VEC;
    const int col0 = (NEAR ? tid / 32 * NV * 32 + lane : tid) * VEC, after = cols - col0;
    auto col = [&](int v) { return col0 + v * apart; };
    auto has = [&](int v) { return v * apart < after; };
    // pairs of vector v (VEC > 1) or of elements v and v + 1 (VEC = 1), zeros behind the row's end
    auto load_pairs = [&](float2 *to, const auto *row, int v) {
        using E = std::remove_cv_t<std::remove_pointer_t<decltype(row)>>;
        if constexpr (VEC > 1) {
            Vec<E, VEC> t;
            t.zero();
            if (has(v)) t.load(row + col(v));
#pragma unroll
            for (int e = 0; e < VEC / 2; ++e) to[e] = t.pair(e);
        } else {
            Vec<E, 1> t0, t1;
            t0.zero();
            t1.zero();
            if (has(v)) t0.load(row + col(v));
            if (has(v + 1)) t1.load(row + col(v + 1));
            to[0] = make_float2(t0.get(0), t1.get(0));
        }
    };
    constexpr int STEP = VEC > 1 ? 1 : 2, PV = VEC > 1 ? VEC / 2 : 1;   // vectors and pairs at a time
    auto load_w = [&](float2 *to, int v) {
        if (weight) {
            load_pairs(to, KEEP_W ? weight : (const W *)kept, v);
#pragma unroll
            for (int e = 0; e < PV; ++e) to[e] = __fadd2_rn(to[e], both(prm.offset));
        } else {
#pragma unroll
            for (int e = 0; e < PV; ++e) to[e] = both(1.f);
        }
    };
    if (warp < all && KEEP_W) {
#pragma unroll
        for (int v = 0; v < NV; v += STEP) load_w(w + v / STEP * PV, v);
    }
    if (warp < all && !KEEP_W && weight) {   // a thread's own columns, for itself
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            Vec<W, VEC> t;
            if (has(v)) t.load(weight + col(v)), t.store(kept + col(v));
        }
    }
    // VEC = 1: where a row starts within its granule
    const T *x0 = (const T *)prm.x + (first + team * R) * prm.stride_x, *dy0 = (const T *)prm.dy + (first + team * R) * prm.stride_dy;
    T *dx = prm.dx ? (T *)prm.dx + (first + team * R) * prm.stride_dx : nullptr;
    const uint8_t *const mine = ring + team * R * pitch;
    const int to_dy = rows * pitch;
    int s = 0, phase = 0;
    for (int i = 0; warp < all && i < rounds; ++i) {
        const int left = (int)min((long long)R, row_end - first - i * step - team * R);   // rows of the team in this round
        const uint8_t *const base = mine + s * 2 * to_dy;
        auto row_x = [&](int r) { return (const T *)(base + r * pitch + (VEC == 1 ? (int)((uintptr_t)(x0 + r * prm.stride_x) & 15) : 0)); };
        auto row_dy = [&](int r) { return (const T *)(base + to_dy + r * pitch + (VEC == 1 ? (int)((uintptr_t)(dy0 + r * prm.stride_dy) & 15) : 0)); };
        // a warp whose wait gives up goes on, through the barriers that the team's other warps are at; its next ones give up soon
        ring_wait<TRIES>(full0 + 8 * s, phase, &abort_flag, 0x701);
        float2 st[R];
        float sum[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float2 a = both(0.f), b = both(0.f);
            st[r] = stats[s][team * R + r];
            if (r < left) {
                const float2 shift = both(st[r].x), scale = both(st[r].y);
                const T *px = row_x(r), *pd = row_dy(r);
#pragma unroll
                for (int v = 0; v < NV; v += STEP) {
                    float2 x[PV], dy[PV];
                    float2 *const wv = KEEP_W ? w + v / STEP * PV : w;
                    if (!KEEP_W) load_w(wv, v);
                    load_pairs(x, px, v);
                    load_pairs(dy, pd, v);
#pragma unroll
                    for (int e = 0; e < PV; ++e) {
                        const int at = v / STEP * PV + e;
                        const float2 n = __fmul2_rn(__fadd2_rn(x[e], shift), scale), g = __fmul2_rn(dy[e], wv[e]);
                        a = __fadd2_rn(a, g);
                        b = __ffma2_rn(g, n, b);
                        dw[at] = __ffma2_rn(dy[e], n, dw[at]);
                        db[at] = __fadd2_rn(db[at], dy[e]);
                    }
                }
            }
            sum[2 * r] = a.x + a.y;
            sum[2 * r + 1] = b.x + b.y;
        }
        if (dx) {
            // lane 32 j / (2 R) is left with sum j over the warp: each step hands half of the sums over
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
            constexpr int SHARE = 32 / (2 * R);
            // part[k] was last read two rounds ago, before the barrier of the round between
            const int k = i & 1;
            if (lane % SHARE == 0) part[k][warp][lane / SHARE] = sum[0];
            if (warps == 1) __syncwarp();
            else asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(threads) : "memory");   // the team
            float2 total[R];
#pragma unroll
            for (int r = 0; r < R; ++r) total[r] = both(0.f);
            for (int q = 0; q < warps; ++q)
#pragma unroll
                for (int r = 0; r < R; ++r)
                    total[r] = __fadd2_rn(total[r], *reinterpret_cast<const float2 *>(&part[k][team * warps + q][2 * r]));
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (r >= left) continue;
                // rstd (g - a - n b), n = (x - mean) rstd
                const float2 shift = both(st[r].x), scale = both(st[r].y);
                const float2 a = both(-st[r].y * (total[r].x * inv_cols)), b = both(-st[r].y * st[r].y * (total[r].y * inv_cols));
                const T *px = row_x(r), *pd = row_dy(r);
                T *const out = dx + r * prm.stride_dx;
#pragma unroll
                for (int v = 0; v < NV; v += STEP) {
                    float2 x[PV], dy[PV];
                    float f[2 * PV];
                    float2 *const wv = KEEP_W ? w + v / STEP * PV : w;
                    if (!KEEP_W) load_w(wv, v);
                    load_pairs(x, px, v);
                    load_pairs(dy, pd, v);
#pragma unroll
                    for (int e = 0; e < PV; ++e) {
                        const float2 d = __ffma2_rn(__fmul2_rn(dy[e], wv[e]), scale, __ffma2_rn(__fadd2_rn(x[e], shift), b, a));
                        f[2 * e] = d.x;
                        f[2 * e + 1] = d.y;
                    }
                    Vec<T, VEC> o;
                    o.set(f);
                    if (has(v)) o.store(out + col(v));
                    if (VEC == 1 && has(v + 1)) {
                        o.set(f + 1);
                        o.store(out + col(v + 1));
                    }
                }
            }
            dx += step * prm.stride_dx;
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(empty0 + 8 * s);
        if (++s == stages) s = 0, phase ^= 1;
        x0 += step * prm.stride_x;
        dy0 += step * prm.stride_dy;
    }
    if (*(volatile int *)&abort_flag) {
        // let every copy already issued land before the CTA retires
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000) {
        }
    }
    if (!prm.dweight && !prm.dbias) return;
    // the teams' sums one after the other through the ring, team 0 first: the order is always the same
    float2 *const sums = reinterpret_cast<float2 *>(ring);   // [pair][thread], dw then db: they fit (see the host)
    for (int t = 1; t < teams; ++t) {
        __syncthreads();
        if (team == t) {
#pragma unroll
            for (int p = 0; p < P; ++p) sums[p * threads + tid] = dw[p], sums[(P + p) * threads + tid] = db[p];
        }
        __syncthreads();
        if (team == 0) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                dw[p] = __fadd2_rn(dw[p], sums[p * threads + tid]);
                db[p] = __fadd2_rn(db[p], sums[(P + p) * threads + tid]);
            }
        }
    }
    if (team != 0) return;
#pragma unroll
    for (int v = 0; v < NV; v += STEP) {
#pragma unroll
        for (int e = 0; e < PV; ++e) {
            const float2 a = dw[v / STEP * PV + e], b = db[v / STEP * PV + e];
            const int c0 = VEC > 1 ? col(v) + 2 * e : col(v), c1 = VEC > 1 ? c0 + 1 : col(v + 1);
            if (c0 < cols) write_sum<W>(prm, 0, c0, a.x), write_sum<W>(prm, 1, c0, b.x);
            if (c1 < cols) write_sum<W>(prm, 0, c1, a.y), write_sum<W>(prm, 1, c1, b.y);
        }
    }
}

// dw, db of a group: the sums of its CTAs added up in a fixed order.  16 columns a block (64 bytes of each CTA's); SUMS rows of
// threads share the CTAs out: 64 for many, 16 where more would only wait.
constexpr int SUM_COLS = 16;
template <class W, int SUMS>
__global__ void __launch_bounds__(SUM_COLS * SUMS)
layer_norm_sums_kernel(const float *partial, void *dweight, void *dbias, int cols, int ctas, long long stride_dw) {
    __shared__ float part[SUMS][SUM_COLS + 1];
    const int lane = threadIdx.x % SUM_COLS, slot = threadIdx.x / SUM_COLS, which = blockIdx.z;
    const int c = blockIdx.x * SUM_COLS + lane;
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
    // LANES lanes for each column
    constexpr int LANES = SUMS < 32 ? SUMS : 32;
    const int col = threadIdx.x / LANES, k = threadIdx.x % LANES;
    if (col < SUM_COLS) {   // whole warps
        sum = part[k][col];
        if (SUMS > 32) sum += part[k + SUMS / 2][col];
        sum = lanes_sum<LANES>(sum);
        const int out = blockIdx.x * SUM_COLS + col;
        if (k == 0 && out < cols) {
            Vec<W, 1> o;
            o.set(&sum);
            o.store((W *)to + blockIdx.y * stride_dw + out);
        }
    }
}

// Do `rows` rows of cols elements, stride apart, share a byte with as many at b?  (Two slices of one tensor may lie side by side.)
bool slices_overlap(const void *a, const void *b, long long stride, long long rows, int cols, size_t esz) {
    if (!a || !b || rows < 1) return false;
    const uintptr_t lo = std::min((uintptr_t)a, (uintptr_t)b), d = std::max((uintptr_t)a, (uintptr_t)b) - lo;
    const uintptr_t row = (uintptr_t)cols * esz, step = rows > 1 ? (uintptr_t)stride * esz : 0;
    if (rows == 1 || step == 0) return d < row;
    if (d >= (uintptr_t)(rows - 1) * step + row) return false;
    return d % step < row || d % step + row > step;
}

// The rows x cols elements at a (row stride sa) and at b: apart, or the very same rows?  Slices of one buffer (equal strides) may
// lie side by side; the address ranges of others have to be apart.
bool rows_overlap(const void *a, long long sa, const void *b, long long sb, long long rows, int cols, size_t esz) {
    if (!a || !b || rows < 1) return false;
    if (sa == sb || rows == 1) return a != b && slices_overlap(a, b, sa, rows, cols, esz);
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

constexpr int MAX_PER_SM = 8;   // CTAs of the backward kernels on one SM

// One warp waits, with a deadline of 2 million cycles, on a barrier that nothing arrives on.
__global__ void layer_norm_timeout_probe() {
    __shared__ uint64_t never;
    __shared__ int abort_flag;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        ptx::mbar_init(ptx::smem_u32(&never), 1);
        ptx::mbar_fence_init();
    }
    __syncthreads();
    ptx::wait_or_abort(ptx::smem_u32(&never), 0, &abort_flag, g_status, 0x7e57, 2000000ll);
}

// How the backward pass is cut up.  lanes > 0: that many lanes have a row; else teams of `warps` warps, `each` columns a
// thread and r rows at a time.
struct BackwardShape {
    int lanes, warps, teams, each, vec, r, pitch;
    long long round() const { return lanes ? (long long)r * (256 / lanes) : (long long)r * teams; }   // rows of a round
};

BackwardShape backward_shape(const Shape &s, bool aligned) {
    BackwardShape g{};
    if (s.cols <= 256 && (aligned || s.cols <= 32)) {
        g.lanes = s.cols <= 8 * 8 && aligned ? 8 : 32;
        g.r = 4;
        return g;
    }
    // Columns of a thread: with 16-byte vectors multiples of 8 (4 in fp32), with 8-byte ones of 4.  The fewest idle slots,
    // then the fewest columns, 8 at least.  More than 16 take 128 registers a thread, which 16 warps with the one that fills the
    // ring can have (17 have 96).
    long long best = -1;
    const int full = aligned ? (int)(16 / s.esz) : 1;
    const bool wide = s.cols > MAX_WARPS * 32 * 16;
    const int most = wide ? 36 : 16;
    for (int warps = wide ? MAX_WARPS - 1 : MAX_WARPS; warps >= 1; --warps)
        for (int vec = full; vec >= std::min(full, 4); vec /= 2) {
            const int unit = std::max(vec, 4), each = (s.cols + 32 * warps * unit - 1) / (32 * warps * unit) * unit;
            if (each > most || (each < 8 && s.cols >= 8 * 32)) continue;
            const long long cost = (long long)each * 32 * warps;
            if (best < 0 || cost < best) {
                best = cost;
                g.warps = warps;
                g.each = each;
                g.vec = vec;
            }
        }
    g.r = g.each <= 8 ? 4 : g.each <= 16 ? 2 : 1;
    g.pitch = (int)((s.cols * s.esz + 15) / 16 * 16) + (aligned ? 0 : 16);
    // Teams: eight computing warps a CTA, sixteen where elements come one by one (40000 x 1024 bf16, us: 1 team of 4 warps 50.2,
    // 2 teams 47.9; 30000 x 1001 bf16 2 teams 93, 4 teams 62.8), but one team of an odd number of warps (36864 x 1152 bf16: 3 warps
    // 58.8, twice 3 71.6).
    g.teams = g.warps & (g.warps - 1) ? 1 : std::max(1, std::min((aligned ? 8 : 16) / g.warps, MAX_ROWS / g.r));
    // Three rounds of the ring in half of an SM, in all of it for a CTA that fills the SM anyway (12000 x 4096 fp32, us: 2 CTAs of
    // one row at a time 118, 1 CTA of two rows 98).
    const int limit = (wide || g.warps == MAX_WARPS ? 200 : 110) << 10;
    while (g.r > 1 && 3 * 2 * g.r * g.teams * g.pitch > limit) g.r /= 2;
    while (g.teams > 1 && 3 * 2 * g.r * g.teams * g.pitch > limit) --g.teams;
    return g;
}

// A call on its way: what the launchers below need and find out.
struct BackwardCall {
    BackwardParams prm;
    BackwardShape g;
    long long groups, rows_per_group;
    bool overlap, sums;        // sums: dweight or dbias are wanted
    void *workspace;
    size_t workspace_bytes;
    int device, sms;
    cudaStream_t stream;
    long long ctas;            // of a group
};

// As many CTAs as run at once, shared out over the groups, none without a round of rows.
int place(BackwardCall &c, int per_sm) {
    const long long most = (c.rows_per_group + c.g.round() - 1) / c.g.round();
    c.ctas = std::max(1ll, std::min(most, (long long)c.sms * std::min(per_sm, MAX_PER_SM) / std::max(1ll, c.groups)));
    c.sums = c.sums && c.ctas > 1;
    if (c.sums) {
        if (!c.workspace || c.workspace_bytes < (size_t)(c.ctas * c.groups) * 2 * (size_t)c.prm.cols * sizeof(float)) return HILBERTA_ERR_BUFFER;
        c.prm.partial = (float *)c.workspace;
    }
    return HILBERTA_OK;
}

template <class T, class W, int VEC, int NV, int R>
int launch_backward(BackwardCall &c) {
    const BackwardShape &g = c.g;
    const auto kernel = layer_norm_bwd_kernel<T, W, VEC, NV, R>;
    // the shared-memory opt-in is an attribute of the kernel on one device
    static std::atomic<uint64_t> opted{0};
    if (!(opted.load() >> c.device & 1)) {
        HB_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 << 10));
        opted.fetch_or(1ull << c.device);
    }
    const int threads = 32 * (g.warps * g.teams + 1), stage = 2 * g.r * g.teams * g.pitch;
    // rows, and afterwards the sums of a team: NV VEC columns, dw and db, of each of its threads
    const int least = g.teams > 1 ? NV * VEC * 8 * 32 * g.warps : 0;
    const int kept = NV * VEC > 16 && c.prm.weight ? g.pitch / (int)sizeof(T) * (int)sizeof(W) : 0;   // weights behind the ring
    auto ring = [&](int stages) { return std::max(stages * stage + kept, least); };
    // As many CTAs as run at once with three rounds each (the driver's count, asked once for each shape in turn), then
    // more rounds if that costs none.
    static std::atomic<uint64_t> asked{0};   // threads, stage, stages and CTAs of the last answer
    const uint64_t key = (uint64_t)threads << 40 | (uint64_t)stage << 8 | (kept ? 1ull << 63 : 0);
    uint64_t known = asked.load();
    if ((known & ~0xffull) != key) {
        int stages = std::min(3, std::max(1, ((220 << 10) - kept) / stage)), per_sm = 0, more = 0;
        HB_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, (size_t)ring(stages)));
        if (stages == 3 && ring(4) <= 220 << 10) {
            HB_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&more, kernel, threads, (size_t)ring(4)));
            if (more >= per_sm) stages = 4;
        }
        known = key | (uint64_t)stages << 4 | (uint64_t)std::max(1, std::min(per_sm, MAX_PER_SM));
        asked.store(known);
    }
    const int stages = (int)(known >> 4 & 15), per_sm = (int)(known & 15);
    c.prm.stages = stages;
    const int rc = place(c, per_sm);
    if (rc != HILBERTA_OK) return rc;
    HB_CUDA(launch_overlapping(kernel, dim3((unsigned)c.ctas, (unsigned)c.groups), threads, (size_t)ring(stages), 1, c.stream, c.overlap, c.prm));
    HB_LAUNCHED();
    return HILBERTA_OK;
}

template <class T, class W, int VEC, int LANES>
int launch_lanes(BackwardCall &c) {
    const int rc = place(c, 4);
    if (rc != HILBERTA_OK) return rc;
    HB_CUDA(launch_overlapping(layer_norm_bwd_lanes_kernel<T, W, VEC, LANES, 4>, dim3((unsigned)c.ctas, (unsigned)c.groups), 256, 0, 1, c.stream,
                               c.overlap, c.prm));
    HB_LAUNCHED();
    return HILBERTA_OK;
}

// The kernels that backward_shape() asks for at some width, type or alignment; no others are built.  (bf16 in vectors of four: what
// vectors of eight leave out.)
template <class T>
constexpr bool reached(int vec, int each, int r) {
    const bool bf16 = sizeof(T) == 2;
    if (each % vec || (each == 4 && vec > 1) || (bf16 && vec == 4 && each % 8 == 0)) return false;
    switch (each) {
        case 4: return r == 4;
        case 8: return r > 1 || !bf16;
        case 12: return r <= 2;
        case 16: return r == 1 || (r == 2 && bf16);
    }
    return r == 1;
}

template <class T, class W, int VEC, int EACH>
int backward_by_rows(BackwardCall &c) {
    if constexpr (reached<T>(VEC, EACH, 4))
        if (c.g.r == 4) return launch_backward<T, W, VEC, EACH / VEC, 4>(c);
    if constexpr (reached<T>(VEC, EACH, 2))
        if (c.g.r == 2) return launch_backward<T, W, VEC, EACH / VEC, 2>(c);
    if constexpr (reached<T>(VEC, EACH, 1))
        if (c.g.r == 1) return launch_backward<T, W, VEC, EACH / VEC, 1>(c);
    return HILBERTA_ERR_UNSUPPORTED;
}

template <class T, class W, int VEC>
int backward_by_each(BackwardCall &c) {
    switch (c.g.each) {
        case 4: return backward_by_rows<T, W, VEC, 4>(c);
        case 8: return backward_by_rows<T, W, VEC, 8>(c);
        case 12: return backward_by_rows<T, W, VEC, 12>(c);
        case 16: return backward_by_rows<T, W, VEC, 16>(c);
        case 20: return backward_by_rows<T, W, VEC, 20>(c);
        case 24: return backward_by_rows<T, W, VEC, 24>(c);
        case 28: return backward_by_rows<T, W, VEC, 28>(c);
        case 32: return backward_by_rows<T, W, VEC, 32>(c);
        case 36: return backward_by_rows<T, W, VEC, 36>(c);
    }
    return HILBERTA_ERR_UNSUPPORTED;
}

template <class T, class W>
int backward_by_cols(BackwardCall &c, bool aligned) {
    if (c.g.lanes == 8) return launch_lanes<T, W, 8, 8>(c);
    if (c.g.lanes) return aligned ? launch_lanes<T, W, 8, 32>(c) : launch_lanes<T, W, 1, 32>(c);
    if constexpr (sizeof(T) == 2)
        if (c.g.vec == 8) return backward_by_each<T, W, 8>(c);
    return c.g.vec == 4 ? backward_by_each<T, W, 4>(c) : backward_by_each<T, W, 1>(c);
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
    if (mean && mean == rstd) return HILBERTA_ERR_INVALID;
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
    long long ctas = 0;
    for (size_t esz : {2, 4})   // whatever the type and the alignment
        for (bool aligned : {false, true}) {
            s.esz = esz;
            const BackwardShape g = backward_shape(s, aligned);
            ctas = std::max(ctas, std::min((s.rows_per_group + g.round() - 1) / g.round(), (long long)sms * MAX_PER_SM / std::max(1ll, s.groups)));
        }
    return ctas > 1 ? (size_t)(ctas * s.groups) * 2 * (size_t)cols * sizeof(float) : 0;
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
    if (slices_overlap(dweight, dbias, stride_dw, std::max(s.groups, 1ll), cols, s.wsz)) return HILBERTA_ERR_INVALID;
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
                       one ? 0 : stride_w, one ? 0 : stride_dw, cols, unit_offset ? 1.f : 0.f, 0, 0, 0};
    // rows on 16-byte boundaries, in whole groups of eight columns
    const bool vectors = cols % 8 == 0 && aligned16(dy, stride_dy, s.esz) && aligned16(x, stride_x, s.esz) && aligned16(dx, stride_dx, s.esz) &&
                         aligned16(weight, prm.stride_w, s.wsz) && aligned16(dweight, prm.stride_dw, s.wsz) &&
                         aligned16(dbias, prm.stride_dw, s.wsz);
    BackwardCall c{};
    c.g = backward_shape(s, vectors);
    prm.team_warps = c.g.warps;
    prm.pitch = c.g.pitch;
    c.prm = prm;
    c.groups = s.groups;
    c.rows_per_group = s.rows_per_group;
    c.overlap = rows * (long long)cols * (long long)s.esz <= (long long)kOverlapBytes;
    c.sums = dweight || dbias;
    c.workspace = workspace;
    c.workspace_bytes = workspace_bytes;
    c.device = dev;
    c.sms = sms;
    c.stream = st;
    return by_types(s, [&](auto t, auto w) {
        using T = decltype(t);
        using W = decltype(w);
        const int rc2 = backward_by_cols<T, W>(c, vectors);
        if (rc2 != HILBERTA_OK || !c.sums) return rc2;
        const bool many = c.ctas > 128;
        HB_CUDA(launch_overlapping(many ? layer_norm_sums_kernel<W, 64> : layer_norm_sums_kernel<W, 16>,
                                   dim3((unsigned)((cols + SUM_COLS - 1) / SUM_COLS), (unsigned)s.groups, 2), SUM_COLS * (many ? 64 : 16), 0, 1,
                                   st, true, (const float *)c.prm.partial, dweight, dbias, cols, (int)c.ctas, (long long)prm.stride_dw));
        HB_LAUNCHED();
        return HILBERTA_OK;
    });
}

extern "C" int hilberta_layer_norm_status(void) {
    int code = 0;
    HB_CUDA(cudaDeviceSynchronize());
    HB_CUDA(cudaMemcpyFromSymbol(&code, g_status, sizeof(int)));
    if (!code) return HILBERTA_OK;
    const int zero[3] = {0, 0, 0};
    HB_CUDA(cudaMemcpyToSymbol(g_status, zero, sizeof(zero)));
    return HILBERTA_ERR_TIMEOUT;
}

extern "C" int hilberta_selftest_layer_norm_timeout(void *stream) {
    int dev = -1;
    HB_CUDA(cudaGetDevice(&dev));
    if (!sm100_count(dev)) return HILBERTA_ERR_ARCH;
    layer_norm_timeout_probe<<<1, 32, 0, (cudaStream_t)stream>>>();
    HB_CUDA(cudaGetLastError());
    HB_LAUNCHED();
    return HILBERTA_OK;
}
