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
};

// A CTA's threads cover the columns (NV vectors of VEC each), so that the sums over rows stay in registers:
// 2 NV VEC of them.  It takes R rows at a time: R is what keeps enough loads in flight, and one barrier serves the
// 2 R sums over columns.  CTA (i, group) has rows i R ... of the group, then those gridDim.x R further on.
template <class T, class W, int VEC, int NV, int R>
__global__ void __launch_bounds__(VEC > 1 ? 512 : 1024)
layer_norm_bwd_kernel(const BackwardParams prm) {
    __shared__ float part[2][32][2 * R];
    const int cols = prm.cols, warps = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const long long row_begin = (long long)blockIdx.y * prm.rows_per_group;
    const long long row_end = min(row_begin + prm.rows_per_group, prm.rows);
    const float inv_cols = 1.f / (float)cols;
    float dw[NV * VEC] = {}, db[NV * VEC] = {};
    Vec<W, VEC> w[NV];
    allow_next();
    wait_for_previous();
    bool in[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * (int)blockDim.x + (int)threadIdx.x) * VEC;
        in[i] = c < cols;
        if (in[i] && prm.weight) w[i].load((const W *)prm.weight + blockIdx.y * prm.stride_w + c);
    }
    auto weight = [&](int i, int e) { return prm.weight ? w[i].get(e) + prm.offset : 1.f; };
    int k = 0;
    for (long long r0 = row_begin + (long long)blockIdx.x * R; r0 < row_end; r0 += (long long)gridDim.x * R, k ^= 1) {
        Vec<T, VEC> x[R][NV], dy[R][NV];
        float mean[R], rstd[R], s[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool live = r0 + r < row_end;
            mean[r] = live ? prm.mean[r0 + r] : 0.f;
            rstd[r] = live ? prm.rstd[r0 + r] : 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * (int)blockDim.x + (int)threadIdx.x) * VEC;
                if (live && in[i]) {
                    x[r][i].load((const T *)prm.x + (r0 + r) * prm.stride_x + c);
                    dy[r][i].load((const T *)prm.dy + (r0 + r) * prm.stride_dy + c);
                } else {
                    x[r][i].zero();
                    dy[r][i].zero();
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float a = 0.f, b = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (!in[i]) continue;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float d = dy[r][i].get(e), n = (x[r][i].get(e) - mean[r]) * rstd[r];
                    const float g = d * weight(i, e);
                    a += g;
                    b = fmaf(g, n, b);
                    dw[i * VEC + e] = fmaf(d, n, dw[i * VEC + e]);
                    db[i * VEC + e] += d;
                }
            }
            s[2 * r] = a;
            s[2 * r + 1] = b;
        }
        if (prm.dx) {
            // part[k] was last read two rounds ago, before the barrier of the round between
#pragma unroll
            for (int j = 0; j < 2 * R; ++j) s[j] = lanes_sum<32>(s[j]);
            if (lane == 0) {
#pragma unroll
                for (int j = 0; j < 2 * R; ++j) part[k][warp][j] = s[j];
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 2 * R; ++j) s[j] = 0.f;
            for (int q = 0; q < warps; ++q)
#pragma unroll
                for (int j = 0; j < 2 * R; ++j) s[j] += part[k][q][j];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (r0 + r >= row_end) continue;
                const float a = s[2 * r] * inv_cols, b = s[2 * r + 1] * inv_cols;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    if (!in[i]) continue;
                    float f[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float n = (x[r][i].get(e) - mean[r]) * rstd[r];
                        f[e] = rstd[r] * (dy[r][i].get(e) * weight(i, e) - a - n * b);
                    }
                    Vec<T, VEC> o;
                    o.set(f);
                    o.store((T *)prm.dx + (r0 + r) * prm.stride_dx + (i * (int)blockDim.x + (int)threadIdx.x) * VEC);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * (int)blockDim.x + (int)threadIdx.x) * VEC;
        if (!in[i]) continue;
        if (prm.partial) {
            float *p = prm.partial + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 2 * cols + c;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                p[e] = dw[i * VEC + e];
                p[cols + e] = db[i * VEC + e];
            }
        } else {
            Vec<W, VEC> o;
            if (prm.dweight) {
                o.set(dw + i * VEC);
                o.store((W *)prm.dweight + blockIdx.y * prm.stride_dw + c);
            }
            if (prm.dbias) {
                o.set(db + i * VEC);
                o.store((W *)prm.dbias + blockIdx.y * prm.stride_dw + c);
            }
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
#pragma unroll 4
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

// The backward grid: threads of a CTA, vectors of a thread, rows at a time, CTAs of a group.
struct BackwardGrid {
    int threads, nv, r;
    long long ctas;
};

BackwardGrid backward_grid(const Shape &s, int vec, int sms) {
    BackwardGrid g;
    const int n = (s.cols + vec - 1) / vec;
    g.nv = 1;
    while (n > g.nv * (vec > 1 ? 512 : 1024)) g.nv *= 2;
    g.threads = ((n + g.nv - 1) / g.nv + 31) / 32 * 32;
    g.r = g.nv == 1 ? 4 : g.nv == 2 ? 2 : 1;
    const long long resident = (long long)sms * std::max(1, 1024 / g.threads);
    const long long most = (s.rows_per_group + g.r - 1) / g.r;   // a round of rows each at least
    g.ctas = std::max(1ll, std::min(most, resident / std::max(1ll, s.groups)));
    return g;
}

template <class T, class W, int VEC, int NV, int R>
int launch_backward(const BackwardParams &prm, const BackwardGrid &g, long long groups, bool overlap, cudaStream_t stream) {
    HB_CUDA(launch_overlapping(layer_norm_bwd_kernel<T, W, VEC, NV, R>, dim3((unsigned)g.ctas, (unsigned)groups), g.threads, 0, 1,
                               stream, overlap, prm));
    HB_LAUNCHED();
    return HILBERTA_OK;
}

template <class T, class W, int VEC>
int backward_by_cols(const BackwardParams &prm, const BackwardGrid &g, long long groups, bool overlap, cudaStream_t stream) {
    switch (g.nv) {
        case 1: return launch_backward<T, W, VEC, 1, 4>(prm, g, groups, overlap, stream);
        case 2: return launch_backward<T, W, VEC, 2, 2>(prm, g, groups, overlap, stream);
        case 4: return launch_backward<T, W, VEC, 4, 1>(prm, g, groups, overlap, stream);
        case 8:   // 16-bit vectors get by with four
            if constexpr (VEC < 8) return launch_backward<T, W, VEC, 8, 1>(prm, g, groups, overlap, stream);
            return HILBERTA_ERR_UNSUPPORTED;
        default:
            if constexpr (VEC == 1) return launch_backward<T, W, 1, 16, 1>(prm, g, groups, overlap, stream);
            return HILBERTA_ERR_UNSUPPORTED;
    }
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
    for (int vec : {1, 4, 8}) {
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
                       one ? 0 : stride_w, one ? 0 : stride_dw, cols, unit_offset ? 1.f : 0.f};
    const int vec = (int)(16 / s.esz);
    const bool vectors = cols % vec == 0 && aligned16(dy, stride_dy, s.esz) && aligned16(x, stride_x, s.esz) && aligned16(dx, stride_dx, s.esz) &&
                         aligned16(weight, prm.stride_w, s.wsz) && aligned16(dweight, prm.stride_dw, s.wsz) &&
                         aligned16(dbias, prm.stride_dw, s.wsz);
    BackwardGrid g = backward_grid(s, vectors ? vec : 1, sms);
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
