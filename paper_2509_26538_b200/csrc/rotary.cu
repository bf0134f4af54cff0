// Rotary positions (the step between the QKV projection and Algorithm 1 in the paper's pipeline): every pair
// (a, b) of a head's rotated part turns by the angle position * frequency,
//   a' = f (a cos t - b sin t),   b' = f (a sin t + b cos t),   t = pos[axis(j)] inv_freq[j],
// and the gradient turns back by the same angle.  On its way a row may move between the original and the
// physical token order, which saves the gather before or after.
//
// Bound by HBM: one read and one write of the tensor.  No table of cosines is read: angles are computed in the
// kernel, exactly for any 32-bit position, as fixed-point fractions of a turn (inv_freq / 2 pi as a 64-bit
// fraction; the product with the position wraps where the angle does), once per token and pair for all the heads
// of a thread.  Only the remainder, at most an eighth of a turn, becomes fp32.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "common.cuh"

namespace hilberta {
namespace {

constexpr int MAX_PAIRS = 128;   // head dim <= 256
constexpr int THREADS = 256;

struct Params {
    const void *x;
    void *out;
    const int *positions;     // nullptr: a token's position is its index
    const int *row_map;       // nullptr, or output token -> input token
    int pos_of_source;        // positions belong to the input token (forward), not the output token
    int axes;
    long long pos_stride_b;   // in positions of `axes` integers
    long long xb, xh, xs, ob, oh, os;   // element strides
    int pairs, dim, heads, heads_per_thread, S;
    long long tokens;         // batch * S
    float factor, sign;
    unsigned long long turns[MAX_PAIRS];   // frequency in 2^-64 turns per position
    unsigned char axis[MAX_PAIRS];
};

// cos and sin of pos * turns
__device__ __forceinline__ float2 cos_sin(int pos, unsigned long long turns) {
    const unsigned long long u = (unsigned long long)(long long)pos * turns;
    const unsigned q = (unsigned)((u + (1ull << 61)) >> 62);
    const int r = (int)((long long)(u - ((unsigned long long)q << 62)) >> 32);   // in [-2^29, 2^29): 2^32 a turn
    float s, c;
    sincospif((float)r * (1.f / 2147483648.f), &s, &c);
    if (q & 1) {
        const float t = c;
        c = -s;
        s = t;
    }
    if (q & 2) c = -c, s = -s;
    return make_float2(c, s);
}

template <class T>
struct Chunk {   // 16 bytes
    uint4 v;
    __device__ __forceinline__ float get(int i) const {
        const uint32_t *w = &v.x;
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float((i & 1) ? (w[i >> 1] & 0xffff0000u) : (w[i >> 1] << 16));
    }
    __device__ __forceinline__ void set(const float *f) {
        uint32_t *w = &v.x;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(f[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
    }
};

// Where a thread's tokens lie.
struct Token {
    long long x, out, pos;   // offsets of head 0 and of the positions
    int index;               // the position without a table
};
__device__ __forceinline__ Token locate(const Params &p, long long token, const Divider &per_batch) {
    const unsigned b = per_batch.quotient((unsigned)token);
    const int s = (int)((unsigned)token - b * per_batch.d), from = p.row_map ? __ldg(p.row_map + s) : s;
    const int at = p.pos_of_source ? from : s;
    return {b * p.xb + from * p.xs, b * p.ob + s * p.os, (b * p.pos_stride_b + at) * p.axes, at};
}

// A thread has 32 bytes of a head -- two runs of 16 in the half layout, `pairs` elements apart, 32 in a row in the
// interleaved one -- of heads_per_thread heads of one token, HU of them in flight; further threads of the row copy
// what is not rotated, 16 bytes each.
template <class T, bool INTERLEAVED, int HU>
__global__ void __launch_bounds__(THREADS)
rotary_kernel(const __grid_constant__ Params p, const Divider per_batch, const Divider per_row) {
    constexpr int N = 16 / (int)sizeof(T);   // pairs of a thread = elements of a run
    allow_next();
    // one 64-bit division a block; the quotient below is of a number under THREADS + a row's threads
    const long long first = (long long)blockIdx.x * THREADS;
    const long long token0 = first / per_row.d;
    const unsigned rest = (unsigned)(first - token0 * per_row.d) + threadIdx.x;
    const unsigned dt = per_row.quotient(rest);
    const int item = (int)(rest - dt * per_row.d);
    const long long token = token0 + dt;
    wait_for_previous();
    if (token >= p.tokens) return;
    const Token at = locate(p, token, per_batch);
    const int h0 = blockIdx.y * p.heads_per_thread, h1 = min(h0 + p.heads_per_thread, p.heads);
    const int rotating = (p.pairs + N - 1) / N;
    if (item >= rotating) {
        const int c = (INTERLEAVED ? rotating * 2 * N : 2 * p.pairs) + (item - rotating) * N;
        for (int h = h0; h < h1; h += HU) {
            uint4 v[HU];
#pragma unroll
            for (int i = 0; i < HU; ++i)
                if (h + i < h1) v[i] = *reinterpret_cast<const uint4 *>((const T *)p.x + at.x + (h + i) * p.xh + c);
#pragma unroll
            for (int i = 0; i < HU; ++i)
                if (h + i < h1) *reinterpret_cast<uint4 *>((T *)p.out + at.out + (h + i) * p.oh + c) = v[i];
        }
        return;
    }
    const int j0 = item * N, ca = INTERLEAVED ? 2 * j0 : j0, cb = INTERLEAVED ? 2 * j0 + N : j0 + p.pairs;
    Chunk<T> a[HU], b[HU];
    auto load = [&](int h) {
#pragma unroll
        for (int i = 0; i < HU; ++i)
            if (h + i < h1) {
                const T *row = (const T *)p.x + at.x + (h + i) * p.xh;
                a[i].v = *reinterpret_cast<const uint4 *>(row + ca);
                // the last threads of an interleaved row may have half a run
                if (!INTERLEAVED || cb < p.dim) b[i].v = *reinterpret_cast<const uint4 *>(row + cb);
            }
    };
    load(h0);   // in flight while the angles are computed
    float cs[N], sn[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int j = j0 + i;
        if (j < p.pairs) {
            const int pos = p.positions ? p.positions[at.pos + p.axis[j]] : at.index;
            const float2 t = cos_sin(pos, p.turns[j]);
            cs[i] = t.x * p.factor;
            sn[i] = t.y * p.factor * p.sign;
        } else {
            cs[i] = sn[i] = 0.f;
        }
    }
    for (int h = h0;;) {
#pragma unroll
        for (int i = 0; i < HU; ++i) {
            if (h + i >= h1) continue;
            float fa[N], fb[N];
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int e = 0; e < N / 2; ++e) {
                    const float x0 = a[i].get(2 * e), y0 = a[i].get(2 * e + 1), x1 = b[i].get(2 * e), y1 = b[i].get(2 * e + 1);
                    // elements behind the rotated part stay, whatever they hold
                    const bool r0 = j0 + e < p.pairs, r1 = j0 + N / 2 + e < p.pairs;
                    fa[2 * e] = r0 ? x0 * cs[e] - y0 * sn[e] : x0;
                    fa[2 * e + 1] = r0 ? x0 * sn[e] + y0 * cs[e] : y0;
                    fb[2 * e] = r1 ? x1 * cs[N / 2 + e] - y1 * sn[N / 2 + e] : x1;
                    fb[2 * e + 1] = r1 ? x1 * sn[N / 2 + e] + y1 * cs[N / 2 + e] : y1;
                }
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float x0 = a[i].get(e), y0 = b[i].get(e);
                    fa[e] = x0 * cs[e] - y0 * sn[e];
                    fb[e] = x0 * sn[e] + y0 * cs[e];
                }
            }
            T *row = (T *)p.out + at.out + (h + i) * p.oh;
            Chunk<T> o;
            o.set(fa);
            *reinterpret_cast<uint4 *>(row + ca) = o.v;
            if (!INTERLEAVED || cb < p.dim) {
                o.set(fb);
                *reinterpret_cast<uint4 *>(row + cb) = o.v;
            }
        }
        h += HU;
        if (h >= h1) break;
        load(h);
    }
}

// Any pair count, stride and alignment: a thread has one pair, or one element that is not rotated.
template <class T, bool INTERLEAVED>
__global__ void __launch_bounds__(THREADS)
rotary_single_kernel(const __grid_constant__ Params p, const Divider per_batch, const Divider per_row) {
    allow_next();
    const long long first = (long long)blockIdx.x * THREADS;
    const long long token0 = first / per_row.d;
    const unsigned rest = (unsigned)(first - token0 * per_row.d) + threadIdx.x;
    const unsigned dt = per_row.quotient(rest);
    const int item = (int)(rest - dt * per_row.d);
    const long long token = token0 + dt;
    wait_for_previous();
    if (token >= p.tokens) return;
    const Token at = locate(p, token, per_batch);
    const int h0 = blockIdx.y * p.heads_per_thread, h1 = min(h0 + p.heads_per_thread, p.heads);
    const T *x = (const T *)p.x + at.x;
    T *out = (T *)p.out + at.out;
    if (item >= p.pairs) {
        const int c = p.pairs + item;
        for (int h = h0; h < h1; ++h) out[h * p.oh + c] = x[h * p.xh + c];
        return;
    }
    const int pos = p.positions ? p.positions[at.pos + p.axis[item]] : at.index;
    float2 t = cos_sin(pos, p.turns[item]);
    t.x *= p.factor;
    t.y *= p.factor * p.sign;
    const int ca = INTERLEAVED ? 2 * item : item, cb = INTERLEAVED ? 2 * item + 1 : item + p.pairs;
#pragma unroll 4
    for (int h = h0; h < h1; ++h) {
        const float a = (float)x[h * p.xh + ca], b = (float)x[h * p.xh + cb];
        out[h * p.oh + ca] = (T)(a * t.x - b * t.y);
        out[h * p.oh + cb] = (T)(a * t.y + b * t.x);
    }
}

// The frequency as a fraction of a turn in 2^-64: (inv_freq / 2 pi) mod 1, in 64-bit mantissas.
unsigned long long to_turns(double inv_freq) {
    const long double two_pi = 6.283185307179586476925286766559005768L;
    long double t = (long double)inv_freq / two_pi;
    t -= std::floor(t);
    const long double scaled = std::floor(t * 18446744073709551616.0L + 0.5L);
    return scaled >= 18446744073709551616.0L ? 0ull : (unsigned long long)scaled;
}

// Elements between the first of [batch, heads, S, dim] with these strides and the one behind the last.
long long extent(const int64_t *st, int batch, int heads, int S, int dim) {
    return st[0] * (batch - 1) + st[1] * (heads - 1) + st[2] * (S - 1) + dim;
}

int launch(const void *x, void *out, const int32_t *positions, const double *inv_freq, const int32_t *axis, int pairs, int axes,
           int interleaved, double factor, const hilberta_plan_t *plan, int batch, int heads, int S, int head_dim, int dtype,
           const int64_t *strides, int64_t pos_stride_b, int backward, cudaStream_t stream) {
    const bool none = batch == 0 || S == 0;
    if ((!none && (!x || !out)) || !inv_freq || !strides || batch < 0 || heads < 1 || S < 0 || head_dim < 1 || pairs < 1 || axes < 1 || pos_stride_b < 0)
        return HILBERTA_ERR_INVALID;
    if (dtype == HILBERTA_FP8_E4M3) return HILBERTA_ERR_UNSUPPORTED;
    if (dtype != HILBERTA_BF16 && dtype != HILBERTA_FP32) return HILBERTA_ERR_INVALID;
    if (2ll * pairs > head_dim || (!positions && axes != 1) || !std::isfinite(factor)) return HILBERTA_ERR_INVALID;
    if (head_dim > 2 * MAX_PAIRS || axes > 16) return HILBERTA_ERR_UNSUPPORTED;
    if (plan && plan->S != S) return HILBERTA_ERR_INVALID;
    const int esz = dtype == HILBERTA_BF16 ? 2 : 4;
    if (((uintptr_t)x | (uintptr_t)out) & (esz - 1) || ((uintptr_t)positions & 3)) return HILBERTA_ERR_INVALID;
    if ((long long)batch * S > 0x7fffffffll) return HILBERTA_ERR_UNSUPPORTED;
    Params p;
    for (int j = 0; j < pairs; ++j) {
        if (!std::isfinite(inv_freq[j])) return HILBERTA_ERR_INVALID;
        const int a = axis ? axis[j] : 0;
        if (a < 0 || a >= axes) return HILBERTA_ERR_INVALID;
        p.turns[j] = to_turns(inv_freq[j]);
        p.axis[j] = (unsigned char)a;
    }
    const int64_t n_of[3] = {batch, heads, S};
    for (int i = 0; i < 6; ++i)
        if (strides[i] < 0 || (i >= 3 && n_of[i - 3] > 1 && strides[i] == 0)) return HILBERTA_ERR_INVALID;
    int dev = -1;
    HB_CUDA(cudaGetDevice(&dev));
    if (plan && plan->device != dev) return HILBERTA_ERR_INVALID;
    const int sms = sm100_count(dev);
    if (!sms) return HILBERTA_ERR_ARCH;
    if (none) return HILBERTA_OK;
    // in place: the very same rows, in the same order
    const bool same = x == out && !plan && std::equal(strides, strides + 3, strides + 3);
    if (!same) {
        const char *a = (const char *)x, *b = (const char *)out;
        if (a < b + extent(strides + 3, batch, heads, S, head_dim) * esz && b < a + extent(strides, batch, heads, S, head_dim) * esz) {
            // ranges meet: let through only slices of one interleaved buffer that share no element
            const bool alike = std::equal(strides, strides + 3, strides + 3);
            if (!alike || hilberta_check_overlap((uint64_t)(uintptr_t)x, (uint64_t)(uintptr_t)out, batch, heads, S, strides[0] * esz,
                                                 strides[1] * esz, strides[2] * esz, (int64_t)head_dim * esz) != 0)
                return HILBERTA_ERR_INVALID;
        }
    }
    p.x = x;
    p.out = out;
    p.positions = positions;
    p.row_map = plan ? (backward ? plan->d_orig2phys : plan->d_phys2orig) : nullptr;
    p.pos_of_source = backward ? 0 : 1;
    p.axes = axes;
    p.pos_stride_b = pos_stride_b;
    p.xb = strides[0], p.xh = strides[1], p.xs = strides[2];
    p.ob = strides[3], p.oh = strides[4], p.os = strides[5];
    p.pairs = pairs;
    p.dim = head_dim;
    p.heads = heads;
    p.S = S;
    p.tokens = (long long)batch * S;
    p.factor = (float)factor;
    p.sign = backward ? -1.f : 1.f;

    const int n = 16 / esz;
    int64_t bits = (int64_t)((uintptr_t)x | (uintptr_t)out);
    for (int i = 0; i < 6; ++i) bits |= strides[i] * esz;
    const bool vectors = (bits & 15) == 0 && head_dim % n == 0 && (interleaved || pairs % n == 0);
    const int rotating = vectors ? (pairs + n - 1) / n : pairs;
    const int beyond = vectors ? std::max(0, head_dim - (interleaved ? rotating * 2 * n : 2 * pairs)) / n : head_dim - 2 * pairs;
    // in place there is nothing to copy
    const int row_threads = rotating + (same ? 0 : beyond);
    // heads of a thread: the angles are shared by them, but a few hundred thousand threads are wanted first
    constexpr int HU = 4;
    const long long units = p.tokens * row_threads;
    int hpt = 1;
    while (hpt < 8 && hpt < heads && units * ((heads + hpt * 2 - 1) / (hpt * 2)) >= (long long)sms * 1024) hpt *= 2;
    p.heads_per_thread = hpt;
    const long long blocks = (units + THREADS - 1) / THREADS;
    const int chunks = (heads + hpt - 1) / hpt;
    if (blocks > 0x7fffffffll || chunks > 65535) return HILBERTA_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks, (unsigned)chunks);
    const bool overlap = (size_t)p.tokens * heads * head_dim * esz <= kOverlapBytes;
    auto go = [&](auto kernel) {
        return launch_overlapping(kernel, grid, THREADS, 0, 1, stream, overlap, p, Divider(S), Divider(row_threads));
    };
    if (dtype == HILBERTA_BF16) {
        if (vectors) HB_CUDA(interleaved ? go(rotary_kernel<__nv_bfloat16, true, HU>) : go(rotary_kernel<__nv_bfloat16, false, HU>));
        else HB_CUDA(interleaved ? go(rotary_single_kernel<__nv_bfloat16, true>) : go(rotary_single_kernel<__nv_bfloat16, false>));
    } else {
        if (vectors) HB_CUDA(interleaved ? go(rotary_kernel<float, true, HU>) : go(rotary_kernel<float, false, HU>));
        else HB_CUDA(interleaved ? go(rotary_single_kernel<float, true>) : go(rotary_single_kernel<float, false>));
    }
    HB_LAUNCHED();
    return HILBERTA_OK;
}

}  // namespace
}  // namespace hilberta

extern "C" int hilberta_rotary(const void *x, void *out, const int32_t *positions, const double *inv_freq, const int32_t *axis,
                               int pairs, int axes, int interleaved, double factor, const hilberta_plan_t *plan, int batch, int heads,
                               int S, int head_dim, int dtype, const int64_t *strides, int64_t position_stride_b, void *stream) {
    return hilberta::launch(x, out, positions, inv_freq, axis, pairs, axes, interleaved, factor, plan, batch, heads, S, head_dim, dtype,
                            strides, position_stride_b, 0, (cudaStream_t)stream);
}

extern "C" int hilberta_rotary_backward(const void *dout, void *dx, const int32_t *positions, const double *inv_freq,
                                        const int32_t *axis, int pairs, int axes, int interleaved, double factor,
                                        const hilberta_plan_t *plan, int batch, int heads, int S, int head_dim, int dtype,
                                        const int64_t *strides, int64_t position_stride_b, void *stream) {
    return hilberta::launch(dout, dx, positions, inv_freq, axis, pairs, axes, interleaved, factor, plan, batch, heads, S, head_dim, dtype,
                            strides, position_stride_b, 1, (cudaStream_t)stream);
}

extern "C" int hilberta_rotary_frequencies(double *inv_freq, int pairs, double base, int scaling, double scale, double context,
                                           double slow, double fast, double *factor) {
    if (!inv_freq || pairs < 1 || !(base > 0.) || !std::isfinite(base)) return HILBERTA_ERR_INVALID;
    if (scaling < HILBERTA_ROTARY_PLAIN || scaling > HILBERTA_ROTARY_BANDS) return HILBERTA_ERR_INVALID;
    if (scaling != HILBERTA_ROTARY_PLAIN && (!(scale >= 1.) || !std::isfinite(scale))) return HILBERTA_ERR_INVALID;
    if (scaling == HILBERTA_ROTARY_BANDS && (!(context > 0.) || !(fast > slow) || !(slow >= 0.) || !std::isfinite(context) || !std::isfinite(fast)))
        return HILBERTA_ERR_INVALID;
    if (scaling == HILBERTA_ROTARY_BASE && pairs > 1) base *= std::pow(scale, pairs / (pairs - 1.));
    const double two_pi = 6.283185307179586476925;
    for (int j = 0; j < pairs; ++j) {
        double f = std::pow(base, -(double)j / pairs);
        if (scaling == HILBERTA_ROTARY_LINEAR) f /= scale;
        if (scaling == HILBERTA_ROTARY_BANDS) {
            const double ramp = std::min(1., std::max(0., (context * f / two_pi - slow) / (fast - slow)));
            f *= ramp + (1. - ramp) / scale;
        }
        inv_freq[j] = f;
    }
    if (factor) *factor = scaling == HILBERTA_ROTARY_BANDS ? 1. + 0.1 * std::log(scale) : 1.;
    return HILBERTA_OK;
}
