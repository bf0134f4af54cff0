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
// Measured (B200, us; share of the copy bandwidth): 12 heads of 16384 tokens fp32 33 (93 %), 24 heads bf16 34 (90 %), with
// the entry gather and three axes 40 (79 %: rows of 256 bytes in Hilbert order); one head has the angles to itself, 100000
// tokens 9.4 (42 %); 16 single tokens of 32 heads 2, a launch.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "common.cuh"

namespace hilberta {
namespace {

constexpr int MAX_PAIRS = 128;   // head dim <= 256
constexpr int THREADS = 128;

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

// The angle pos * turns as a quarter turn 0 ... 3 and a remainder of at most an eighth of a turn, 2^32 to a turn.  The low
// half of the 64-bit product is dropped (2^-32 of a turn).
__device__ __forceinline__ int remainder_of(int pos, unsigned long long turns, unsigned &quarter) {
    const unsigned lo = (unsigned)turns, hi = (unsigned)(turns >> 32);
    const unsigned u = __umulhi((unsigned)pos, lo) + (unsigned)pos * hi - (pos < 0 ? lo : 0u);
    quarter = (u + (1u << 29)) >> 30;
    return (int)(u - (quarter << 30));
}

// cos and sin of two angles by their Taylor series, |angle| <= pi / 4: the first terms left out are below 2^-32 and 2^-28 of
// the result.  Packed arithmetic: two angles an instruction (the library's sincospif for each, 3.2 million angles and no more
// than one head to use them, took 14.5 us in all).
__device__ __forceinline__ void cos_sin2(const int *pos, const unsigned long long *turns, float2 &cos, float2 &sin) {
    unsigned q0, q1;
    const int r0 = remainder_of(pos[0], turns[0], q0), r1 = remainder_of(pos[1], turns[1], q1);
    const float unit = 1.4629180792671596e-9f;   // 2 pi / 2^32
    const float2 x = __fmul2_rn(make_float2((float)r0, (float)r1), make_float2(unit, unit)), z = __fmul2_rn(x, x);
    auto c2 = [](float v) { return make_float2(v, v); };
    float2 s = __ffma2_rn(z, c2(1.f / 362880.f), c2(-1.f / 5040.f));
    s = __ffma2_rn(s, z, c2(1.f / 120.f));
    s = __ffma2_rn(s, z, c2(-1.f / 6.f));
    s = __ffma2_rn(__fmul2_rn(s, z), x, x);
    float2 c = __ffma2_rn(z, c2(-1.f / 3628800.f), c2(1.f / 40320.f));
    c = __ffma2_rn(c, z, c2(-1.f / 720.f));
    c = __ffma2_rn(c, z, c2(1.f / 24.f));
    c = __ffma2_rn(c, z, c2(-0.5f));
    c = __ffma2_rn(c, z, c2(1.f));
    auto turn = [](unsigned q, float c, float s, float &co, float &si) {
        const float a = q & 1 ? s : c, b = q & 1 ? c : s;   // |cos|, |sin|
        co = __uint_as_float(__float_as_uint(a) ^ (((q + 1) & 2) << 30));
        si = __uint_as_float(__float_as_uint(b) ^ ((q & 2) << 30));
    };
    turn(q0, c.x, s.x, cos.x, sin.x);
    turn(q1, c.y, s.y, cos.y, sin.y);
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
    // elements 2 i and 2 i + 1 as `from` has them, bit for bit (a NaN does not survive the way through fp32)
    __device__ __forceinline__ void copy_pair(int i, const Chunk &from) {
        uint32_t *w = &v.x;
        const uint32_t *o = &from.v.x;
        if constexpr (sizeof(T) == 4) w[2 * i] = o[2 * i], w[2 * i + 1] = o[2 * i + 1];
        else w[i] = o[i];
    }
};

// The frequencies, from the parameters (where lanes that want different ones are served one after the other) to shared
// memory once a block.
struct Table {
    unsigned long long turns[MAX_PAIRS + 8];
    int axis[MAX_PAIRS + 8];
};
__device__ __forceinline__ void fill_table(Table &t, const Params &p) {
    for (int i = threadIdx.x; i < p.pairs; i += THREADS) {
        t.turns[i] = p.turns[i];
        t.axis[i] = p.axis[i];
    }
    __syncthreads();
}

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

// factor times cos and sin of N pairs from j0 on (N even; past the last pair: zeros)
template <int N>
__device__ __forceinline__ void angles(const Params &p, const Table &table, const Token &at, int j0, float *cs, float *sn) {
    int pos[N];
    unsigned long long turns[N];
    const int one = p.positions ? p.axes == 1 ? p.positions[at.pos] : 0 : at.index;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int j = min(j0 + i, p.pairs - 1);
        turns[i] = table.turns[j];
        pos[i] = p.axes == 1 ? one : p.positions[at.pos + table.axis[j]];
    }
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        float2 c, s;
        cos_sin2(pos + i, turns + i, c, s);
        const float f = p.factor, g = p.factor * p.sign;
        cs[i] = c.x * f;
        cs[i + 1] = c.y * f;
        sn[i] = s.x * g;
        sn[i + 1] = s.y * g;
    }
}

// One element of a turned pair, rounded alike in every kernel: sn is negative for the first of the two.
__device__ __forceinline__ float turned(float x, float partner, float cs, float sn) { return __fmaf_rn(x, cs, __fmul_rn(partner, sn)); }

// A thread has 32 bytes of a head -- two runs of 16 in the half layout, `pairs` elements apart, 32 in a row in the
// interleaved one -- of heads_per_thread heads of one token, HU of them in flight; further threads of the row copy
// what is not rotated, 16 bytes each.
template <class T, bool INTERLEAVED, int HU>
__global__ void __launch_bounds__(THREADS, 6)
rotary_kernel(const __grid_constant__ Params p, const Divider per_batch, const Divider per_row) {
    constexpr int N = 16 / (int)sizeof(T);   // pairs of a thread = elements of a run
    __shared__ Table table;
    allow_next();
    fill_table(table, p);
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
    angles<N>(p, table, at, j0, cs, sn);
    for (int h = h0;;) {
#pragma unroll
        for (int i = 0; i < HU; ++i) {
            if (h + i >= h1) continue;
            float fa[N], fb[N];
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int e = 0; e < N / 2; ++e) {
                    const float x0 = a[i].get(2 * e), y0 = a[i].get(2 * e + 1), x1 = b[i].get(2 * e), y1 = b[i].get(2 * e + 1);
                    fa[2 * e] = turned(x0, y0, cs[e], -sn[e]);
                    fa[2 * e + 1] = turned(y0, x0, cs[e], sn[e]);
                    fb[2 * e] = turned(x1, y1, cs[N / 2 + e], -sn[N / 2 + e]);
                    fb[2 * e + 1] = turned(y1, x1, cs[N / 2 + e], sn[N / 2 + e]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float x0 = a[i].get(e), y0 = b[i].get(e);
                    fa[e] = turned(x0, y0, cs[e], -sn[e]);
                    fb[e] = turned(y0, x0, cs[e], sn[e]);
                }
            }
            T *row = (T *)p.out + at.out + (h + i) * p.oh;
            // interleaved: elements behind the rotated part stay, whatever they hold
            Chunk<T> o;
            o.set(fa);
#pragma unroll
            for (int e = 0; INTERLEAVED && e < N / 2; ++e)
                if (j0 + e >= p.pairs) o.copy_pair(e, a[i]);
            __stcs(reinterpret_cast<uint4 *>(row + ca), o.v);
            if (!INTERLEAVED || cb < p.dim) {
                o.set(fb);
#pragma unroll
                for (int e = 0; INTERLEAVED && e < N / 2; ++e)
                    if (j0 + N / 2 + e >= p.pairs) o.copy_pair(e, b[i]);
                __stcs(reinterpret_cast<uint4 *>(row + cb), o.v);
            }
        }
        h += HU;
        if (h >= h1) break;
        load(h);
    }
}

// Half layout with a pair count that leaves the second half unaligned: a thread has 16 bytes of the output of
// heads_per_thread heads and reads the elements they are paired with one by one.  Not in place: those belong to other
// threads.  (8 heads of 16384 tokens, head dim 128, 33 pairs, bf16: 53 us with a pair a thread, 17 so.)
template <class T>
__global__ void __launch_bounds__(THREADS)
rotary_shifted_kernel(const __grid_constant__ Params p, const Divider per_batch, const Divider per_row) {
    constexpr int N = 16 / (int)sizeof(T);
    __shared__ Table table;
    allow_next();
    fill_table(table, p);
    const long long first = (long long)blockIdx.x * THREADS;
    const long long token0 = first / per_row.d;
    const unsigned rest = (unsigned)(first - token0 * per_row.d) + threadIdx.x;
    const unsigned dt = per_row.quotient(rest);
    const int c0 = (int)(rest - dt * per_row.d) * N;   // first element
    const long long token = token0 + dt;
    wait_for_previous();
    if (token >= p.tokens) return;
    const Token at = locate(p, token, per_batch);
    const int h0 = blockIdx.y * p.heads_per_thread, h1 = min(h0 + p.heads_per_thread, p.heads);
    float cs[N], sn[N];   // out = cs * x[c] + sn * x[partner]
    int partner[N];
    {
        int pos[N];
        unsigned long long turns[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = c0 + i, j = min(c < p.pairs ? c : c - p.pairs, p.pairs - 1);
            turns[i] = table.turns[j];
            pos[i] = p.positions ? p.positions[at.pos + table.axis[j]] : at.index;
            partner[i] = c >= 2 * p.pairs ? c : c < p.pairs ? c + p.pairs : c - p.pairs;
        }
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            float2 c, s;
            cos_sin2(pos + i, turns + i, c, s);
            cs[i] = c.x * p.factor;
            cs[i + 1] = c.y * p.factor;
            sn[i] = s.x * p.factor * p.sign * (c0 + i < p.pairs ? -1.f : 1.f);
            sn[i + 1] = s.y * p.factor * p.sign * (c0 + i + 1 < p.pairs ? -1.f : 1.f);
        }
    }
    for (int h = h0; h < h1; ++h) {
        const T *row = (const T *)p.x + at.x + h * p.xh;
        Chunk<T> a, o;
        a.v = *reinterpret_cast<const uint4 *>(row + c0);
        float f[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float x = a.get(i);
            f[i] = c0 + i < 2 * p.pairs ? turned(x, (float)row[partner[i]], cs[i], sn[i]) : x;
        }
        o.set(f);
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
            if (c0 + 2 * i >= 2 * p.pairs) o.copy_pair(i, a);
        *reinterpret_cast<uint4 *>((T *)p.out + at.out + h * p.oh + c0) = o.v;
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
    const int pos = p.positions ? p.positions[at.pos + p.axis[item]] : at.index, two[2] = {pos, pos};
    const unsigned long long turns[2] = {p.turns[item], p.turns[item]};
    float2 c, s;
    cos_sin2(two, turns, c, s);
    const float cs = c.x * p.factor, sn = s.x * p.factor * p.sign;
    const int ca = INTERLEAVED ? 2 * item : item, cb = INTERLEAVED ? 2 * item + 1 : item + p.pairs;
#pragma unroll 4
    for (int h = h0; h < h1; ++h) {
        const float a = (float)x[h * p.xh + ca], b = (float)x[h * p.xh + cb];
        out[h * p.oh + ca] = (T)turned(a, b, cs, -sn);
        out[h * p.oh + cb] = (T)turned(b, a, cs, sn);
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
    const bool aligned = (bits & 15) == 0 && head_dim % n == 0, vectors = aligned && (interleaved || pairs % n == 0);
    const bool shifted = aligned && !vectors && !same;   // half layout
    const int rotating = vectors ? (pairs + n - 1) / n : pairs;
    const int beyond = vectors ? std::max(0, head_dim - (interleaved ? rotating * 2 * n : 2 * pairs)) / n : head_dim - 2 * pairs;
    // in place there is nothing to copy
    const int row_threads = shifted ? head_dim / n : rotating + (same ? 0 : beyond);
    // Heads of a thread: the angles are shared by them, but a few hundred thousand threads are wanted first.  Four of them in
    // flight, or two where a thread has no more (registers: 100000 tokens of one head of 64, us, 4 / 2: 10.6 / 8.5; 24 heads of
    // 16384 tokens 33.8 / 36.0).
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
        if (vectors) HB_CUDA(hpt >= 4 ? (interleaved ? go(rotary_kernel<__nv_bfloat16, true, 4>) : go(rotary_kernel<__nv_bfloat16, false, 4>))
                                 : (interleaved ? go(rotary_kernel<__nv_bfloat16, true, 2>) : go(rotary_kernel<__nv_bfloat16, false, 2>)));
        else if (shifted) HB_CUDA(go(rotary_shifted_kernel<__nv_bfloat16>));
        else HB_CUDA(interleaved ? go(rotary_single_kernel<__nv_bfloat16, true>) : go(rotary_single_kernel<__nv_bfloat16, false>));
    } else {
        if (vectors) HB_CUDA(hpt >= 4 ? (interleaved ? go(rotary_kernel<float, true, 4>) : go(rotary_kernel<float, false, 4>))
                                 : (interleaved ? go(rotary_kernel<float, true, 2>) : go(rotary_kernel<float, false, 2>)));
        else if (shifted) HB_CUDA(go(rotary_shifted_kernel<float>));
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
