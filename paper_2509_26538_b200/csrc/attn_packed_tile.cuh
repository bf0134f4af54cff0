// What the forward and backward kernels of the packed attention share: how the units of work are found.
//
// The sequences' lengths are known on the device only, so every CTA finds its own units from cu_seqlens; no list is
// made beforehand and no counter is shared.  A sequence of n tokens has blocks of `per` tokens; with a causal mask a
// block's work grows with its distance from the end (dk, dv) or the start (out, dq) of its sequence.  Level l holds
// one block of every sequence with more than l blocks, all of the same work, so going through the levels from the
// highest down is going through the units longest first, and CTA c of G takes units c, 2 G - 1 - c, 2 G + c, ...: the
// loads of a round are evened out by the next.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace hilberta {
namespace packed {

// Limit of `total`: a unit over so many keys still ends well within the bounded waits.
constexpr int MAX_TOTAL = 1 << 26;
constexpr int MAX_SEQ = 65536;

struct Sequences {
    const int *cu;      // [n + 1]
    int n, total;
    int shift;          // blocks of 1 << shift tokens
};

struct Unit {
    int row0, len;      // the sequence: first row, tokens; len < 0: no more units
    int block, head;    // block of its tokens, counted by level from the top (see above); index among the heads' parts
};

// Runs of levels, from the highest down: levels low .. top belong to the same `count` sequences, `before` blocks lie
// in the levels above.
struct Levels {
    int top = 0x7fffffff, low = 0x7fffffff, count = 0;
    long long before = 0;
};

__device__ __forceinline__ int blocks_of(const Sequences &s, int i, int &row0, int &len) {
    // whatever cu_seqlens holds, rows stay inside [0, total)
    row0 = min(max(s.cu[i], 0), s.total);
    len = min(max(s.cu[i + 1], row0), s.total) - row0;
    return (int)(((long long)len + (1 << s.shift) - 1) >> s.shift);
}

// Block k (0 = first) in level order, called by a whole warp with k not smaller than before.  false: there are fewer.
__device__ __forceinline__ bool find_block(const Sequences &s, Levels &st, long long k, int &row0, int &len, int &level) {
    const int lane = threadIdx.x & 31;
    for (;;) {
        const long long in_run = (long long)(st.top - st.low + 1) * st.count;
        if (k < st.before + in_run) break;
        st.before += in_run;
        if (st.low == 0) return false;
        st.top = st.low - 1;
        int count = 0, low = 0;
        for (int i = lane; i < s.n; i += 32) {
            int a, b;
            const int nb = blocks_of(s, i, a, b);
            if (nb > st.top) ++count;
            else low = max(low, nb);
        }
        st.count = (int)__reduce_add_sync(0xffffffffu, (unsigned)count);
        st.low = (int)__reduce_max_sync(0xffffffffu, (unsigned)low);
    }
    const long long at = k - st.before;
    level = st.top - (int)(at / st.count);
    int j = (int)(at % st.count);
    for (int i0 = 0; i0 < s.n; i0 += 32) {
        int a = 0, b = 0;
        const bool has = i0 + lane < s.n && blocks_of(s, i0 + lane, a, b) > st.top;
        const unsigned who = __ballot_sync(0xffffffffu, has);
        const int c = __popc(who);
        if (j < c) {
            const bool it = has && __popc(who & ((1u << lane) - 1u)) == j;
            const int src = __ffs((int)__ballot_sync(0xffffffffu, it)) - 1;
            row0 = __shfl_sync(0xffffffffu, a, src);
            len = __shfl_sync(0xffffffffu, b, src);
            return true;
        }
        j -= c;
    }
    return false;   // cu_seqlens changed under the kernel
}

// Unit number `round` of CTA `cta` of `ctas`.
__device__ __forceinline__ bool find_unit(const Sequences &s, Levels &st, int parts, int cta, int ctas, int round, Unit &u) {
    const long long n = (long long)round * ctas + ((round & 1) ? ctas - 1 - cta : cta);
    u.head = (int)(n % parts);
    return find_block(s, st, n / parts, u.row0, u.len, u.block);
}

// Tensor map of [rows, heads, head_dim] bf16: boxes of 64 columns x box_heads x box_rows, 128-byte swizzled rows.
int make_map(CUtensorMap *m, const void *base, int rows, int heads, int head_dim, long long stride_row, long long stride_head,
             int box_heads, int box_rows);

// The largest power of two that divides the heads of a group, at most 16: so many heads of one token are rows of a
// query tile next to one another.
inline int packed_heads(int group) {
    int g = 1;
    while (g < 16 && group % (2 * g) == 0) g *= 2;
    return g;
}

}  // namespace packed
}  // namespace hilberta
