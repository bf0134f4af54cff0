// What the forward and backward kernels of the packed attention share: how the units of work are found.
//
// The sequences' lengths are known on the device only, so every CTA finds its own units from cu_seqlens; no list is
// made beforehand and no counter is shared.  Units come longest first, and CTA c of G takes units c, 2 G - 1 - c,
// 2 G + c, ...: the loads of a round are evened out by the next.  A sequence of n tokens has blocks of 1 << shift tokens.
//   causal      A block's work grows with its distance from the start (out, dq) or the end (dk, dv) of its sequence.
//               Level l holds one block of every sequence with more than l blocks, all of the same work; the levels
//               are gone through from the highest down.
//   not causal  All blocks of a sequence have the same work; sequences with more blocks come first.
// Either way the order consists of runs in which the same sequences take part, and a pass over cu_seqlens finds the
// next run.
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
    int causal;
};

struct Unit {
    int row0, len;      // the sequence: first row, tokens; len < 0: no more units
    int block, head;    // causal: the block's level, else the block; index among the heads' parts
};

// A run: `count` sequences take part.  causal: the levels low .. top of those with more than `top` blocks.  Else all
// blocks of those with `low` blocks.  `before` blocks lie in earlier runs.
struct Runs {
    int top = 0x7fffffff, low = 0x7fffffff, count = 0;
    long long before = 0;
};

__device__ __forceinline__ int blocks_of(const Sequences &s, int i, int &row0, int &len) {
    // whatever cu_seqlens holds, rows stay inside [0, total)
    row0 = min(max(s.cu[i], 0), s.total);
    len = min(max(s.cu[i + 1], row0), s.total) - row0;
    return (int)(((long long)len + (1 << s.shift) - 1) >> s.shift);
}

// Block k (0 = first) in this order, called by a whole warp with k not smaller than before.  false: there are fewer.
__device__ __forceinline__ bool find_block(const Sequences &s, Runs &st, long long k, int &row0, int &len, int &block) {
    const int lane = threadIdx.x & 31;
    for (;;) {
        const long long in_run = (long long)(s.causal ? st.top - st.low + 1 : st.low) * st.count;
        if (k < st.before + in_run) break;
        st.before += in_run;
        if (st.low == 0) return false;
        st.top = st.low - 1;
        int count = 0, low = 0;
        for (int i = lane; i < s.n; i += 32) {
            int a, b;
            const int nb = blocks_of(s, i, a, b);
            if (nb <= st.top) low = max(low, nb);
            else ++count;
        }
        st.low = (int)__reduce_max_sync(0xffffffffu, (unsigned)low);
        if (!s.causal) {
            count = 0;
            for (int i = lane; i < s.n; i += 32) {
                int a, b;
                count += blocks_of(s, i, a, b) == st.low ? 1 : 0;
            }
        }
        st.count = (int)__reduce_add_sync(0xffffffffu, (unsigned)count);
    }
    const long long at = k - st.before;
    int j;   // the block is one of the run's j-th sequence
    if (s.causal) {
        block = st.top - (int)(at / st.count);
        j = (int)(at % st.count);
    } else {
        j = (int)(at / st.low);
        block = (int)(at % st.low);
    }
    for (int i0 = 0; i0 < s.n; i0 += 32) {
        int a = 0, b = 0, nb = 0;
        if (i0 + lane < s.n) nb = blocks_of(s, i0 + lane, a, b);
        const bool has = s.causal ? nb > st.top : nb == st.low;   // a run has at least one block: low > 0 here
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
__device__ __forceinline__ bool find_unit(const Sequences &s, Runs &st, int parts, int cta, int ctas, int round, Unit &u) {
    const long long n = (long long)round * ctas + ((round & 1) ? ctas - 1 - cta : cta);
    u.head = (int)(n % parts);
    return find_block(s, st, n / parts, u.row0, u.len, u.block);
}

// Tensor map of [rows, heads, head_dim] bf16: boxes of 64 columns x box_heads x box_rows, 128-byte swizzled rows.
int make_map(CUtensorMap *m, const void *base, int rows, int heads, int head_dim, long long stride_row, long long stride_head,
             int box_heads, int box_rows);

int check(const void *const *tensors, int n, const int64_t *strides, const int32_t *cu, int n_seq, int total, int heads, int kv_heads,
          int head_dim, int dtype);
bool overlap(const void *a, const int64_t *sa, int ha, const void *b, const int64_t *sb, int hb, int total, int head_dim);

// Codes of waits that gave up, of the forward and the backward kernels: read and cleared.
int forward_status(bool *expired);
int backward_status(bool *expired);

// The largest power of two that divides the heads of a group, at most 16: so many heads of one token are rows of a
// query tile next to one another.
inline int packed_heads(int group) {
    int g = 1;
    while (g < 16 && group % (2 * g) == 0) g *= 2;
    return g;
}

}  // namespace packed
}  // namespace hilberta
