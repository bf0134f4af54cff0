// What the forward and backward kernels of the packed attention share: how the units of work are found.
//
// The sequences' lengths are known on the device only, so every CTA finds its units from cu_seqlens; no list is made
// beforehand.  A launch has a CTA for every unit there may be, in the order in which they should start, longest first; a CTA
// that runs goes on with the next one that has not started by cancelling its launch (clusterlaunchcontrol), so SMs stay busy
// to the end without a counter in memory.  A sequence of n tokens has blocks of 1 << shift tokens.
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

// Limit of `total`: rows of a streamed block's coordinates, 16 heads to a token, stay well below 2^31.
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
    int mode;           // of the backward kernel
};

// A run: `count` sequences take part.  causal: the levels low .. top of those with more than `top` blocks.  Else all
// blocks of those with `low` blocks.  `before` blocks lie in earlier runs.
struct Runs {
    int top = 0x7fffffff, low = 0x7fffffff, count = 0;
    unsigned before = 0;
};

struct Span {
    int row0, len, blocks;
};
__device__ __forceinline__ Span span_of(const Sequences &s, int i) {
    Span p{0, 0, 0};
    if (i < s.n) {
        // whatever cu_seqlens holds, rows stay inside [0, total)
        p.row0 = min(max(s.cu[i], 0), s.total);
        p.len = min(max(s.cu[i + 1], p.row0), s.total) - p.row0;
        p.blocks = (p.len + (1 << s.shift) - 1) >> s.shift;   // len <= 2^26
    }
    return p;
}

// Block k (0 = first) in this order, called by a whole warp; mine: span_of(s, lane), so that up to 32 sequences are read
// once.  false: there are fewer.  All numbers of blocks and units fit 31 bits: the host sees to it.
__device__ __forceinline__ bool find_block(const Sequences &s, const Span &mine, Runs &st, unsigned k, int &row0, int &len, int &block) {
    const int lane = threadIdx.x & 31;
    if (k < st.before) st = Runs();
    for (;;) {
        const unsigned in_run = (unsigned)(s.causal ? st.top - st.low + 1 : st.low) * (unsigned)st.count;
        if (k < st.before + in_run) break;
        if (st.low == 0) return false;   // the last run stays: more of the missing blocks may be asked for
        st.before += in_run;
        st.top = st.low - 1;
        int count = 0, low = 0;
        for (int i = 0; i < s.n; i += 32) {
            const int nb = i == 0 ? mine.blocks : span_of(s, i + lane).blocks;
            if (nb <= st.top) low = max(low, nb);
            else ++count;
        }
        st.low = (int)__reduce_max_sync(0xffffffffu, (unsigned)low);
        if (!s.causal) {
            count = 0;
            for (int i = 0; i < s.n; i += 32) count += (i == 0 ? mine.blocks : span_of(s, i + lane).blocks) == st.low ? 1 : 0;
        }
        st.count = (int)__reduce_add_sync(0xffffffffu, (unsigned)count);
    }
    const unsigned at = k - st.before;
    unsigned j;   // the block is one of the run's j-th sequence
    if (s.causal) {
        j = at % (unsigned)st.count;
        block = st.top - (int)(at / (unsigned)st.count);
    } else {
        j = at / (unsigned)st.low;
        block = (int)(at % (unsigned)st.low);
    }
    for (int i0 = 0; i0 < s.n; i0 += 32) {
        const Span p = i0 == 0 ? mine : span_of(s, i0 + lane);
        const bool has = s.causal ? p.blocks > st.top : p.blocks == st.low;   // a run has at least one block: low > 0 here
        const unsigned who = __ballot_sync(0xffffffffu, has), c = (unsigned)__popc(who);
        if (j < c) {
            const bool it = has && (unsigned)__popc(who & ((1u << lane) - 1u)) == j;
            const int src = __ffs((int)__ballot_sync(0xffffffffu, it)) - 1;
            row0 = __shfl_sync(0xffffffffu, p.row0, src);
            len = __shfl_sync(0xffffffffu, p.len, src);
            return true;
        }
        j -= c;
    }
    return false;   // cu_seqlens changed under the kernel
}

// Unit n of a launch: heads' part n % parts of block n / parts.
__device__ __forceinline__ bool find_unit(const Sequences &s, const Span &mine, Runs &st, int parts, unsigned n, Unit &u) {
    u.head = (int)(n % (unsigned)parts);
    return find_block(s, mine, st, n / (unsigned)parts, u.row0, u.len, u.block);
}

// The next CTA of the grid that has not started: asked for by one thread, answered (16 bytes) at `to`.
__device__ __forceinline__ void ask_next_cta(uint32_t to, uint32_t bar) {
    ptx::mbar_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(to), "r"(bar)
                 : "memory");
}
// Its number; false: all have started, and nothing may be asked for again.
__device__ __forceinline__ bool next_cta(uint32_t from, unsigned &cta) {
    uint32_t got, x;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b128 r;\n\t"
        "ld.shared.b128 r, [%2];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
        "selp.u32 %0, 1, 0, p;\n\tmov.u32 %1, 0;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, _, _, _}, r;\n\t}\n"
        : "=r"(got), "=r"(x)
        : "r"(from)
        : "memory");
    cta = x;
    return got != 0;
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

// Deadline of waits that last a whole unit -- for the next unit, or for the end of this one in a role with little to do -- where the
// others last a block.  A unit of up to `blocks` streamed blocks takes some 4000 cycles for each: four times that, behind the
// usual second.  (64 heads to a key head and 2^20 tokens: 524288 blocks in a unit, more than a second.)  Nor is there a next unit
// at once where many sequences are empty: an SM asks for its share of the launch's `ctas` one after the other, some 900 cycles each.
inline long long unit_wait(long long blocks, long long ctas, int sms) { return ptx::WAIT_CYCLES + 16384 * (blocks + ctas / sms); }

// The largest power of two that divides the heads of a group, at most 16: so many heads of one token are rows of a
// query tile next to one another.
inline int packed_heads(int group) {
    int g = 1;
    while (g < 16 && group % (2 * g) == 0) g *= 2;
    return g;
}

}  // namespace packed
}  // namespace hilberta
