// Gradients of the attention over packed sequences, for sm_100a.  With P = exp(s q k^T - lse), dP = dO V^T,
// delta = rowsum(dO * O) and dS = P * (dP - delta):   dQ = s dS K,   dK = s dS^T Q,   dV = P^T dO.
//
// Two launches, three where key tiles are few (key_splits): a bandwidth-bound pass that leaves (lse log2 e, delta) of every
// row in the workspace, then one tensor-core kernel whose CTAs work in one of two modes:
//   mode DQ    resident tile = 128 query rows (Q_i, dO_i: 128 / g tokens of g heads, see the forward kernel),
//              streamed = their keys (K_j, V_j):   A = Q_i K_j^T, B = dO_i V_j^T, dS -> TMEM, dQ_i += dS K_j
//   mode DKV   resident tile = 128 keys (K_j, V_j), streamed = the query rows of the group's heads (or of a part of them) that see them:
//              A = K_j Q_i^T, B = V_j dO_i^T (a thread owns a KEY row), P^T, dS^T -> TMEM, dV_j += P^T dO_i, dK_j += dS^T Q_i
// Seven products where one pass that adds dQ up in memory would take five, but no atomics: every sum is taken in a
// fixed order, the heads of a group among them, and no fp32 copy of dQ is written and read.
// Sequences of up to 128 tokens: the statistics' delta carries the rounding of O to bf16, which a row of few keys
// feels most, its dS being a small difference; there all keys of a row are in one block, and the element-wise step takes
// delta = sum_j P_ij dP_ij itself.  (Error of dq against 64 bits, sequences of 2 ... 5 tokens 4.6e-3 and 2.5e-3 of the
// norm, 64 ... 77 tokens 3.1e-3 and 2.4e-3, 300 tokens 2.9e-3 and 2.5e-3.)
// P and dS are rounded to bf16 before the products over queries or keys, as the tensor cores take them; each in two parts, which
// would keep 16 bits, takes three products more than these seven.  (Gradients off by 2.4e-3 ... 2.9e-3 of their norm; rounding
// the results alone: 1.7e-3.)
// Bound by the chain dP -> phase 2 -> output products -> next dP: 2.1 us a block in DKV mode (four products, 1.5 at the matrix
// rate of a large library product), 1.4 in DQ mode (three, 1.1); tensor pipe 61 % of the cycles.  Measured (B200, us): four
// documents of 333 ... 4096 tokens, 16 heads over 4 key heads, causal, head dim 128: 300 (statistics 15 of it), with each mode's
// CTAs and their units fixed beforehand 379.  Few short prompts: 35 for eight of 1 ... 511 tokens, three heads to a key head, 30 of it
// 336 units of one to four blocks on 148 SMs.
// Per block the tensor pipe sees  A(s+1) | out(s) | B(s+1)  back to back: the element-wise step turns scores into
// weights as soon as A is written (phase 1) and frees A for the next block; phase 2 overwrites B in place with P and dS.
#include <algorithm>
#include <mutex>
#include <type_traits>

#include "attn_packed_tile.cuh"

namespace hilberta {
using namespace ptx;

namespace {

constexpr int BM = 128;   // resident rows
constexpr int BK = 128;   // streamed rows per block
constexpr int TILE_BYTES = BM * 128 * 2;
constexpr int SLAB_BYTES = TILE_BYTES / 2;
constexpr int NT1 = 3;    // ring of the streamed operand that is read twice
constexpr int NT2 = 2;    // ring of the streamed operand of dP
constexpr int UNITS = 2;
constexpr int STAT_BYTES = 2 * BK * 4;
constexpr int THREADS = 512;
constexpr uint32_t TMEM_COLS = 512;
constexpr int MODE_DQ = 0, MODE_DKV = 1;

enum Bar {
    RES_FULL = 0, RES_EMPTY, OUT_FULL, EPI_DONE, DRAIN,
    S_FULL, A_DONE, DP_FULL,
    P_READY,                      // [part]
    T1_FULL = P_READY + 2, T1_EMPTY = T1_FULL + NT1,
    T2_FULL = T1_EMPTY + NT1, T2_EMPTY = T2_FULL + NT2,
    SHORT = T2_EMPTY + NT2,       // the element-wise threads among themselves (256 arrivals)
    NEXT, WANT,                   // see the forward kernel
    U_FULL, U_EMPTY = U_FULL + UNITS,   // U_EMPTY: two producers, issuer, 8 element-wise and 4 epilogue warps
    NUM_BARS = U_EMPTY + UNITS
};
constexpr int UNIT_READERS = 15;

constexpr int OFF_R1 = 0, OFF_R2 = TILE_BYTES, OFF_T1 = 2 * TILE_BYTES, OFF_T2 = OFF_T1 + NT1 * TILE_BYTES;
constexpr int OFF_STAT = OFF_T2 + NT2 * TILE_BYTES;
constexpr int OFF_BARS = OFF_STAT + NT2 * STAT_BYTES;
constexpr int OFF_UNITS = OFF_BARS + NUM_BARS * 8;
constexpr int OFF_NEXT = (OFF_UNITS + UNITS * 20 + 15) / 16 * 16;
constexpr int OFF_MISC = OFF_NEXT + 16;
constexpr int SMEM_USED = OFF_MISC + 16;
constexpr int SMEM_BYTES = 232448;   // the 227 KB a CTA may have; SMEM_USED and the gap to a 1024-byte boundary must fit
static_assert(SMEM_USED <= SMEM_BYTES, "shared memory of one CTA");

__device__ int g_status[64];

struct Params {
    packed::Sequences queries, keys;   // blocks of a DQ unit (128 / g tokens) and of a DKV unit (128 tokens)
    int kv_heads, odd, group, g_shift, heads;   // group = odd << g_shift
    // DKV: the group's heads in `splits` parts of k_odd << k_shift, a unit each; more than one part leaves partial sums
    int splits, k_odd, k_shift;
    float *partial;   // [splits, 2 (dk, dv), total, kv_heads, head_dim], nullptr with one part
    unsigned dkv_units;   // CTAs of the launch that stand for units of the DKV mode
    const float *lse2, *delta;   // [total, heads]
    __nv_bfloat16 *dq, *dk, *dv;
    long long dq_t, dq_h, dk_t, dk_h, dv_t, dv_h;
    float scale, scale_log2;
    int align32;
    long long unit_wait;   // of waits that last a whole unit
};

// What every role derives from a unit.
struct Work {
    int row0, len;
    int tok0;          // first token of the resident tile
    int kv_head, head0;
    int first, count;  // streamed blocks of each of `reps` head parts: first ... first + count - 1
};
template <int MODE>
__device__ __forceinline__ Work work_of(const Params &p, const packed::Unit &u) {
    Work w;
    w.row0 = u.row0;
    w.len = u.len;
    if (MODE == MODE_DQ) {
        const int tpt = BM >> p.g_shift;
        w.tok0 = u.block * tpt;
        w.kv_head = u.head / p.odd;
        w.head0 = w.kv_head * p.group + ((u.head % p.odd) << p.g_shift);
        const int end = p.queries.causal ? min(w.len, w.tok0 + tpt) : w.len;
        w.first = 0;
        w.count = (end + BK - 1) / BK;
    } else {
        const int blocks = (w.len + BM - 1) / BM;
        // a causal level counts from the block with the fewest queries, the last one
        const int b = p.keys.causal ? blocks - 1 - u.block : u.block;
        w.tok0 = b * BM;
        w.kv_head = u.head / p.splits;
        w.head0 = w.kv_head * p.group + (u.head % p.splits) * (p.k_odd << p.k_shift);
        w.first = p.keys.causal ? b << p.k_shift : 0;
        w.count = (int)((((long long)w.len << p.k_shift) + BK - 1) / BK) - w.first;
    }
    return w;
}

template <int HD>
__device__ __forceinline__ void issue_rt(uint32_t tmem_acc, uint32_t sR, uint32_t sT) {
    constexpr uint32_t IDESC = idesc_bf16_f32(BM, BK, 0, 0);
    const uint64_t da = smem_desc_sw128(sR, 16, 1024), db = smem_desc_sw128(sT, 16, 1024);
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
        const uint64_t off = (uint64_t)(((k >> 2) * SLAB_BYTES + (k & 3) * 32) >> 4);
        mma_ss(tmem_acc, da + off, db + off, IDESC, k > 0);
    }
}

// out (+)= A T: A from TMEM; the bf16 pairs of streamed rows [32 g, 32 g + 32) sit 16 columns wide at column 32 g of
// region B (+ a_off); part 0 is g = 0, 2, part 1 g = 1, 3.
template <int HD>
__device__ __forceinline__ void issue_at(uint32_t tmem_out, uint32_t tmem_b, uint32_t a_off, uint32_t sT, int part, bool accumulate) {
    constexpr uint32_t IDESC = idesc_bf16_f32(BM, HD, 0, 1);
    const uint64_t db = smem_desc_sw128(sT, SLAB_BYTES, 1024);
#pragma unroll
    for (int i = 0; i < BK / 32; ++i) {
        const int k = (i >> 1) * 4 + part * 2 + (i & 1);
        mma_ts(tmem_out, tmem_b + (k >> 1) * 32 + a_off + (k & 1) * 8, db + (uint64_t)((k * 2048) >> 4), IDESC,
               (accumulate || part > 0 || i > 0) ? 1u : 0u);
    }
}

__device__ __forceinline__ void cp_async4(uint32_t dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// Every role goes through the CTA's units, DKV units and then DQ units, with code of its own for each mode; barriers and
// rings do not care which it is.
template <int HD>
__global__ void __launch_bounds__(THREADS, 1)
packed_bwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                  const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmdO,
                  const __grid_constant__ CUtensorMap tmQs, const __grid_constant__ CUtensorMap tmdOs,   // as DKV streams them
                  const __grid_constant__ Params prm) {
    extern __shared__ uint8_t smem_raw[];
    constexpr uint32_t REG_A = 0, REG_B = 128, OUT_A = 256, OUT_B = 384;   // TMEM columns
    constexpr int NSLAB = HD / 64;
    constexpr uint32_t TILE_TX = BM * HD * 2;

    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    if ((int)(smem - smem_raw) + SMEM_USED > SMEM_BYTES) {
        // the dynamic area starts too far from a 1024-byte boundary for everything to fit
        if (threadIdx.x == 0) atomicCAS(g_status, 0, 0x900);
        return;
    }
    const uint32_t sbase = smem_u32(smem);
    const uint32_t sR1 = sbase + OFF_R1, sR2 = sbase + OFF_R2, sT1 = sbase + OFF_T1, sT2 = sbase + OFF_T2;
    float *stats = reinterpret_cast<float *>(smem + OFF_STAT);
    const uint32_t bar0 = sbase + OFF_BARS;
    packed::Unit *const units = reinterpret_cast<packed::Unit *>(smem + OFF_UNITS);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + OFF_MISC);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + OFF_MISC + 4);
    int *const status = g_status;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g_shift = prm.g_shift;
    auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };

    if (tid == 0) {
        *abort_flag = 0;
        for (int i = 0; i < NUM_BARS; ++i) {
            uint32_t count = 1;
            if (i == EPI_DONE) count = 128;
            if (i == A_DONE || i == P_READY || i == P_READY + 1 || i == SHORT) count = 256;
            // ring 2 also carries the row statistics (DKV), copied by the 32 lanes of its producer warp
            if (i >= T2_FULL && i < T2_FULL + NT2) count = 33;
            if (i >= U_EMPTY) count = UNIT_READERS;
            mbar_init(bar(i), count);
        }
        mbar_fence_init();
    }
    if (warp == 8) {
        tmem_alloc(smem_u32(tmem_slot), TMEM_COLS);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    allow_next();
    wait_for_previous();
    const uint32_t tmem = *tmem_slot;

    // The next unit; whoever calls this with `release` has read it for its whole role or warp.
    uint32_t uc = 0;
    auto next_unit = [&](packed::Unit &u, bool release, int code) {
        const uint32_t s = uc % UNITS;
        if (!wait_or_abort(bar(U_FULL + s), (uc / UNITS) & 1, abort_flag, status, code, prm.unit_wait)) return false;
        u = units[s];
        ++uc;
        if (release) mbar_arrive(bar(U_EMPTY + s));
        return u.len >= 0;
    };

    using Dq = std::integral_constant<int, MODE_DQ>;
    using Dkv = std::integral_constant<int, MODE_DKV>;
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    }
    if (warp == 8 || warp == 10) {
        // ------------------------------------------------ producers of the streamed blocks
        // warp 8 feeds ring 1 (K_j in DQ mode, Q_i in DKV mode), warp 10 ring 2 (V_j / dO_i and, in DKV mode, the
        // statistics of the streamed query rows)
        const bool second = warp == 10;   // the whole warp takes part
        const bool leader = second ? lane == 0 : elect_one();
        if (leader || second) {
            const int nslot = second ? NT2 : NT1;
            const int FULL = second ? T2_FULL : T1_FULL, EMPTY = second ? T2_EMPTY : T1_EMPTY;
            const uint32_t ring = second ? sT2 : sT1;
            uint32_t g = 0;
            bool ok = true;
            auto stream = [&](auto mode, const packed::Unit &u) {
                constexpr int MODE = decltype(mode)::value;
                const CUtensorMap *tm = MODE == MODE_DKV ? (second ? &tmdOs : &tmQs) : (second ? &tmV : &tmK);
                const int g_shift = prm.k_shift;   // of the streamed rows, DKV
                const int tps = MODE == MODE_DKV ? BK >> g_shift : BK;   // tokens of a streamed block
                const Work w = work_of<MODE>(prm, u);
                // head parts that are streamed one after the other
                for (int rep = 0; ok && rep < (MODE == MODE_DKV ? prm.k_odd : 1); ++rep) {
                    const int head = MODE == MODE_DKV ? w.head0 + (rep << g_shift) : w.kv_head;
                    for (int j = 0; j < w.count; ++j, ++g) {
                        const int tok = (w.first + j) * tps;
                        const uint32_t s = g % nslot, ph = (g / nslot) & 1;
                        if (leader) ok = wait_or_abort(bar(EMPTY + s), ph ^ 1, abort_flag, status, 0x402 + (second ? 1 : 0));
                        if (second) ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
                        if (!ok) break;
                        if (leader) {
                            const uint32_t dst = ring + s * TILE_BYTES;
                            mbar_expect_tx(bar(FULL + s), TILE_TX);
#pragma unroll
                            for (int sl = 0; sl < NSLAB; ++sl)
                                tma_load_4d(dst + sl * SLAB_BYTES, tm, bar(FULL + s), 64 * sl, head, w.row0 + tok, 0);
                        }
                        if (second) {
                            // DKV: statistics of the block's rows that belong to the sequence (the others are masked by position
                            // later); the arrival fires when the copies land
                            const uint32_t sdst = sbase + OFF_STAT + s * STAT_BYTES;
#pragma unroll
                            for (int i = 0; MODE == MODE_DKV && i < BK / 32; ++i) {
                                const int c = lane + 32 * i, t = tok + (c >> g_shift);
                                if (t < w.len) {
                                    const long long at = (long long)(w.row0 + t) * prm.heads + head + (c & ((1 << g_shift) - 1));
                                    cp_async4(sdst + 4 * c, prm.lse2 + at);
                                    cp_async4(sdst + 4 * (BK + c), prm.delta + at);
                                }
                            }
                            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar(FULL + s)) : "memory");
                        }
                    }
                }
            };
            packed::Unit u;
            for (;;) {
                ok = next_unit(u, false, 0x400 + (second ? 1 : 0));
                if (second) ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (leader) mbar_arrive(bar(U_EMPTY + (uc - 1) % UNITS));
                if (u.mode == MODE_DKV) stream(Dkv{}, u);
                else stream(Dq{}, u);
                if (!ok) break;
                if (leader && !second) mbar_arrive(bar(WANT));
            }
            if (second) asm volatile("cp.async.wait_all;" ::: "memory");
            if (*abort_flag && leader) {
                // let every copy already issued land before the CTA retires
                const long long t0 = clock64();
                while (clock64() - t0 < 2000000) {
                }
            }
        }
    } else if (warp == 11) {
        // ------------------------------------------------ finds the units and loads their resident tiles
        if (lane == 0) {
            prefetch_tmap(&tmQ);
            prefetch_tmap(&tmK);
            prefetch_tmap(&tmV);
            prefetch_tmap(&tmdO);
            prefetch_tmap(&tmQs);
            prefetch_tmap(&tmdOs);
        }
        packed::Runs key_runs, query_runs;
        const packed::Span key_span = packed::span_of(prm.keys, lane), query_span = packed::span_of(prm.queries, lane);
        const uint32_t next = sbase + OFF_NEXT;
        unsigned n = blockIdx.x;
        uint32_t asked = 0;
        bool more = true, ok = true;
        auto find = [&](packed::Unit &u) {
            u.mode = n < prm.dkv_units ? MODE_DKV : MODE_DQ;
            return n < prm.dkv_units ? packed::find_unit(prm.keys, key_span, key_runs, prm.kv_heads * prm.splits, n, u)
                                     : packed::find_unit(prm.queries, query_span, query_runs, prm.kv_heads * prm.odd, n - prm.dkv_units, u);
        };
        auto ask_next = [&] {
            if (lane == 0) {
                fence_proxy_async_smem();   // the last answer has been read
                packed::ask_next_cta(next, bar(NEXT));
                ok = wait_or_abort(bar(NEXT), asked & 1, abort_flag, status, 0x407);
                if (ok) more = packed::next_cta(next, n);
            }
            ++asked;
            n = __shfl_sync(0xffffffffu, n, 0);
            more = __shfl_sync(0xffffffffu, (int)more, 0) != 0;
            ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
        };
        for (uint32_t i = 0; ok; ++i) {
            packed::Unit u;
            // the launch has a CTA for every unit there may be; some are not there
            bool found = more && find(u);
            while (ok && more && !found) {
                ask_next();
                found = ok && more && find(u);
            }
            if (!ok) break;
            if (!found) u.len = -1;
            if (lane == 0) {
                const uint32_t s = i % UNITS;
                ok = wait_or_abort(bar(U_EMPTY + s), ((i / UNITS) & 1) ^ 1, abort_flag, status, 0x406, prm.unit_wait);
                if (ok) {
                    units[s] = u;
                    mbar_arrive(bar(U_FULL + s));
                    // free once the last R T^T MMA of the previous unit has retired
                    if (found && i > 0) ok = wait_or_abort(bar(RES_EMPTY), (i - 1) & 1, abort_flag, status, 0x401, prm.unit_wait);
                    if (found && ok) {
                        const bool dkv = u.mode == MODE_DKV;
                        const Work w = dkv ? work_of<MODE_DKV>(prm, u) : work_of<MODE_DQ>(prm, u);
                        const int head = dkv ? w.kv_head : w.head0;
                        mbar_expect_tx(bar(RES_FULL), 2 * TILE_TX);
#pragma unroll
                        for (int sl = 0; sl < NSLAB; ++sl) {
                            tma_load_4d(sR1 + sl * SLAB_BYTES, dkv ? &tmK : &tmQ, bar(RES_FULL), 64 * sl, head, w.row0 + w.tok0, 0);
                            tma_load_4d(sR2 + sl * SLAB_BYTES, dkv ? &tmV : &tmdO, bar(RES_FULL), 64 * sl, head, w.row0 + w.tok0, 0);
                        }
                        // not before the producer is through with this unit: one that another CTA could start sooner is left to it
                        ok = wait_or_abort(bar(WANT), i & 1, abort_flag, status, 0x408, prm.unit_wait);
                    }
                }
            }
            ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
            if (!found || !ok) break;
            ask_next();
        }
        if (*abort_flag && lane == 0) {
            const long long t0 = clock64();
            while (clock64() - t0 < 2000000) {
            }
        }
    } else if (warp >= 12) {
        // ------------------------------------------------ epilogue: accumulators -> bf16 -> global
        // Its own warpgroup, so that the element-wise warps move on to the next unit at once.
        const int r = tid & 127;
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        bool ok = true;
        packed::Unit u;
        for (uint32_t n = 0;; ++n) {
            ok = next_unit(u, false, 0x600);
            __syncwarp();
            if (!ok) break;
            if (lane == 0) mbar_arrive(bar(U_EMPTY + (uc - 1) % UNITS));
            ok = wait_or_abort(bar(OUT_FULL), n & 1, abort_flag, status, 0x607, prm.unit_wait);
            if (!ok) break;
            tc_fence_after();
            auto store = [&](auto mode) {
                constexpr int MODE = decltype(mode)::value;
                const Work w = work_of<MODE>(prm, u);
                const int tok = w.tok0 + (MODE == MODE_DQ ? r >> g_shift : r);
                const int head = MODE == MODE_DQ ? w.head0 + (r & ((1 << g_shift) - 1)) : w.kv_head;
                const long long row = w.row0 + tok;
                __nv_bfloat16 *const out_a = MODE == MODE_DQ ? prm.dq + row * prm.dq_t + head * prm.dq_h : prm.dk + row * prm.dk_t + head * prm.dk_h;
                __nv_bfloat16 *const out_b = prm.dv + row * prm.dv_t + head * prm.dv_h;
                constexpr int CPO = HD / 32;                              // 32-column chunks per output
                constexpr int NCH = (MODE == MODE_DKV) ? 2 * CPO : CPO;   // DKV: dK then dV
#pragma unroll
                for (int c = 0; c < NCH; ++c) {
                    uint32_t o[32];
                    tmem_ld32(tmem + lane_addr + (c >= CPO ? OUT_B + (c - CPO) * 32 : OUT_A + c * 32), o);
                    tmem_wait_ld();
                    if (tok < w.len && MODE == MODE_DKV && prm.partial) {
                        const long long which = (u.head % prm.splits) * 2 + (c >= CPO ? 1 : 0);
                        float *const to = prm.partial + ((which * prm.keys.total + row) * prm.kv_heads + head) * HD + (c % CPO) * 32;
#pragma unroll
                        for (int i = 0; i < 32; i += 4) *reinterpret_cast<uint4 *>(to + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    } else if (tok < w.len) {
                        __nv_bfloat16 *orow = (c >= CPO ? out_b : out_a) + (c % CPO) * 32;
                        const float mul = c >= CPO ? 1.f : prm.scale;
                        uint32_t v[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            v[i] = pack_bf16(__uint_as_float(o[2 * i]) * mul, __uint_as_float(o[2 * i + 1]) * mul);
                        if (prm.align32) {
                            st_global_v8(orow, v);
                            st_global_v8(orow + 16, v + 8);
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; i += 4)
                                *reinterpret_cast<uint4 *>(orow + 2 * i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                        }
                    }
                }
            };
            if (u.mode == MODE_DKV) store(Dkv{});
            else store(Dq{});
            tc_fence_before();
            mbar_arrive(bar(EPI_DONE));
        }
    } else if (warp == 9) {
        // ---------------------------------------------------------- MMA issuer
        if (elect_one()) {
            uint32_t g = 0, n_unit = 0;   // g: blocks issued so far (ring positions and barrier phases)
            bool ok = true;
            auto t1 = [&](uint32_t e) { return sT1 + (e % NT1) * TILE_BYTES; };
            auto t2 = [&](uint32_t e) { return sT2 + (e % NT2) * TILE_BYTES; };
            auto multiply = [&](auto mode, const packed::Unit &u) {
                constexpr int MODE = decltype(mode)::value;
                const int n = work_of<MODE>(prm, u).count * (MODE == MODE_DKV ? prm.k_odd : 1);
                ok = wait_or_abort(bar(RES_FULL), n_unit & 1, abort_flag, status, 0x501);
                if (!ok) return;
                // scores and dP of the first block
                ok = wait_or_abort(bar(T1_FULL + g % NT1), (g / NT1) & 1, abort_flag, status, 0x502);
                if (!ok) return;
                tc_fence_after();
                issue_rt<HD>(tmem + REG_A, sR1, t1(g));
                mma_commit(bar(S_FULL));
                ok = wait_or_abort(bar(T2_FULL + g % NT2), (g / NT2) & 1, abort_flag, status, 0x503);
                if (!ok) return;
                tc_fence_after();
                issue_rt<HD>(tmem + REG_B, sR2, t2(g));
                mma_commit(bar(DP_FULL));
                if (MODE == MODE_DQ) mma_commit(bar(T2_EMPTY + g % NT2));
                if (n == 1) mma_commit(bar(RES_EMPTY));
                for (int s = 0; s < n; ++s) {
                    const uint32_t e = g + s;
                    const bool more = s + 1 < n;
                    if (more) {
                        // scores of the next block, as soon as phase 1 has read this block's
                        ok = wait_or_abort(bar(T1_FULL + (e + 1) % NT1), ((e + 1) / NT1) & 1, abort_flag, status, 0x504);
                        if (!ok) break;
                        ok = wait_or_abort(bar(A_DONE), e & 1, abort_flag, status, 0x505);
                        if (!ok) break;
                        tc_fence_after();
                        issue_rt<HD>(tmem + REG_A, sR1, t1(e + 1));
                        mma_commit(bar(S_FULL));
                    }
                    if (s == 0 && n_unit > 0) {
                        // the previous unit's accumulators have been read out
                        ok = wait_or_abort(bar(EPI_DONE), (n_unit - 1) & 1, abort_flag, status, 0x506);
                        if (!ok) break;
                    }
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        ok = wait_or_abort(bar(P_READY + part), e & 1, abort_flag, status, 0x507);
                        if (!ok) break;
                        tc_fence_after();
                        issue_at<HD>(tmem + OUT_A, tmem + REG_B, 16, t1(e), part, s > 0);                       // dS  x T1
                        if (MODE == MODE_DKV) issue_at<HD>(tmem + OUT_B, tmem + REG_B, 0, t2(e), part, s > 0);   // P^T x T2
                    }
                    if (!ok) break;
                    mma_commit(bar(T1_EMPTY + e % NT1));
                    if (MODE == MODE_DKV) mma_commit(bar(T2_EMPTY + e % NT2));
                    if (more) {
                        // dP of the next block overwrites P / dS of this one: after the MMAs above
                        ok = wait_or_abort(bar(T2_FULL + (e + 1) % NT2), ((e + 1) / NT2) & 1, abort_flag, status, 0x508);
                        if (!ok) break;
                        tc_fence_after();
                        issue_rt<HD>(tmem + REG_B, sR2, t2(e + 1));
                        mma_commit(bar(DP_FULL));
                        if (MODE == MODE_DQ) mma_commit(bar(T2_EMPTY + (e + 1) % NT2));
                        if (s + 2 == n) mma_commit(bar(RES_EMPTY));   // last read of the resident tiles
                    }
                }
                if (!ok) return;
                mma_commit(bar(OUT_FULL));
                g += n;
            };
            packed::Unit u;
            for (; ok && next_unit(u, true, 0x500); ++n_unit) {
                if (u.mode == MODE_DKV) multiply(Dkv{}, u);
                else multiply(Dq{}, u);
            }
            // every MMA issued above has retired before TMEM is released
            mma_commit(bar(DRAIN));
            wait_or_abort(bar(DRAIN), 0, abort_flag, status, 0x509);
        }
    } else if (warp < 8) {
        // ------------------------------------ element-wise step, warpgroup wg: columns [64 wg, +64)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
        const int wg = warp >> 2;
        const int r = tid & 127;
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tA = tmem + lane_addr + REG_A + wg * 64, tB = tmem + lane_addr + REG_B + wg * 64;
        const float scale_log2 = prm.scale_log2;
        uint32_t g = 0, n_short = 0;
        bool ok = true;
        packed::Unit u;
        auto meet = [&] {   // all element-wise threads
            mbar_arrive(bar(SHORT));
            return wait_or_abort(bar(SHORT), n_short++ & 1, abort_flag, status, 0x608);
        };
        while (ok) {
            const bool any = next_unit(u, false, 0x601);
            __syncwarp();
            if (!any) break;
            if (lane == 0) mbar_arrive(bar(U_EMPTY + (uc - 1) % UNITS));
            auto weigh = [&](auto mode) {
                constexpr int MODE = decltype(mode)::value;
                const Work w = work_of<MODE>(prm, u);
                // DQ: this thread's query row; rows behind the sequence get lse = +inf, which turns their weights into zeros
                float row_l2 = __int_as_float(0x7f800000), row_dl = 0.f;
                const int tok = w.tok0 + (MODE == MODE_DQ ? r >> g_shift : r);   // the query's (DQ) or the key's (DKV) token
                if (MODE == MODE_DQ && tok < w.len) {
                    const long long at = (long long)(w.row0 + tok) * prm.heads + w.head0 + (r & ((1 << g_shift) - 1));
                    row_l2 = prm.lse2[at];   // plain loads: the kernel before this one writes them while this one starts
                    row_dl = prm.delta[at];
                }
                for (int rep = 0; ok && rep < (MODE == MODE_DKV ? prm.k_odd : 1); ++rep) {
                    for (int j = 0; j < w.count; ++j, ++g) {
                        // Pairs that exist: streamed columns lo <= c < hi of this warpgroup's 64; dS is zero below lo_ds
                        // (and above hi_ds) too, since a query with one key has no gradient through its weight of one.
                        int lo = 0, hi = 64, lo_ds = 0, hi_ds = 64, beyond;   // beyond: the block's rows of the sequence
                        bool masked;
                        if (MODE == MODE_DQ) {
                            beyond = w.len - j * BK;
                            const int end = (prm.queries.causal ? min(tok + 1, w.len) : w.len);
                            masked = (j + 1) * BK > (prm.queries.causal ? min(w.tok0 + 1, w.len) : w.len);
                            hi = end - j * BK - wg * 64;
                            hi_ds = end == 1 ? 0 : hi;
                        } else {
                            const int k_shift = prm.k_shift, t0 = (w.first + j) << (7 - k_shift);
                            beyond = (w.len - t0) << k_shift;
                            masked = beyond < BK || w.len == 1;
                            hi = beyond - wg * 64;
                            if (prm.keys.causal) {
                                masked |= t0 < w.tok0 + BM;
                                lo = (tok - t0) * (1 << k_shift) - wg * 64;
                                lo_ds = max(lo, (1 - t0) * (1 << k_shift) - wg * 64);
                            } else if (w.len == 1) {
                                lo_ds = 64;
                            }
                        }
                        float *const slot = stats + (g % NT2) * (2 * BK);   // DKV: lse2, then delta
                        const float4 *const st_l = reinterpret_cast<const float4 *>(slot + wg * 64), *const st_d = st_l + BK / 4;
                        if (MODE == MODE_DKV) {
                            // the statistics arrive with ring 2
                            ok = wait_or_abort(bar(T2_FULL + g % NT2), (g / NT2) & 1, abort_flag, status, 0x602);
                            if (!ok) break;
                        }
                        // ---- phase 1: weights from the scores
                        ok = wait_or_abort(bar(S_FULL), g & 1, abort_flag, status, 0x603 + wg);
                        if (!ok) break;
                        tc_fence_after();
                        uint32_t a[64];
                        tmem_ld32(tA, *reinterpret_cast<uint32_t(*)[32]>(&a[0]));
                        tmem_ld32(tA + 32, *reinterpret_cast<uint32_t(*)[32]>(&a[32]));
                        tmem_wait_ld();
                        tc_fence_before();
                        mbar_arrive(bar(A_DONE));   // region A may take the next block's scores
                        auto phase1 = [&](auto MASKED) {
#pragma unroll
                            for (int c4 = 0; c4 < 16; ++c4) {
                                float4 l4 = make_float4(row_l2, row_l2, row_l2, row_l2);
                                if (MODE == MODE_DKV) l4 = st_l[c4];
                                const float2 x0 = __ffma2_rn(make_float2(__uint_as_float(a[4 * c4]), __uint_as_float(a[4 * c4 + 1])),
                                                             make_float2(scale_log2, scale_log2), make_float2(-l4.x, -l4.y));
                                const float2 x1 = __ffma2_rn(make_float2(__uint_as_float(a[4 * c4 + 2]), __uint_as_float(a[4 * c4 + 3])),
                                                             make_float2(scale_log2, scale_log2), make_float2(-l4.z, -l4.w));
                                float p[4] = {ex2(x0.x), ex2(x0.y), ex2(x1.x), ex2(x1.y)};
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    if (decltype(MASKED)::value && (4 * c4 + i < lo || 4 * c4 + i >= hi)) p[i] = 0.f;
                                    a[4 * c4 + i] = __float_as_uint(p[i]);
                                }
                            }
                        };
                        if (masked) phase1(std::true_type{});
                        else phase1(std::false_type{});
                        // ---- phase 2: dS = P * (dP - delta), written over dP together with P
                        ok = wait_or_abort(bar(DP_FULL), g & 1, abort_flag, status, 0x605 + wg);
                        if (!ok) break;
                        tc_fence_after();
                        if (beyond < BK) {
                            // Streamed rows behind the sequence belong to others: weights and dS are zero there, and so
                            // are the rows themselves from here on, whatever they hold.  Both products that read them
                            // for A and B are done; those that multiply them by zeros wait for P_READY.
                            if ((MODE == MODE_DKV || wg == 0) && r >= beyond) {
                                const uint32_t base = (wg == 0 ? sT1 + (g % NT1) * TILE_BYTES : sT2 + (g % NT2) * TILE_BYTES) + r * 128;
                                const uint32_t zero[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                                for (int c = 0; c < NSLAB * 8; ++c) st_shared_v4(base + (c >> 3) * SLAB_BYTES + (c & 7) * 16, zero);
                            }
                            fence_proxy_async_smem();
                        }
                        const bool exact = w.len <= BK;   // the row's or column's delta from this block alone
                        if (exact) {
                            float sum[2] = {0.f, 0.f};   // DQ: of this row; DKV: of columns lane and 32 + lane over this warp's keys
#pragma unroll
                            for (int h2 = 0; h2 < 2; ++h2) {
                                uint32_t d[32];
                                float x[32];
                                tmem_ld32(tB + h2 * 32, d);
                                tmem_wait_ld();
#pragma unroll
                                for (int i = 0; i < 32; ++i) {
                                    // a weight of zero, whatever the other factor; keys behind the sequence count for nothing
                                    const float p = __uint_as_float(a[h2 * 32 + i]);
                                    x[i] = p == 0.f || (MODE == MODE_DKV && tok >= w.len) ? 0.f : p * __uint_as_float(d[i]);
                                }
                                if (MODE == MODE_DQ) {
#pragma unroll
                                    for (int i = 0; i < 32; ++i) sum[0] += x[i];
                                } else {
                                    // lane c is left with the sum of column c: each step hands half of the columns over
#pragma unroll
                                    for (int o = 16; o > 0; o >>= 1) {
                                        const bool up = (lane & o) != 0;
#pragma unroll
                                        for (int i = 0; i < o; ++i) {
                                            const float keep = up ? x[i + o] : x[i], give = up ? x[i] : x[i + o];
                                            x[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                                        }
                                    }
                                    sum[h2] = x[0];
                                }
                            }
                            if (MODE == MODE_DQ) {
                                // the other 64 columns' sum through tensor memory, in the place of this thread's first dP for a while
                                const uint32_t dp0 = tmem_ld1(tB);
                                tmem_wait_ld();
                                tmem_st1(tB, __float_as_uint(sum[0]));
                                tmem_wait_st();
                                tc_fence_before();
                                ok = meet();
                                if (!ok) break;
                                tc_fence_after();
                                const uint32_t other = tmem_ld1(tmem + lane_addr + REG_B + (1 - wg) * 64);
                                tmem_wait_ld();
                                tc_fence_before();
                                ok = meet();
                                if (!ok) break;
                                tc_fence_after();
                                tmem_st1(tB, dp0);
                                tmem_wait_st();
                                row_dl = wg ? __uint_as_float(other) + sum[0] : sum[0] + __uint_as_float(other);
                            } else {
                                // four warps' sums become two in the place of lse2 and delta, which nobody needs any more
                                float *const to = slot + (warp & 1) * BK + wg * 64 + lane;
                                ok = meet();
                                if (!ok) break;
                                if ((warp & 2) == 0) to[0] = sum[0], to[32] = sum[1];
                                ok = meet();
                                if (!ok) break;
                                if ((warp & 2) != 0) to[0] += sum[0], to[32] += sum[1];
                                ok = meet();
                                if (!ok) break;
                            }
                        }
                        auto phase2 = [&](auto MASKED) {
#pragma unroll
                            for (int h2 = 0; h2 < 2; ++h2) {
                                uint32_t d[32];
                                tmem_ld32(tB + h2 * 32, d);
                                tmem_wait_ld();
                                uint32_t pk[16], dk[16];
#pragma unroll
                                for (int i4 = 0; i4 < 8; ++i4) {
                                    const int c0 = h2 * 32 + 4 * i4;
                                    float4 d4 = make_float4(row_dl, row_dl, row_dl, row_dl);
                                    if (MODE == MODE_DKV) {
                                        d4 = st_d[c0 >> 2];
                                        if (decltype(MASKED)::value && exact) {
                                            const float4 e4 = st_l[c0 >> 2];
                                            d4.x += e4.x, d4.y += e4.y, d4.z += e4.z, d4.w += e4.w;
                                        }
                                    }
                                    const float2 pa = make_float2(__uint_as_float(a[c0]), __uint_as_float(a[c0 + 1]));
                                    const float2 pb = make_float2(__uint_as_float(a[c0 + 2]), __uint_as_float(a[c0 + 3]));
                                    const float2 sa = __fmul2_rn(__fadd2_rn(make_float2(__uint_as_float(d[4 * i4]), __uint_as_float(d[4 * i4 + 1])),
                                                                            make_float2(-d4.x, -d4.y)), pa);
                                    const float2 sb = __fmul2_rn(__fadd2_rn(make_float2(__uint_as_float(d[4 * i4 + 2]), __uint_as_float(d[4 * i4 + 3])),
                                                                            make_float2(-d4.z, -d4.w)), pb);
                                    float s[4] = {sa.x, sa.y, sb.x, sb.y};
                                    if (decltype(MASKED)::value) {
                                        // P is zero there already; dP - delta may be anything
#pragma unroll
                                        for (int i = 0; i < 4; ++i)
                                            if (c0 + i < max(lo, lo_ds) || c0 + i >= min(hi, hi_ds)) s[i] = 0.f;
                                    }
                                    pk[2 * i4] = pack_bf16(pa.x, pa.y);
                                    pk[2 * i4 + 1] = pack_bf16(pb.x, pb.y);
                                    dk[2 * i4] = pack_bf16(s[0], s[1]);
                                    dk[2 * i4 + 1] = pack_bf16(s[2], s[3]);
                                }
                                // the 32 columns just read take P (16 columns of bf16 pairs) and dS (16)
                                if (MODE == MODE_DKV) tmem_st16(tB + h2 * 32, pk);
                                tmem_st16(tB + h2 * 32 + 16, dk);
                                tmem_wait_st();
                                tc_fence_before();
                                mbar_arrive(bar(P_READY + h2));
                            }
                        };
                        if (masked || exact) phase2(std::true_type{});
                        else phase2(std::false_type{});
                    }
                }
            };
            if (u.mode == MODE_DKV) weigh(Dkv{});
            else weigh(Dq{});
        }
    }

    tc_fence_before();
    __syncthreads();
    __syncwarp();
    if (warp == 8) tmem_dealloc(tmem, TMEM_COLS);
}

// lse2[t, h] = lse[h, t] * log2 e, delta[t, h] = sum_d dO[t, h, d] * O[t, h, d]: HD / 8 lanes per row (16 bytes each),
// four rows in flight per lane group.  Rows outside the sequences are read like the others and used by nobody.
template <int HD>
__global__ void __launch_bounds__(256)
packed_delta_kernel(const __nv_bfloat16 *dout, const __nv_bfloat16 *out, const float *lse, float *lse2, float *delta, int total, Divider heads,
                    long long do_t, long long do_h, long long o_t, long long o_h) {
    constexpr int LPR = HD / 8;
    const unsigned sub = threadIdx.x % LPR, n_rows = (unsigned)total * heads.d;   // below 2^31, see the host
    const unsigned row0 = (blockIdx.x * (256 / LPR) + threadIdx.x / LPR) * 4;
    unsigned t[4], h[4];
    t[0] = heads.quotient(row0);
    h[0] = row0 - t[0] * heads.d;
#pragma unroll
    for (int i = 1; i < 4; ++i) {
        const bool wrap = h[i - 1] + 1 == heads.d;
        h[i] = wrap ? 0 : h[i - 1] + 1;
        t[i] = t[i - 1] + (wrap ? 1 : 0);
    }
    uint4 a[4], c[4];
    float l[4];
    allow_next();
    wait_for_previous();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = c[i] = make_uint4(0u, 0u, 0u, 0u);
        l[i] = 0.f;
        if (row0 + i < n_rows) {
            a[i] = *reinterpret_cast<const uint4 *>(dout + t[i] * do_t + h[i] * do_h + sub * 8);
            c[i] = *reinterpret_cast<const uint4 *>(out + t[i] * o_t + h[i] * o_h + sub * 8);
            if (sub == 0) l[i] = lse[(long long)h[i] * total + t[i]];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float acc = 0.f;
        const uint32_t *ua = reinterpret_cast<const uint32_t *>(&a[i]), *uc = reinterpret_cast<const uint32_t *>(&c[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&ua[e]));
            const float2 y = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&uc[e]));
            acc = fmaf(x.x, y.x, fmaf(x.y, y.y, acc));
        }
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
        if (row0 + i < n_rows && sub == 0) {
            lse2[row0 + i] = l[i] * 1.4426950408889634f;
            delta[row0 + i] = acc;
        }
    }
}

// dk, dv of the sequences' rows from the parts' sums, in the parts' order: four columns a thread.
template <int HD>
__global__ void __launch_bounds__(256)
packed_sum_kernel(const float *partial, const int *cu, int n_seq, __nv_bfloat16 *dk, __nv_bfloat16 *dv, int splits, int total, Divider kv_heads,
                  long long dk_t, long long dk_h, long long dv_t, long long dv_h, float scale) {
    const unsigned at = blockIdx.x * 256 + threadIdx.x, row = at / (HD / 4), c = at % (HD / 4) * 4, which = blockIdx.y;
    const unsigned t = kv_heads.quotient(row), h = row - t * kv_heads.d;
    allow_next();
    wait_for_previous();
    // rows between the first sequence's first and the last one's last belong to one of them
    if ((int)t < max(cu[0], 0) || (int)t >= min(cu[n_seq], total)) return;
    const long long size = (long long)total * kv_heads.d * HD;
    const float *p = partial + which * size + (long long)row * HD + c;
    float4 a = *reinterpret_cast<const float4 *>(p);
    for (int i = 1; i < splits; ++i) {
        const float4 b = *reinterpret_cast<const float4 *>(p + 2 * size * i);
        a.x += b.x, a.y += b.y, a.z += b.z, a.w += b.w;
    }
    const float mul = which ? 1.f : scale;
    __nv_bfloat16 *const to = which ? dv + t * dv_t + h * dv_h + c : dk + t * dk_t + h * dk_h + c;
    *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(a.x * mul, a.y * mul), pack_bf16(a.z * mul, a.w * mul));
}

// Into how many parts DKV units take the group's heads.  Few key tiles with many heads would leave SMs idle while the longest
// streams all heads' queries one after the other: a unit an SM is wanted, the smallest divisor of the group that gives it.  More
// cost partial sums in memory and a launch to add them up; eight units an SM are the most, which bounds the sums to 155 MB where
// the group's next divisor is a large one.  A sequence of one block gains nothing.  (4096 tokens, eight heads and one key head,
// causal, us: one part 464, four 154, eight 121; eight prompts of 1 ... 511 tokens, three heads to a key head: one 41, three 35;
// 2048 tokens, 32 heads over 8, causal, 153 in one part: 139 in two, 161 in four.)
int key_splits(long long total, int n_seq, int heads, int kv_heads, int sms) {
    const int group = heads / kv_heads;
    if (total <= BM) return 1;
    const long long units = (total / BM + std::min((long long)n_seq, total)) * kv_heads;
    const long long most = std::min((long long)group, 8ll * sms / units);
    int splits = 1;
    for (int i = 2; i <= most && units * splits < sms; ++i)
        if (group % i == 0) splits = i;
    return splits;
}

constexpr size_t statistics_bytes(long long total, long long heads) { return (2 * (size_t)total * (size_t)heads * sizeof(float) + 255) / 256 * 256; }

int opt_in(int device) {
    static std::mutex mutex;
    static bool done[64] = {};
    std::lock_guard<std::mutex> lock(mutex);
    if (device < 0 || device >= 64) return HILBERTA_ERR_INVALID;
    if (done[device]) return HILBERTA_OK;
    HB_CUDA(cudaFuncSetAttribute(packed_bwd_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES));
    HB_CUDA(cudaFuncSetAttribute(packed_bwd_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES));
    done[device] = true;
    return HILBERTA_OK;
}

}  // namespace

int packed::backward_status(bool *expired) {
    int code = 0;
    HB_CUDA(cudaMemcpyFromSymbol(&code, g_status, sizeof(int)));
    if (code) {
        const int zero[3] = {0, 0, 0};
        HB_CUDA(cudaMemcpyToSymbol(g_status, zero, sizeof(zero)));
        *expired = true;
    }
    return HILBERTA_OK;
}

}  // namespace hilberta

using namespace hilberta;

extern "C" size_t hilberta_packed_workspace(int total, int heads) {
    if (total <= 0 || heads <= 0) return 0;
    // statistics of every row; where key tiles are few, partial sums: the most that any number of key heads and sequences takes
    const size_t stats = 2 * (size_t)total * (size_t)heads * sizeof(float);
    int dev = -1;
    const int sms = cudaGetDevice(&dev) == cudaSuccess ? sm100_count(dev) : 0;
    size_t most = 0;
    for (int kv = 1; kv <= heads && kv < sms; ++kv) {
        if (heads % kv) continue;
        const int splits = key_splits(total, 1, heads, kv, sms);
        if (splits > 1) most = std::max(most, (size_t)splits * 2 * (size_t)total * (size_t)kv * 128 * sizeof(float));
    }
    return most ? statistics_bytes(total, heads) + most : stats;
}

extern "C" int hilberta_packed_backward(const void *dout, const void *q, const void *k, const void *v, const void *out, const float *lse,
                                        void *dq, void *dk, void *dv, void *workspace, size_t workspace_bytes, const int32_t *cu_seqlens,
                                        int n_seq, int total, int heads, int kv_heads, int head_dim, int dtype, const int64_t *strides,
                                        int causal, float scale, void *stream) {
    const void *tensors[8] = {dout, q, k, v, out, dq, dk, dv};
    const int n_heads[8] = {heads, heads, kv_heads, kv_heads, heads, heads, kv_heads, kv_heads};
    int rc = packed::check(tensors, 8, strides, cu_seqlens, n_seq, total, heads, kv_heads, head_dim, dtype);
    if (rc != HILBERTA_OK) return rc;
    const bool none = total == 0 || n_seq == 0;
    if (((uintptr_t)lse & 3) || ((uintptr_t)workspace & 15) || !(scale == scale) || (!none && !lse)) return HILBERTA_ERR_INVALID;
    for (int i = 5; !none && i < 8; ++i)
        for (int j = 0; j < i; ++j)
            if (packed::overlap(tensors[i], strides + 2 * i, n_heads[i], tensors[j], strides + 2 * j, n_heads[j], total, head_dim))
                return HILBERTA_ERR_INVALID;
    if (!none && (!workspace || workspace_bytes < hilberta_packed_workspace(total, heads))) return HILBERTA_ERR_BUFFER;
    int dev = -1;
    HB_CUDA(cudaGetDevice(&dev));
    const int sms = sm100_count(dev);
    if (!sms) return HILBERTA_ERR_ARCH;
    if (none) return HILBERTA_OK;
    if ((rc = opt_in(dev)) != HILBERTA_OK) return rc;

    Params p;
    p.kv_heads = kv_heads;
    p.heads = heads;
    p.group = heads / kv_heads;
    const int g = packed::packed_heads(p.group), per_tile = BM / g;
    p.g_shift = __builtin_ctz((unsigned)g);
    p.odd = p.group / g;
    p.queries = {cu_seqlens, n_seq, total, __builtin_ctz((unsigned)per_tile), causal != 0};
    p.keys = {cu_seqlens, n_seq, total, 7, causal != 0};
    float *lse2 = (float *)workspace, *delta = lse2 + (size_t)total * heads;
    p.lse2 = lse2;
    p.delta = delta;
    p.dq = (__nv_bfloat16 *)dq;
    p.dk = (__nv_bfloat16 *)dk;
    p.dv = (__nv_bfloat16 *)dv;
    p.dq_t = strides[10], p.dq_h = strides[11];
    p.dk_t = strides[12], p.dk_h = strides[13];
    p.dv_t = strides[14], p.dv_h = strides[15];
    p.scale = scale > 0.f ? scale : 1.f / sqrtf((float)head_dim);
    p.scale_log2 = p.scale * 1.4426950408889634f;
    int64_t bits = (int64_t)((uintptr_t)dq | (uintptr_t)dk | (uintptr_t)dv);
    for (int i = 10; i < 16; ++i) bits |= 2 * strides[i];
    p.align32 = (bits & 31) == 0;
    p.splits = key_splits(total, n_seq, heads, kv_heads, sms);
    const int k_heads = p.group / p.splits, gk = packed::packed_heads(k_heads);
    p.k_shift = __builtin_ctz((unsigned)gk);
    p.k_odd = k_heads / gk;
    auto units = [&](int per, int parts) { return (unsigned)(((long long)total / per + std::min(n_seq, total)) * parts); };   // at most
    p.dkv_units = units(BM, kv_heads * p.splits);
    const unsigned ctas = p.dkv_units + units(per_tile, kv_heads * p.odd);
    // blocks of the longest unit there may be: keys of a query tile, or queries of the heads of a key tile
    p.unit_wait = packed::unit_wait((((long long)total << p.k_shift) + BK - 1) / BK * p.k_odd, ctas, sms);
    p.partial = p.splits > 1 ? (float *)((char *)workspace + statistics_bytes(total, heads)) : nullptr;
    CUtensorMap mq, mk, mv, mdo, mqs, mdos;
    if ((rc = packed::make_map(&mdo, dout, total, heads, head_dim, strides[0], strides[1], g, per_tile)) != HILBERTA_OK) return rc;
    if ((rc = packed::make_map(&mq, q, total, heads, head_dim, strides[2], strides[3], g, per_tile)) != HILBERTA_OK) return rc;
    if ((rc = packed::make_map(&mk, k, total, kv_heads, head_dim, strides[4], strides[5], 1, BM)) != HILBERTA_OK) return rc;
    if ((rc = packed::make_map(&mv, v, total, kv_heads, head_dim, strides[6], strides[7], 1, BM)) != HILBERTA_OK) return rc;
    mqs = mq;
    mdos = mdo;
    if (gk != g) {
        if ((rc = packed::make_map(&mdos, dout, total, heads, head_dim, strides[0], strides[1], gk, BM / gk)) != HILBERTA_OK) return rc;
        if ((rc = packed::make_map(&mqs, q, total, heads, head_dim, strides[2], strides[3], gk, BM / gk)) != HILBERTA_OK) return rc;
    }
    cudaStream_t st = (cudaStream_t)stream;
    const bool overlap = (size_t)total * heads * head_dim * 2 <= kOverlapBytes / 4;
    const int rows_per_block = 256 / (head_dim / 8) * 4;
    const long long blocks = ((long long)total * heads + rows_per_block - 1) / rows_per_block;
    if (blocks > 0x7fffffffll) return HILBERTA_ERR_UNSUPPORTED;
    HB_CUDA(launch_overlapping(head_dim == 128 ? packed_delta_kernel<128> : packed_delta_kernel<64>, (unsigned)blocks, 256, 0, 1, st, overlap,
                               (const __nv_bfloat16 *)dout, (const __nv_bfloat16 *)out, lse, lse2, delta, total, Divider(heads), (long long)strides[0],
                               (long long)strides[1], (long long)strides[8], (long long)strides[9]));
    HB_LAUNCHED();
    HB_CUDA(launch_overlapping(head_dim == 128 ? packed_bwd_kernel<128> : packed_bwd_kernel<64>, ctas, THREADS, (size_t)SMEM_BYTES, 1, st,
                               true, mq, mk, mv, mdo, mqs, mdos, p));
    HB_LAUNCHED();
    if (p.splits > 1) {
        const long long vectors = (long long)total * kv_heads * (head_dim / 4);   // splits are few where this is large: below 2^31
        HB_CUDA(launch_overlapping(head_dim == 128 ? packed_sum_kernel<128> : packed_sum_kernel<64>, dim3((unsigned)((vectors + 255) / 256), 2), 256, 0,
                                   1, st, true, (const float *)p.partial, cu_seqlens, n_seq, p.dk, p.dv, p.splits, total, Divider(kv_heads), p.dk_t,
                                   p.dk_h, p.dv_t, p.dv_h, p.scale));
        HB_LAUNCHED();
    }
    return HILBERTA_OK;
}
