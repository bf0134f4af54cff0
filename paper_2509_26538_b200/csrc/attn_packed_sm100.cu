// Attention over packed sequences for sm_100a, forward: TMA loads, tcgen05 MMAs with accumulators in tensor memory,
// online softmax in fp32.  out = softmax(scale q k^T) v within each sequence, causal or not, heads in groups.
//
// A query tile has 128 rows: 128 / g consecutive tokens of a sequence times g query heads of one key head
// (g the largest power of two, up to 16, that divides the group), token by token.  With g > 1 the rows of a tile
// need nearly the same keys and short sequences fill a tile sooner; K and V are read once for the g heads.  A unit of
// work is two consecutive tiles (one where that would leave SMs idle) with one stream of K and V blocks of 128 keys.
// Causal: a tile ends with the block of its last token; the keys behind a row's token in that block, and those behind
// the end of the sequence, are masked by column.
//
// Roles of a CTA (one per SM; it goes on with the units of CTAs that have not started):
//   warps 0-3  softmax and epilogue of query tile 0, thread r owns row r (TMEM lane r); warps 4-7 tile 1
//   warp 8     TMA producer   warp 9  MMA issuer   warp 10  finds the units, two ahead   warp 11 idle
// The two tiles take turns: while one tile's softmax runs, the tensor core works on the other's P V and next Q K^T.
// TMEM columns: S_t at [128 t, +128), overwritten in place by P_t (bf16); O_t at [256 + 128 t, +128).
//
// Bound by the chain scores -> softmax -> P V of its two tiles, like the sparse forward kernel whose loop this is: 2.0 us for
// 128 keys of two tiles at head dim 128, 1.5 at the matrix rate of a large library product.  Measured (B200, us; TFLOP/s of
// the pairs that count): 4608 tokens of 24 heads 216 (1210), causal 121 (1080); four documents of 1911 ... 4096 tokens, 32
// heads over 8 key heads, causal 297 (1100).  What it took: the unit kept in shared memory and not in registers beside 128
// scores 530 -> 316 (documents, spills); sequences by length 765 -> 382 (images of three sizes); bulk stores 316 -> 296.
// A handful of prompts is latency: 8 us for ten of 1 ... 77 tokens, of which the launch, finding the unit and one block.
// Weights are rounded to bf16 before they meet V, as the tensor cores take them: out is off by 2.0e-3 of its norm (1.7e-3 by its
// own rounding); the row sum has them in fp32.
#include <algorithm>
#include <mutex>

#include "attn_packed_tile.cuh"
#include "attn_softmax_math.cuh"

namespace hilberta {
using namespace ptx;

namespace {

constexpr int BM = 128, BN = 128, QT = 2;
// K / V ring slots (K0 V0 K1 V1 ...); beside them 32 KB in which finished rows wait for their bulk stores, 4 KB a warp
constexpr int NSTAGE = 5;
__host__ __device__ constexpr int ring_slots(int hd) { return hd == 128 ? 4 : NSTAGE; }
constexpr int STAGE_BYTES = 8 * 4096;
constexpr int UNITS = 2;                 // units found ahead
constexpr int SLAB_BYTES = BN * 128;     // 64 columns of 128 rows
constexpr int THREADS = 384;
constexpr uint32_t TMEM_COLS = 512;
constexpr float RESCALE_THRESHOLD = 8.0f;   // log2: the reference maximum moves only when a score exceeds it by 2^8
constexpr int POLY_DEG = 4;              // of the exponentials on the FMA pipes; with 3, lse is off by 2e-6 of itself, and no call is faster
constexpr int SPLIT_AT = 2;              // P goes to the MMA issuer as the keys of 32-key chunks 0 .. 2, then the rest
__host__ __device__ constexpr int tile_bytes(int hd) { return BN * hd * 2; }
__host__ __device__ constexpr int smem_bytes(int hd) { return (QT + ring_slots(hd)) * tile_bytes(hd) + STAGE_BYTES + 1024; }

enum Bar {
    Q_FULL = 0, Q_EMPTY, DRAIN,
    S_FULL,
    P_READY = S_FULL + QT,        // [2 t + part], 128 arrivals
    PV_DONE = P_READY + 2 * QT,
    KV_FULL = PV_DONE + QT, KV_EMPTY = KV_FULL + NSTAGE,
    NEXT = KV_EMPTY + NSTAGE,                               // the number of the next CTA has arrived
    WANT = NEXT + 1,                                        // the producer has asked for all of a unit's blocks
    U_FULL = WANT + 1, U_EMPTY = U_FULL + UNITS,            // U_EMPTY: producer, issuer, eight softmax warps
    NUM_BARS = U_EMPTY + UNITS
};

__device__ int g_status[64];   // [0]: code of the first wait that gave up

struct Params {
    packed::Sequences seq;
    int parts, odd, group, g_shift;   // parts = kv_heads * odd; group = odd << g_shift
    int tiles;                        // query tiles of a unit, 1 or 2
    long long stride_t, stride_h;     // of out
    __nv_bfloat16 *out;
    float *lse;
    float scale_log2;
    long long unit_wait;              // of waits that last a whole unit
};

// What every role derives from a unit.
struct Work {
    int row0, len, tok0, nt, kv_head, head0;
    int n[QT];   // key blocks of each tile
};
__device__ __forceinline__ Work work_of(const Params &p, const packed::Unit &u) {
    Work w;
    const int tpt = BM >> p.g_shift;
    w.row0 = u.row0;
    w.len = u.len;
    w.tok0 = u.block << p.seq.shift;
    w.kv_head = u.head / p.odd;
    w.head0 = w.kv_head * p.group + ((u.head % p.odd) << p.g_shift);
    w.nt = (p.tiles > 1 && w.tok0 + tpt < w.len) ? 2 : 1;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int end = p.seq.causal ? min(w.len, w.tok0 + (t + 1) * tpt) : w.len;
        w.n[t] = t < w.nt ? (end + BN - 1) / BN : 0;
    }
    return w;
}

template <int HD>
__device__ __forceinline__ void issue_qk(uint32_t tmem_s, uint32_t sQt, uint32_t sKslot) {
    constexpr uint32_t IDESC = idesc_bf16_f32(BM, BN, 0, 0);
    const uint64_t dq = smem_desc_sw128(sQt, 16, 1024), dk = smem_desc_sw128(sKslot, 16, 1024);
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
        const uint64_t off = (uint64_t)(((k >> 2) * SLAB_BYTES + (k & 3) * 32) >> 4);
        mma_ss(tmem_s, dq + off, dk + off, IDESC, k > 0);
    }
}

// O_t (+)= P_t V, P from tensor memory; the keys of part 0 or 1
template <int HD>
__device__ __forceinline__ void issue_pv(uint32_t tmem_o, uint32_t tmem_p, uint32_t sVslot, int part, bool accumulate) {
    constexpr uint32_t IDESC = idesc_bf16_f32(BM, HD, 0, 1);
    const uint64_t dv = smem_desc_sw128(sVslot, SLAB_BYTES, 1024);
    constexpr int C1 = 2 * (SPLIT_AT + 1), C2 = BN / 16;
    if (part == 0) {
#pragma unroll
        for (int k = 0; k < C1; ++k)
            mma_ts(tmem_o, tmem_p + k * 8, dv + (uint64_t)((k * 2048) >> 4), IDESC, (accumulate || k > 0) ? 1u : 0u);
    } else {
#pragma unroll
        for (int k = C1; k < C2; ++k) mma_ts(tmem_o, tmem_p + k * 8, dv + (uint64_t)((k * 2048) >> 4), IDESC, 1u);
    }
}

template <int HD>
__global__ void __launch_bounds__(THREADS, 1)
packed_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
              const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmO, const __grid_constant__ Params prm) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[NUM_BARS];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ packed::Unit units[UNITS];
    __shared__ __align__(16) uint4 next[1];
    constexpr int TILE_BYTES = tile_bytes(HD);
    constexpr int NSLAB = HD / 64, NS = ring_slots(HD);

    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t sQ = smem_u32(smem), sKV = sQ + QT * TILE_BYTES, sStage = sKV + NS * TILE_BYTES;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t bar0 = smem_u32(&bars[0]);
    int *const status = g_status;
    auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
    auto slot_of = [](uint32_t e) { return e % NS; };
    auto phase_of = [](uint32_t e) { return (e / NS) & 1; };

    if (tid == 0) {
        abort_flag = 0;
        for (int i = 0; i < NUM_BARS; ++i) {
            uint32_t count = 1;
            if (i >= P_READY && i < P_READY + 2 * QT) count = 128;
            if (i >= U_EMPTY) count = 10;
            mbar_init(bar(i), count);
        }
        mbar_fence_init();
    }
    if (warp == 8) {
        tmem_alloc(smem_u32(&tmem_slot), TMEM_COLS);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    allow_next();
    wait_for_previous();

    // the number of the next CTA that has not started, for a whole warp
    auto ask_next = [&](unsigned &n, bool &more, uint32_t &asked) {
        bool ok = true;
        if (lane == 0) {
            fence_proxy_async_smem();   // the last answer has been read
            packed::ask_next_cta(smem_u32(next), bar(NEXT));
            ok = wait_or_abort(bar(NEXT), asked & 1, &abort_flag, status, 0x109);
            if (ok) more = packed::next_cta(smem_u32(next), n);
        }
        ++asked;
        n = __shfl_sync(0xffffffffu, n, 0);
        more = __shfl_sync(0xffffffffu, (int)more, 0) != 0;
        return __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
    };

    // the next unit, for a role of one thread
    uint32_t uc = 0;
    auto next_unit = [&](packed::Unit &u, int code) {
        const uint32_t s = uc % UNITS, ph = (uc / UNITS) & 1;
        if (!wait_or_abort(bar(U_FULL + s), ph, &abort_flag, status, code, prm.unit_wait)) return false;
        u = units[s];
        ++uc;
        mbar_arrive(bar(U_EMPTY + s));
        return u.len >= 0;
    };

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    }
    if (warp == 10) {
        // ------------------------------------------------------------ finds the units
        packed::Runs runs;
        const packed::Span mine = packed::span_of(prm.seq, lane);
        unsigned n = blockIdx.x;
        bool more = true, ok = true;
        for (uint32_t i = 0, asked = 0; ok; ++i) {
            packed::Unit u;
            // the launch has a CTA for every unit there may be; some are not there
            bool found = more && packed::find_unit(prm.seq, mine, runs, prm.parts, n, u);
            while (ok && more && !found) {
                ok = ask_next(n, more, asked);
                found = ok && more && packed::find_unit(prm.seq, mine, runs, prm.parts, n, u);
            }
            if (!ok) break;
            if (!found) u.len = -1;
            const uint32_t s = i % UNITS, ph = (i / UNITS) & 1;
            if (lane == 0) {
                ok = wait_or_abort(bar(U_EMPTY + s), ph ^ 1, &abort_flag, status, 0x108, prm.unit_wait);
                if (ok) {
                    units[s] = u;
                    mbar_arrive(bar(U_FULL + s));
                }
            }
            ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
            if (!found || !ok) break;
            // not before the producer is through with this unit: a unit that another CTA could start sooner is left to it
            if (lane == 0) ok = wait_or_abort(bar(WANT), i & 1, &abort_flag, status, 0x10a, prm.unit_wait);
            ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0 && ask_next(n, more, asked);
        }
    } else if (warp == 8) {
        // ------------------------------------------------------------ producer
        if (elect_one()) {
            prefetch_tmap(&tmQ);
            prefetch_tmap(&tmK);
            prefetch_tmap(&tmV);
            uint32_t kvc = 0, qc = 0;
            bool ok = true;
            auto emit = [&](const CUtensorMap *tm, int row, int h) {
                const uint32_t s = slot_of(kvc), ph = phase_of(kvc);
                ++kvc;
                if (!wait_or_abort(bar(KV_EMPTY + s), ph ^ 1, &abort_flag, status, 0x102)) return false;
                mbar_expect_tx(bar(KV_FULL + s), TILE_BYTES);
#pragma unroll
                for (int sl = 0; sl < NSLAB; ++sl)
                    tma_load_4d(sKV + s * TILE_BYTES + sl * SLAB_BYTES, tm, bar(KV_FULL + s), 64 * sl, h, row, 0);
                return true;
            };
            packed::Unit u;
            while (ok && next_unit(u, 0x100)) {
                const Work w = work_of(prm, u);
                ok = wait_or_abort(bar(Q_EMPTY), (qc & 1) ^ 1, &abort_flag, status, 0x101);
                if (!ok) break;
                ++qc;
                mbar_expect_tx(bar(Q_FULL), w.nt * TILE_BYTES);
                for (int t = 0; t < w.nt; ++t) {
#pragma unroll
                    for (int sl = 0; sl < NSLAB; ++sl)
                        tma_load_4d(sQ + t * TILE_BYTES + sl * SLAB_BYTES, &tmQ, bar(Q_FULL), 64 * sl, w.head0,
                                    w.row0 + w.tok0 + t * (BM >> prm.g_shift), 0);
                }
                const int n = max(w.n[0], w.n[1]);
                for (int j = 0; ok && j < n; ++j)
                    ok = emit(&tmK, w.row0 + j * BN, w.kv_head) && emit(&tmV, w.row0 + j * BN, w.kv_head);
                mbar_arrive(bar(WANT));
            }
            if (abort_flag) {
                // let every copy already issued land before the CTA retires
                const long long t0 = clock64();
                while (clock64() - t0 < 2000000) {
                }
            }
        }
    } else if (warp == 9) {
        // ---------------------------------------------------------- MMA issuer
        if (elect_one()) {
            uint32_t ent = 0, qc = 0;   // ring entries and query loads consumed so far
            uint32_t cP[QT] = {0, 0};
            bool ok = true;
            auto tile_turn = [&](int t, uint32_t eV, uint32_t eKn, bool accumulate, bool more) {
                if (!wait_or_abort(bar(P_READY + t * 2), cP[t] & 1, &abort_flag, status, 0x205 + t)) return false;
                tc_fence_after();
                issue_pv<HD>(tmem + 256 + t * HD, tmem + t * BN, sKV + slot_of(eV) * TILE_BYTES, 0, accumulate);
                if (!wait_or_abort(bar(P_READY + t * 2 + 1), cP[t] & 1, &abort_flag, status, 0x205 + t)) return false;
                ++cP[t];
                tc_fence_after();
                issue_pv<HD>(tmem + 256 + t * HD, tmem + t * BN, sKV + slot_of(eV) * TILE_BYTES, 1, true);
                mma_commit(bar(PV_DONE + t));
                if (more) {
                    issue_qk<HD>(tmem + t * BN, sQ + t * TILE_BYTES, sKV + slot_of(eKn) * TILE_BYTES);
                    mma_commit(bar(S_FULL + t));
                }
                return true;
            };
            packed::Unit u;
            while (ok && next_unit(u, 0x200)) {
                const Work w = work_of(prm, u);
                const int n = max(w.n[0], w.n[1]);
                ok = wait_or_abort(bar(Q_FULL), qc & 1, &abort_flag, status, 0x201);
                if (!ok) break;
                ++qc;
                ok = wait_or_abort(bar(KV_FULL + slot_of(ent)), phase_of(ent), &abort_flag, status, 0x202);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    if (t >= w.nt) continue;
                    issue_qk<HD>(tmem + t * BN, sQ + t * TILE_BYTES, sKV + slot_of(ent) * TILE_BYTES);
                    mma_commit(bar(S_FULL + t));
                }
                mma_commit(bar(KV_EMPTY + slot_of(ent)));
                if (n == 1) mma_commit(bar(Q_EMPTY));
                for (int j = 0; j < n; ++j, ent += 2) {
                    const uint32_t eV = ent + 1, eKn = ent + 2;
                    const bool more = j + 1 < n;
                    if (more) {
                        ok = wait_or_abort(bar(KV_FULL + slot_of(eKn)), phase_of(eKn), &abort_flag, status, 0x203);
                        if (!ok) break;
                    }
                    ok = wait_or_abort(bar(KV_FULL + slot_of(eV)), phase_of(eV), &abort_flag, status, 0x204);
                    if (!ok) break;
#pragma unroll
                    for (int t = 0; t < QT; ++t)
                        if (ok && j < w.n[t]) ok = tile_turn(t, eV, eKn, j > 0, j + 1 < w.n[t]);
                    if (!ok) break;
                    mma_commit(bar(KV_EMPTY + slot_of(eV)));
                    if (more) {
                        mma_commit(bar(KV_EMPTY + slot_of(eKn)));
                        if (j + 2 == n) mma_commit(bar(Q_EMPTY));
                    }
                }
            }
            // every MMA issued above has retired before TMEM is released
            mma_commit(bar(DRAIN));
            wait_or_abort(bar(DRAIN), 0, &abort_flag, status, 0x207);
        }
    } else if (warp < 8) {
        // ------------------------------------------------- softmax + epilogue, tile t
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const int t = warp >> 2;
        const int r = tid & 127;
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lane_addr + t * BN;
        const uint32_t tO = tmem + lane_addr + 256 + t * HD;
        const float scale_log2 = prm.scale_log2;
        uint32_t cS = 0, cPV = 0, ent = 0;
        bool ok = true;
        while (ok) {
            // The unit stays in its slot to the end, so that little of it lives in registers beside the scores.
            const uint32_t slot = uc % UNITS;
            ok = wait_or_abort(bar(U_FULL + slot), (uc / UNITS) & 1, &abort_flag, status, 0x300, prm.unit_wait);
            ++uc;
            const volatile packed::Unit &u = units[slot];
            if (!ok || u.len < 0) break;
            auto work = [&] {
                packed::Unit c;
                c.row0 = u.row0, c.len = u.len, c.block = u.block, c.head = u.head;
                return work_of(prm, c);
            };
            auto release = [&] {
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(U_EMPTY + slot));
            };
            const uint32_t ent0 = ent;
            int n, first_masked;   // key blocks of this tile; from here on a row's keys may end within a block
            {
                const Work w = work();
                ent += 2 * (uint32_t)max(w.n[0], w.n[1]);
                n = t ? w.n[1] : w.n[0];
                first_masked = (prm.seq.causal ? min(w.tok0 + t * (BM >> prm.g_shift), w.len) : w.len) / BN;
            }
            if (n == 0) {   // this tile is absent
                release();
                continue;
            }
            float m_ref = 0.f, l = 0.f;
            float l_fix = 0.f;   // rounding errors of the blocks' largest weights: part of the output's normaliser, not of lse
            for (int j = 0; j < n; ++j) {
                ok = wait_or_abort(bar(S_FULL + t), cS & 1, &abort_flag, status, 0x301 + t);
                if (!ok) break;
                ++cS;
                tc_fence_after();
                uint32_t s[BN];
#pragma unroll
                for (int c = 0; c < BN / 32; ++c) tmem_ld32(tS + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&s[c * 32]));
                tmem_wait_ld();
                if (j >= first_masked) {
                    const Work w = work();
                    const int tok = w.tok0 + ((t * BM + r) >> prm.g_shift), valid = w.len - j * BN;
                    const int lim = prm.seq.causal ? min(tok + 1 - j * BN, valid) : valid;   // keys of the block that this row sees
#pragma unroll
                    for (int i = 0; i < BN; ++i)
                        if (i >= lim) s[i] = 0xff800000u;  // -inf
                    // Rows of the V tile behind the sequence belong to others: their weights are zero, and so are
                    // they from here on, whatever they hold.  (Both tiles do this; the zeros are the same.)
                    if (valid < BN) {
                        const uint32_t e = ent0 + 2 * (uint32_t)j + 1;
                        ok = wait_or_abort(bar(KV_FULL + slot_of(e)), phase_of(e), &abort_flag, status, 0x309);
                        if (!ok) break;
                        if (r >= valid) {
                            const uint32_t zero[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                            for (int c = 0; c < NSLAB * 8; ++c)
                                st_shared_v4(sKV + slot_of(e) * TILE_BYTES + (c >> 3) * SLAB_BYTES + r * 128 + (c & 7) * 16, zero);
                        }
                        fence_proxy_async_smem();
                    }
                }
                // Eight independent max chains, then a short tree; chains 3 and 7 hold the scores whose exponentials
                // the FMA pipes will compute (pairs 3 modulo 4), the other six those of the MUFU unit.
                static_assert(HB_POLY_MASK == 3, "the chain seeding below assumes pairs 3 mod 4 on the polynomial");
                float mxa[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) mxa[i] = __uint_as_float(s[i == 3 ? 6 : (i == 6 ? 3 : i)]);
#pragma unroll
                for (int i = 8; i < BN; i += 2) {
                    const int c = (i >> 1) & 7;
                    mxa[c] = max3(mxa[c], __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
                }
                const float mx_fma = fmaxf(mxa[3], mxa[7]);
                const float mx_mufu = fmaxf(max3(mxa[0], mxa[1], mxa[2]), max3(mxa[4], mxa[5], mxa[6]));
                const float mx_raw = fmaxf(mx_fma, mx_mufu);
                const bool top_on_fma = mx_fma > mx_mufu;
                const float mx = mx_raw * scale_log2;
                if (j == 0) {
                    // A row behind the sequence has no vote on the warp's references, which would change the roundings of the
                    // others with what a neighbour's query happens to be: nothing exceeds its own.  (A register for the
                    // threshold instead costs 1 %.)
                    const Work w = work();
                    m_ref = w.tok0 + ((t * BM + r) >> prm.g_shift) < w.len ? mx : __int_as_float(0x7f800000);
                } else if (__any_sync(0xffffffffu, mx > m_ref + RESCALE_THRESHOLD)) {
                    // the accumulator of the blocks so far belongs to the old reference
                    ok = wait_or_abort(bar(PV_DONE + t), (cPV - 1) & 1, &abort_flag, status, 0x303 + t);
                    if (!ok) break;
                    tc_fence_after();
                    const float m_new = fmaxf(m_ref, mx);
                    const float alpha = ex2(m_ref - m_new);
                    m_ref = m_new;
                    l *= alpha;
                    l_fix *= alpha;
#pragma unroll
                    for (int c = 0; c < HD / 32; ++c) {
                        uint32_t o[32];
                        tmem_ld32(tO + c * 32, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                        tmem_st32(tO + c * 32, o);
                    }
                }
                const float2 sc2 = make_float2(scale_log2, scale_log2), nm2 = make_float2(-m_ref, -m_ref);
                float2 sum[4] = {{0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}};
                {
                    // The row sum is taken over the fp32 weights, the MMA sees them in bf16: the rounding error of the
                    // block's largest weight, computed exactly as below, goes into the output's normaliser.
                    const float xm = fmaf(mx_raw, scale_log2, -m_ref);
                    const float pm_fma = ex2_poly1<POLY_DEG>(xm);
                    const float pm = top_on_fma ? pm_fma : ex2(xm);
                    l_fix += __uint_as_float(pack_bf16(0.f, pm) & 0xffff0000u) - pm;
                }
#pragma unroll
                for (int c = 0; c < BN / 32; ++c) {
                    uint32_t pk[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float2 x = __ffma2_rn(make_float2(__uint_as_float(s[c * 32 + 2 * i]), __uint_as_float(s[c * 32 + 2 * i + 1])),
                                                    sc2, nm2);
                        float2 p;
                        if ((i & HB_POLY_MASK) == HB_POLY_MASK) {
                            p = ex2_poly2<POLY_DEG>(x);
                        } else {
                            p.x = ex2(x.x);
                            p.y = ex2(x.y);
                        }
                        pk[i] = pack_bf16(p.x, p.y);
                        sum[i & 3] = __fadd2_rn(sum[i & 3], p);
                    }
                    tmem_st16(tS + c * 16, pk);
                    if (c == SPLIT_AT || c == BN / 32 - 1) {
                        tmem_wait_st();
                        tc_fence_before();
                        mbar_arrive(bar(P_READY + t * 2 + (c == BN / 32 - 1 ? 1 : 0)));
                    }
                }
                const float2 sa = __fadd2_rn(__fadd2_rn(sum[0], sum[1]), __fadd2_rn(sum[2], sum[3]));
                l += sa.x + sa.y;
                ++cPV;
            }
            if (!ok) break;
            // epilogue: O / l -> bf16 -> global; rows behind the sequence are dropped
            ok = wait_or_abort(bar(PV_DONE + t), (cPV - 1) & 1, &abort_flag, status, 0x305 + t);
            if (!ok) break;
            tc_fence_after();
            const Work w = work();
            const int tok = w.tok0 + ((t * BM + r) >> prm.g_shift);
            const bool in = tok < w.len;
            const int head = w.head0 + (r & ((1 << prm.g_shift) - 1));
            const float inv = 1.f / (l + l_fix);
            if (prm.lse && in)
                prm.lse[(long long)head * prm.seq.total + w.row0 + tok] = 0.6931471805599453f * (m_ref + log2f(l));
            // Rows through shared memory and one bulk tensor store per 64 columns and warp where the warp's 32 rows (32 / g
            // tokens of g heads: a box) all belong to the sequence; else per lane, rows behind it dropped.
            const int warp_tok = w.tok0 + ((t * BM + (warp & 3) * 32) >> prm.g_shift);
            if (warp_tok + (32 >> prm.g_shift) <= w.len) {
                const uint32_t stage = sStage + warp * 4096;
#pragma unroll
                for (int rd = 0; rd < HD / 64; ++rd) {
                    // the bulk store that last used the space has read it
                    if (lane == 0) bulk_wait_group_read0();
                    __syncwarp();
#pragma unroll
                    for (int c2 = 0; c2 < 2; ++c2) {
                        uint32_t o[32];
                        tmem_ld32(tO + rd * 64 + c2 * 32, o);
                        tmem_wait_ld();
                        uint32_t v[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] = pack_bf16(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
                        // row `lane` of a 128-byte-swizzled box: 16-byte chunk k sits at k ^ (row & 7)
#pragma unroll
                        for (int k = 0; k < 4; ++k) st_shared_v4(stage + lane * 128 + (((c2 * 4 + k) ^ (lane & 7)) << 4), v + 4 * k);
                    }
                    fence_proxy_async_smem();   // generic-proxy writes -> the bulk copy's reads
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_4d(&tmO, stage, 64 * rd, w.head0, w.row0 + warp_tok, 0);
                        bulk_commit_group();
                    }
                }
            } else {
                __nv_bfloat16 *orow = prm.out + (long long)(w.row0 + tok) * prm.stride_t + (long long)head * prm.stride_h;
#pragma unroll
                for (int c = 0; c < HD / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld32(tO + c * 32, o);
                    tmem_wait_ld();
                    if (in) {
                        uint32_t v[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] = pack_bf16(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
#pragma unroll
                        for (int i = 0; i < 16; i += 4)
                            *reinterpret_cast<uint4 *>(orow + c * 32 + 2 * i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                    }
                }
            }
            tc_fence_before();
            release();
        }
    }
    // the epilogue's bulk stores are complete before the CTA gives up its shared memory
    if (warp < 8 && lane == 0) bulk_wait_group0();
    tc_fence_before();
    __syncthreads();
    __syncwarp();
    if (warp == 8) tmem_dealloc(tmem, TMEM_COLS);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = (EncodeTiledFn)p;
    });
    return fn;
}

int opt_in(int device) {
    static std::mutex mutex;
    static bool done[64] = {};
    std::lock_guard<std::mutex> lock(mutex);
    if (device < 0 || device >= 64) return HILBERTA_ERR_INVALID;
    if (done[device]) return HILBERTA_OK;
    HB_CUDA(cudaFuncSetAttribute(packed_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes(128)));
    HB_CUDA(cudaFuncSetAttribute(packed_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes(64)));
    done[device] = true;
    return HILBERTA_OK;
}

}  // namespace

namespace packed {

int make_map(CUtensorMap *m, const void *base, int rows, int heads, int head_dim, long long stride_row, long long stride_head,
             int box_heads, int box_rows) {
    EncodeTiledFn enc = encode_fn();
    if (!enc) return HILBERTA_ERR_CUDA;
    cuuint64_t dims[4] = {(cuuint64_t)head_dim, (cuuint64_t)heads, (cuuint64_t)rows, 1};
    cuuint64_t strides[3] = {(cuuint64_t)stride_head * 2, (cuuint64_t)stride_row * 2, (cuuint64_t)stride_row * 2};
    cuuint32_t box[4] = {64u, (cuuint32_t)box_heads, (cuuint32_t)box_rows, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        g_last_cuda_error = (int)cudaErrorInvalidValue;
        return HILBERTA_ERR_CUDA;
    }
    return HILBERTA_OK;
}

// Checks that the forward and backward calls share.
int check(const void *const *tensors, int n, const int64_t *strides, const int32_t *cu, int n_seq, int total,
          int heads, int kv_heads, int head_dim, int dtype) {
    if (n_seq < 0 || total < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads || !strides) return HILBERTA_ERR_INVALID;
    if (dtype == HILBERTA_FP32 || dtype == HILBERTA_FP8_E4M3) return HILBERTA_ERR_UNSUPPORTED;
    if (dtype != HILBERTA_BF16 || head_dim < 1) return HILBERTA_ERR_INVALID;
    if ((head_dim != 64 && head_dim != 128) || n_seq > MAX_SEQ || total > MAX_TOTAL || heads > 65536) return HILBERTA_ERR_UNSUPPORTED;
    if ((long long)total * heads > (1ll << 31) - (1ll << 24)) return HILBERTA_ERR_UNSUPPORTED;   // units are counted in 31 bits
    if ((uintptr_t)cu & 3) return HILBERTA_ERR_INVALID;
    for (int i = 0; i < n; ++i) {
        const int64_t st = strides[2 * i], sh = strides[2 * i + 1];
        if (st < 1 || sh < 1 || (st & 7) || (sh & 7) || st > (1ll << 38) || sh > (1ll << 38)) return HILBERTA_ERR_INVALID;
        if ((uintptr_t)tensors[i] & 15) return HILBERTA_ERR_INVALID;
    }
    if (total > 0 && n_seq > 0) {
        if (!cu) return HILBERTA_ERR_INVALID;
        for (int i = 0; i < n; ++i)
            if (!tensors[i]) return HILBERTA_ERR_INVALID;
    }
    return HILBERTA_OK;
}

// Does [total, ha, head_dim] at a share a byte with [total, hb, head_dim] at b?  Slices of one buffer (equal strides) may
// lie side by side within a token, or interleave head by head; other tensors' address ranges have to be apart.
bool overlap(const void *a, const int64_t *sa, int ha, const void *b, const int64_t *sb, int hb, int total, int head_dim) {
    const uint64_t pa = (uint64_t)(uintptr_t)a, pb = (uint64_t)(uintptr_t)b;
    const uint64_t ea = 2ull * (uint64_t)((total - 1) * sa[0] + (ha - 1) * sa[1] + head_dim);
    const uint64_t eb = 2ull * (uint64_t)((total - 1) * sb[0] + (hb - 1) * sb[1] + head_dim);
    if (pa >= pb + eb || pb >= pa + ea) return false;
    if (sa[0] != sb[0]) return true;
    const uint64_t row_a = 2ull * (uint64_t)((ha - 1) * sa[1] + head_dim), row_b = 2ull * (uint64_t)((hb - 1) * sb[1] + head_dim);
    const uint64_t step = 2ull * (uint64_t)sa[0];
    if (row_a <= step && row_b <= step) {
        const uint64_t d = pb >= pa ? (pb - pa) % step : (step - (pa - pb) % step) % step;   // b's row behind a's
        if (d >= row_a && d + row_b <= step) return false;
    }
    if (sa[1] != sb[1] || ha != hb) return true;
    return hilberta_check_overlap(pa, pb, 1, ha, total, 0, 2 * sa[1], 2 * sa[0], 2 * head_dim) != 0;
}

int forward_status(bool *expired) {
    int code = 0;
    HB_CUDA(cudaMemcpyFromSymbol(&code, g_status, sizeof(int)));
    if (code) {
        const int zero[3] = {0, 0, 0};
        HB_CUDA(cudaMemcpyToSymbol(g_status, zero, sizeof(zero)));
        *expired = true;
    }
    return HILBERTA_OK;
}

}  // namespace packed
}  // namespace hilberta

using namespace hilberta;

extern "C" int hilberta_packed_status(void) {
    bool expired = false;
    // kernels on every stream: the copies below wait for none on a non-blocking one
    HB_CUDA(cudaDeviceSynchronize());
    int rc = packed::forward_status(&expired);
    if (rc == HILBERTA_OK) rc = packed::backward_status(&expired);
    return rc != HILBERTA_OK ? rc : expired ? HILBERTA_ERR_TIMEOUT : HILBERTA_OK;
}

extern "C" int hilberta_packed_forward(const void *q, const void *k, const void *v, void *out, float *lse, const int32_t *cu_seqlens,
                                       int n_seq, int total, int heads, int kv_heads, int head_dim, int dtype, const int64_t *strides,
                                       int causal, float scale, void *stream) {
    const void *tensors[4] = {q, k, v, out};
    const int n_heads[4] = {heads, kv_heads, kv_heads, heads};
    int rc = packed::check(tensors, 4, strides, cu_seqlens, n_seq, total, heads, kv_heads, head_dim, dtype);
    if (rc != HILBERTA_OK) return rc;
    if (((uintptr_t)lse & 3) || !(scale == scale)) return HILBERTA_ERR_INVALID;
    const bool none = total == 0 || n_seq == 0;
    for (int i = 0; !none && i < 3; ++i)
        if (packed::overlap(out, strides + 6, heads, tensors[i], strides + 2 * i, n_heads[i], total, head_dim)) return HILBERTA_ERR_INVALID;
    int dev = -1;
    HB_CUDA(cudaGetDevice(&dev));
    const int sms = sm100_count(dev);
    if (!sms) return HILBERTA_ERR_ARCH;
    if (none) return HILBERTA_OK;
    if ((rc = opt_in(dev)) != HILBERTA_OK) return rc;

    Params p;
    p.group = heads / kv_heads;
    const int g = packed::packed_heads(p.group);
    p.g_shift = __builtin_ctz((unsigned)g);
    p.odd = p.group / g;
    p.parts = kv_heads * p.odd;
    const int per_tile = BM / g;
    // one tile a unit where two would leave SMs without a unit
    auto units = [&](int tiles) {
        return ((long long)total / (tiles * per_tile) + std::min((long long)n_seq, (long long)total)) * p.parts;   // at most
    };
    p.tiles = units(2) >= sms ? 2 : 1;
    p.seq = {cu_seqlens, n_seq, total, __builtin_ctz((unsigned)(p.tiles * per_tile)), causal != 0};
    p.stride_t = strides[6];
    p.stride_h = strides[7];
    p.out = (__nv_bfloat16 *)out;
    p.lse = lse;
    const float s = scale > 0.f ? scale : 1.f / sqrtf((float)head_dim);
    p.scale_log2 = s * 1.4426950408889634f;
    const unsigned ctas = (unsigned)units(p.tiles);
    p.unit_wait = packed::unit_wait(((long long)total + BN - 1) / BN, ctas, sms);
    CUtensorMap mq, mk, mv, mo;
    if ((rc = packed::make_map(&mq, q, total, heads, head_dim, strides[0], strides[1], g, per_tile)) != HILBERTA_OK) return rc;
    if ((rc = packed::make_map(&mk, k, total, kv_heads, head_dim, strides[2], strides[3], 1, BN)) != HILBERTA_OK) return rc;
    if ((rc = packed::make_map(&mv, v, total, kv_heads, head_dim, strides[4], strides[5], 1, BN)) != HILBERTA_OK) return rc;
    if ((rc = packed::make_map(&mo, out, total, heads, head_dim, strides[6], strides[7], g, 32 / g)) != HILBERTA_OK) return rc;
    const bool overlap = (size_t)total * heads * head_dim * 2 <= kOverlapBytes / 4;
    HB_CUDA(launch_overlapping(head_dim == 128 ? packed_kernel<128> : packed_kernel<64>, ctas, THREADS, (size_t)smem_bytes(head_dim), 1,
                               (cudaStream_t)stream, overlap, mq, mk, mv, mo, p));
    HB_LAUNCHED();
    return HILBERTA_OK;
}
