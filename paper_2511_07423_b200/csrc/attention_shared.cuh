// Attention of a batch whose requests share prefixes: the tokens of all requests that share a run of keys meet them
// together, once, on the tensor-memory path (shared_plan.h cuts the work; the formula is attention.cuh's).
//
// An item is some query tokens (of one request or of many), a kv head and a range of keys.  Its rows (row = j * G + g) are one
// or two tiles of 128; every item leaves fp32 partials (m, l, O) per row, which shared_merge_kernel joins:
//   out = sum_k 2^(m_k - m) O_k / sum_k 2^(m_k - m) l_k,  m = max_k m_k.
// Both products run on tcgen05.mma with M = 128, over half stages of 64 keys (a stage, 128 keys, is what the loads move):
//   S = Q K^T : A = a Q tile, B = 64 keys of K, D = S in tensor memory (64 columns a group of warps);
//   O += P V  : A = P in half precision in tensor memory (two buffers of 32 columns), B = V as it lies in the cache, D = O.
// P in tensor memory leaves shared memory's bandwidth to the operands: with both of a product's operands there, a k-step of 64
// cycles would read 8 KB, all that 128 bytes a cycle can deliver.
// Two groups of four softmax warps (thread = row), each with its own S, P and O (SharedMode).  With two tiles a group owns a
// tile: one read of K and V from L2 serves 256 rows.  With one tile the groups take alternate stages and leave separate partials,
// or, where an item has few stages, one of them takes it while the other has the next item.
//
// Warp roles: warp 3 streams pages and Q tiles (K and V have rings of their own), one thread of warp 1 and one of warp 2 issue the
// MMAs of a group each, warps 4..7 and 8..11 are the softmax groups.  tcgen05 operations of one thread complete in order, and a
// commit tells that all before it are done.  The maximum that P is relative to is raised only when a half stage exceeds it by 2^8; P is
// scaled by 2^7 besides (at most 2^15 in half precision, so that weights down to 2^-21 of the largest keep all their bits).
// Every wait on a barrier in shared memory is bounded.  The turns are named barriers, which are not: a wait that has run out takes the work out of
// a group's loop but leaves its turns, so both groups meet on them equally often whatever has failed.
//
// What bounds it, on an 8B-shaped layer (32 query and 8 kv heads of 128): with two tiles a stage takes 3 430 cycles where the tensor
// cores need 2 048 and the exponentials (16 a cycle) 2 048 too; a group's warps, one to a scheduler, wait for the latencies of
// their own instructions, 860 cycles a half stage for the exponentials alone, which the two groups take in turns (shr_turn).  Above about
// 900 TFLOP/s the power cap takes back what cycles are saved (1.6 GHz).  256 requests of 8 tokens on 12 016 shared keys: 413 us, 986 TFLOP/s
// (24 chunks of 32 on 32 768 keys: 407 us, 1 027).  With one tile the keys' bytes: three requests on 131 072 keys 94 us, 5.7 TB/s.  These are
// times in a graph of 20 launches with their merges; a row of calls without pause takes 483, 479 and 107 us, at the power cap's clocks.
// Tried and slower (256 requests): P over S in shared columns with 128-key stages 490 us, one issuer for both groups 571; exponentials
// not in turns 4 230 cycles a stage; a quarter of them by a polynomial on the multiply-add units 3 780; no maximum but a check of
// the sum 4 800; the next half stage's scores fetched before this one's exponentials 750 us.
#pragma once
#include "attention2.cuh"
#include "shared_plan.h"

namespace syn {

constexpr int SHR_THREADS = 384, SHR_BAR_BYTES = 768;
constexpr int SHR_PAGES = SHARED_STAGE / 16, SHR_HALF = SHARED_STAGE / 2;
constexpr int SHR_SOFTMAX_REGS = 208, SHR_OTHER_REGS = 88;
static_assert(8 * SHR_SOFTMAX_REGS + 4 * SHR_OTHER_REGS <= 12 * ATT_LAUNCH_REGS, "the increase must fit in what the others give back");
constexpr int SHR_PRODUCER_WARP = 3, SHR_MMA_WARP0 = 1, SHR_ALLOC_WARP = 0;
constexpr float SHR_P_SCALE_LOG2 = 7.0f;

struct SharedParams {
    const SharedItem* items;     // by CTA
    const int* cta_begin;        // [n_cta + 1]
    const int* page_tables;      // [B][max_pages]
    int max_pages, n_kv_heads, group, q_dim;
    int tile_tokens;             // tokens of a tile: 128 / G
    int layer_block0;            // 2 * layer * n_pages * Hkv: first (K|V) block of this layer in the pool map
    float scale_log2;            // log2(e) / sqrt(hd)
    float* part_o;               // [n_rows][hd]
    float2* part_ml;             // [n_rows] (reference exponent, sum)
    int* status;                 // 0 ok, 1 a bounded wait ran out, 2 the work list failed a bounds check
    const int *seg_of_token, *seg_first, *list_begin, *list;   // SharedPlan's
    op16* out;                   // [T][q_dim]
    int n_items, n_req, n_tokens, n_pages, n_rows;
};

// The work list is host-made; the kernel still refuses an item that would index out of bounds.
__device__ __forceinline__ bool shared_item_ok(const SharedItem& it, const SharedParams& p) {
    const int stages = (it.kv_end - it.kv_begin + SHARED_STAGE - 1) / SHARED_STAGE;
    const int64_t rows = (int64_t)it.n_tok * p.group * (it.mode == SHARED_STAGES ? 2 : 1);
    return it.q_tok >= 0 && it.n_tok >= 1 && it.q_tok + it.n_tok <= p.n_tokens && it.mode >= 0 && it.mode <= 3 &&
           it.n_tok <= (it.mode == SHARED_TILES ? 2 : 1) * p.tile_tokens && (it.mode != SHARED_STAGES || stages > 1) &&
           it.kvh >= 0 && it.kvh < p.n_kv_heads && it.req >= 0 && it.req < p.n_req && it.kv_begin >= 0 && (it.kv_begin & 15) == 0 &&
           it.kv_begin < it.kv_end && ((it.kv_end - 1) >> 4) < p.max_pages && it.base >= 0 && it.base + rows <= p.n_rows;
}

template <int HD>
struct SharedSmem {
    static constexpr int HALVES = HD / 64;
    static constexpr int GROUP_BYTES = HALVES * 1024;                 // 8 keys: [64-dim half][8 rows][128 bytes]
    static constexpr int BOX_BYTES = 2 * GROUP_BYTES;                 // the K rows (or the V rows) of a page
    static constexpr int K_BYTES = SHR_PAGES * BOX_BYTES;             // K (or V) of a stage
    static constexpr int Q_HALF = 128 * 128, Q_BYTES = HALVES * Q_HALF;   // a tile: [half][128 rows][128 bytes]
    static constexpr int OUT_COLS = HD / 4;                           // columns that the epilogue turns around at a time: 128 rows in half a Q tile
    static constexpr int K_SLOTS = HD == 128 ? 2 : 5, V_SLOTS = HD == 128 ? 3 : 6;
    static constexpr int TOTAL = 1024 + 2 * Q_BYTES + (K_SLOTS + V_SLOTS) * K_BYTES + SHR_BAR_BYTES;
    static_assert(TOTAL <= 232448, "shared memory of one CTA");
    static constexpr int TMEM_COLS = 512;   // O of the two groups at 0 and 128; S and P at 256 and 384
};

// D[tmem] (+)= A[tmem] * B[smem]; one thread issues.
__device__ __forceinline__ void umma_f16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// The exponentials of the two groups' warps that share a scheduler, one warp after the other (a named barrier of each, which the
// other arrives on when it is done): in step they compete for the special-function unit and then leave it idle together.  Both
// groups have as many turns (items of two tiles); the second group's first arrival lets the first begin.
__device__ __forceinline__ void shr_turn(int wg, int wq) { asm volatile("bar.sync %0, 64;" ::"r"(1 + wg * 4 + wq) : "memory"); }
__device__ __forceinline__ void shr_turn_over(int wg, int wq) { asm volatile("bar.arrive %0, 64;" ::"r"(1 + (wg ^ 1) * 4 + wq) : "memory"); }

template <int HD>
__global__ void __launch_bounds__(SHR_THREADS, 1)
attn_shared_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmKV, SharedParams p) {
    using SM = SharedSmem<HD>;
    constexpr int HALVES = SM::HALVES, KS = SM::K_SLOTS, VS = SM::V_SLOTS;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* qbuf = smem;                               // two slots
    uint8_t* kring = qbuf + 2 * SM::Q_BYTES;
    uint8_t* vring = kring + KS * SM::K_BYTES;
    // A wait on a phase's parity must not be two phases off: whoever waits on a barrier has to see every one of its phases.  So
    // a slot has three "full" barriers, for stages of group 0, of group 1 and of both, and the Q slots are watched by both issuers.
    // "Empty" barriers count two commits: both issuers' where both use the slot, twice the one's where it is the only one.
    uint64_t* k_full = reinterpret_cast<uint64_t*>(vring + VS * SM::K_BYTES);   // [who][slot]
    uint64_t* k_empty = k_full + 3 * KS; // every score of the stage is complete
    uint64_t* v_full = k_empty + KS;     // [who][slot]
    uint64_t* v_empty = v_full + 3 * VS; // every P V of the stage is complete
    uint64_t* q_full = v_empty + VS;     // [slot]
    uint64_t* q_done = q_full + 2;       // [slot] the last Q K^T that reads it is complete
    uint64_t* q_empty = q_done + 2;      // [slot] nor do the softmax warps use it any more
    uint64_t* s_full = q_empty + 2;      // [group] scores of a half stage are complete
    uint64_t* s_empty = s_full + 2;      // [group] its warps hold them in registers
    uint64_t* p_full = s_empty + 2;      // [group][buffer] P of a half stage is in tensor memory (and O rescaled if need be)
    uint64_t* pv_done = p_full + 4;      // [group][buffer] its P V is complete
    uint64_t* o_full = pv_done + 4;      // [group] the item's last P V is complete
    uint64_t* o_empty = o_full + 2;      // [group] its warps have read O
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_empty + 2);
    static_assert((4 * KS + 4 * VS + 22) * 8 + 4 <= SHR_BAR_BYTES, "barrier area");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int it_begin = p.cta_begin[blockIdx.x], it_end = p.cta_begin[blockIdx.x + 1];
    const int G = p.group;
    const bool list_ok = it_begin >= 0 && it_begin <= it_end && it_end <= p.n_items;

    if (threadIdx.x == 0) {
        tma_prefetch_desc(&tmQ);
        tma_prefetch_desc(&tmKV);
        for (int s = 0; s < 3 * KS; ++s) mbar_init(&k_full[s], 1);
        for (int s = 0; s < 3 * VS; ++s) mbar_init(&v_full[s], 1);
        for (int s = 0; s < KS; ++s) mbar_init(&k_empty[s], 2);
        for (int s = 0; s < VS; ++s) mbar_init(&v_empty[s], 2);
        for (int s = 0; s < 2; ++s) {
            mbar_init(&q_full[s], 1);
            mbar_init(&q_done[s], 2);
            mbar_init(&q_empty[s], 8);
            mbar_init(&s_full[s], 1);
            mbar_init(&s_empty[s], 4);
            for (int b = 0; b < 2; ++b) {
                mbar_init(&p_full[2 * s + b], 4);
                mbar_init(&pv_done[2 * s + b], 1);
            }
            mbar_init(&o_full[s], 1);
            mbar_init(&o_empty[s], 4);
        }
        mbar_fence_init();
        if (!list_ok) atomicExch(p.status, 2);
    }
    if (warp == SHR_ALLOC_WARP) {
        tmem_alloc(tmem_slot, SM::TMEM_COLS);
        tmem_relinquish();
    }
    pdl_launch_dependents();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    pdl_wait();   // Q and the chunk's K/V come from the preceding kernel

    if (warp < 4) {
        reg_dealloc<SHR_OTHER_REGS>();
        if (warp == SHR_PRODUCER_WARP) {
            // -------------------------------------------------------- producer: lanes 0..7 request a page each
            uint32_t st = 0, qs = 0;   // stages, Q slots so far
            bool ok = true;
            for (int it = it_begin; list_ok && it < it_end && ok; ++it) {
                const SharedItem item = p.items[it];
                if (!shared_item_ok(item, p)) break;   // the other roles flag it and stop as well
                const int tiles = item.mode == SHARED_TILES ? 2 : 1;
                if (lane == 0) {
                    for (int w = 0; w < tiles && ok; ++w) {
                        const uint32_t s = qs + w, slot = s & 1u;
                        if (s >= 2) ok = mbar_wait(&q_empty[slot], ((s >> 1) - 1) & 1u, p.status);
                        if (!ok) break;
                        mbar_expect_tx(&q_full[slot], (uint32_t)p.tile_tokens * G * HD * 2u);
                        for (int h = 0; h < HALVES; ++h)
                            tma_load_4d(qbuf + slot * SM::Q_BYTES + h * SM::Q_HALF, &tmQ, &q_full[slot], 0, h, item.kvh * G, item.q_tok + w * p.tile_tokens);
                    }
                }
                qs += tiles;
                ok = __shfl_sync(0xFFFFFFFFu, ok ? 1 : 0, 0) != 0;
                if (!ok) break;
                // page-table entries: the warp holds those of 4 stages (32 pages, one per lane) and fetches the next 32 meanwhile
                const int* pt = p.page_tables + (size_t)item.req * p.max_pages;
                const int first_page = item.kv_begin >> 4, last_page = (item.kv_end - 1) >> 4;
                int ent_cur = first_page + lane <= last_page ? pt[first_page + lane] : 0;
                int ent_next = first_page + 32 + lane <= last_page ? pt[first_page + 32 + lane] : 0;
                int k = 0;
                for (int kv0 = item.kv_begin; kv0 < item.kv_end; kv0 += SHARED_STAGE, ++st, ++k) {
                    if (k > 0 && (k & 3) == 0) {
                        ent_cur = ent_next;
                        const int nidx = first_page + (k >> 2) * 32 + 32 + lane;
                        ent_next = nidx <= last_page ? pt[nidx] : 0;
                    }
                    int page = __shfl_sync(0xFFFFFFFFu, ent_cur, ((k & 3) * SHR_PAGES + (lane & 7)) & 31);
                    const int npg = min(SHR_PAGES, (item.kv_end - kv0 + 15) >> 4);
                    if (lane < npg && (unsigned)page >= (unsigned)p.n_pages) {
                        atomicExch(p.status, 2);
                        page = 0;
                    }
                    const int block = p.layer_block0 + 2 * (page * p.n_kv_heads + item.kvh);
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        const uint32_t n = v ? VS : KS, s = st % n;
                        uint64_t* full = (v ? v_full : k_full) + (item.mode == SHARED_STAGES ? k & 1 : item.mode) * n;
                        if (lane == 0) {
                            if (st >= n) ok = mbar_wait(&(v ? v_empty : k_empty)[s], ((st / n) - 1) & 1u, p.status);
                            if (ok) mbar_expect_tx(&full[s], (uint32_t)npg * SM::BOX_BYTES);
                        }
                        ok = __shfl_sync(0xFFFFFFFFu, ok ? 1 : 0, 0) != 0;
                        if (!ok) break;
                        if (lane < npg)
                            tma_load_5d((v ? vring : kring) + s * SM::K_BYTES + lane * SM::BOX_BYTES, &tmKV, &full[s], 0, 0, 0, 0, block + v);
                    }
                    if (!ok) break;
                }
            }
        } else if ((warp == SHR_MMA_WARP0 || warp == SHR_MMA_WARP0 + 1) && elect_one()) {
            // -------------------------------------------------------- MMA issuers, one a group
            // A group works through half stages of 64 keys with one buffer of scores and two of P: as soon as its warps hold the
            // scores of half u in registers, those of half u + 1 are computed, beside its exponentials; P V of half u follows.
            const int w = warp - SHR_MMA_WARP0;
            const uint32_t idesc_pv = umma_idesc_f16_bmn(128, HD), idesc_qk = umma_idesc_f16(128, SHR_HALF);
            const uint32_t o_tmem = tmem_base + w * 128, s_tmem = tmem_base + 256 + w * 128;
            const uint64_t k_desc0 = umma_desc_k128s(smem_u32(kring), SM::GROUP_BYTES), v_desc0 = umma_desc_mn128(smem_u32(vring), 1024, SM::GROUP_BYTES);
            constexpr uint32_t SLOT16 = SM::K_BYTES >> 4, HALF16 = SLOT16 / 2;
            // the P V to come: pages | V slot << 4 | half << 8 | first << 9 | last << 10 | wait for V << 11 | its phase's parity << 12 |
            // end of the stage << 13 | stage of both << 14; 0: none
            uint32_t todo = 0;
            uint32_t use = 0, o_use = 0;     // P V's so far, and items among them
            uint32_t st = 0, qs = 0;         // stage and Q slot of the item's first
            uint32_t k_own = 0, k_both = 0, v_own = 0, v_both = 0;   // bit s: parity of the next phase of slot s
            bool ok = true;
            auto pv = [&]() {
                const uint32_t f = todo, pages = f & 15u, vs = (f >> 4) & 15u, buf = use & 1u;
                todo = 0;
                const bool first = (f >> 9) & 1u;
                if ((f >> 11) & 1u) ok = mbar_wait(&v_full[((f >> 14) & 1u ? 2 : w) * VS + vs], (f >> 12) & 1u, p.status);
                if (ok && first && o_use > 0) ok = mbar_wait(&o_empty[w], (o_use - 1) & 1u, p.status);
                if (ok) ok = mbar_wait(&p_full[2 * w + buf], (use >> 1) & 1u, p.status);
                if (!ok) return;
                tc_fence_after();
                const uint32_t p_tmem = s_tmem + 64 + buf * 32;
                const uint64_t b = v_desc0 + vs * SLOT16 + ((f >> 8) & 1u) * HALF16;
#pragma unroll
                for (uint32_t i = 0; i < SHR_PAGES / 2; ++i)   // step i: the 16 keys of a page; an item's first P V starts its O afresh
                    if (i < pages) umma_f16_ta(o_tmem, p_tmem + 8 * i, b + i * (SM::BOX_BYTES >> 4), idesc_pv, !first || i != 0);
                umma_commit(&pv_done[2 * w + buf]);
                if ((f >> 13) & 1u) {
                    umma_commit(&v_empty[vs]);
                    if (!((f >> 14) & 1u)) umma_commit(&v_empty[vs]);
                }
                if ((f >> 10) & 1u) {
                    umma_commit(&o_full[w]);
                    ++o_use;
                }
                ++use;
            };
            for (int it = it_begin; list_ok && it < it_end && ok; ++it) {
                const SharedItem item = p.items[it];
                if (!shared_item_ok(item, p)) break;
                const bool two = item.mode == SHARED_TILES, both = item.mode == SHARED_STAGES;
                const uint32_t tiles = two ? 2 : 1;
                const int n_pages = (item.kv_end - item.kv_begin + 15) >> 4;
                const uint32_t n_st = (uint32_t)(n_pages + SHR_PAGES - 1) / SHR_PAGES, step = both ? 2 : 1;
                const uint64_t a = umma_desc_k128(smem_u32(qbuf + ((qs + (two ? w : 0)) & 1u) * SM::Q_BYTES));
                for (uint32_t q = qs; q < qs + tiles && ok; ++q) ok = mbar_wait(&q_full[q & 1u], (q >> 1) & 1u, p.status);
                if (!ok) break;
                uint32_t kb = two ? k_both : k_own, vb = two ? v_both : v_own;
                const bool none = !two && !both && item.mode != w;                 // the other group's
                if (none) {
                    mbar_arrive(&q_done[qs & 1u]);
                    for (int i = 0; i < 4; ++i) mbar_arrive(&q_empty[qs & 1u]);
                }
                uint32_t k = none ? n_st : both ? w : 0, ks = (st + k) % KS, vs = (st + k) % VS;
                for (; k < n_st && ok; k += step) {
                    const uint32_t pages = (uint32_t)min(SHR_PAGES, n_pages - (int)k * SHR_PAGES);
                    uint64_t* kf = &k_full[(two ? 2 : w) * KS + ks];
                    if (todo && !mbar_test(kf, (kb >> ks) & 1u)) pv();      // K is not there yet: P V need not wait for it
                    if (ok) ok = mbar_wait(kf, (kb >> ks) & 1u, p.status);
                    if (!ok) break;
                    const uint32_t v_parity = (vb >> vs) & 1u;
                    kb ^= 1u << ks;
                    vb ^= 1u << vs;
#pragma unroll
                    for (uint32_t h = 0; h < 2; ++h) {
                        if (!ok || h * (SHR_PAGES / 2) >= pages) continue;
                        const uint32_t u = use + (todo != 0);               // half stages of the group before this one
                        if (u > 0) ok = mbar_wait(&s_empty[w], (u - 1) & 1u, p.status);
                        if (!ok) continue;
                        tc_fence_after();
                        const uint32_t here = min((uint32_t)SHR_PAGES / 2, pages - h * (SHR_PAGES / 2));
                        const uint64_t b = k_desc0 + ks * SLOT16 + h * HALF16;
                        const uint32_t idesc = here == SHR_PAGES / 2 ? idesc_qk : umma_idesc_f16(128, 16 * here);
#pragma unroll
                        for (uint32_t i = 0; i < HD / 16; ++i)   // step i: 16 dims, of the second half from step 4 on
                            umma_bf16(s_tmem, a + (i >> 2) * (SM::Q_HALF >> 4) + 2 * (i & 3), b + (i >> 2) * (1024 >> 4) + 2 * (i & 3), idesc, i != 0);
                        umma_commit(&s_full[w]);
                        const bool end = (h + 1) * (SHR_PAGES / 2) >= pages, first = k < step && h == 0, last = k + step >= n_st && end;
                        if (end) {
                            umma_commit(&k_empty[ks]);
                            if (!two) umma_commit(&k_empty[ks]);
                        }
                        if (last)
                            for (uint32_t q = qs; q < qs + tiles; ++q) umma_commit(&q_done[q & 1u]);
                        if (todo) pv();
                        todo = here | vs << 4 | h << 8 | (uint32_t)first << 9 | (uint32_t)last << 10 | (uint32_t)(h == 0) << 11 | v_parity << 12 |
                               (uint32_t)end << 13 | (uint32_t)two << 14;
                    }
                    ks += step;
                    if (ks >= (uint32_t)KS) ks -= KS;
                    vs += step;
                    if (vs >= (uint32_t)VS) vs -= VS;
                }
                (two ? k_both : k_own) = kb;
                (two ? v_both : v_own) = vb;
                // The last P V does not wait for the next item's scores: the group writes its results meanwhile, and the slots that it
                // holds are needed before the producer, who works in order, can bring what those wait for.
                if (ok && todo) pv();
                st += n_st;
                qs += tiles;
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ softmax groups (thread = row)
        // A wait that runs out sets `ok` = false; the warp then skips all further waits and tensor-memory traffic.
        reg_alloc<SHR_SOFTMAX_REGS>();
        const int wg = (warp - 4) >> 2, wq = (warp - 4) & 3, row = wq * 32 + lane;   // group, lane quarter, row of the tile
        const uint32_t t_lane = tmem_base + ((uint32_t)(wq * 32) << 16);
        const uint32_t o_col = (uint32_t)wg * 128, s_col = 256 + (uint32_t)wg * 128;
        uint32_t qs = 0, use = 0, o_use = 0;
        uint32_t v_own = 0, v_both = 0;   // as the issuer's
        bool ok = true;   // uniform over the warp: the tensor-memory loads and stores are warp-wide
        if (wg == 1) shr_turn_over(wg, wq);
        auto wait_all = [&](uint64_t* bar, uint32_t parity) {
            if (__all_sync(0xFFFFFFFFu, mbar_test(bar, parity))) return true;
            const bool r = mbar_wait(bar, parity, p.status);
            return __all_sync(0xFFFFFFFFu, r) != 0;
        };
        uint32_t vs = 0;                  // V slot of the item's first stage
        for (int it = it_begin; list_ok && it < it_end; ++it) {
            const SharedItem item = p.items[it];
            if (!shared_item_ok(item, p)) {   // uniform over the CTA
                if (threadIdx.x == 128) atomicExch(p.status, 2);
                break;
            }
            const bool two = item.mode == SHARED_TILES, both = item.mode == SHARED_STAGES;
            const int first_tok = two ? wg * p.tile_tokens : 0;       // of the group's tile, within the item
            const int rows = (two && wg == 0 ? p.tile_tokens : item.n_tok - first_tok) * G;
            const bool live = row < rows;
            const bool wlive = wq * 32 < rows;   // a warp none of whose rows exist only keeps the barriers' counts
            const int n_st = (item.kv_end - item.kv_begin + SHARED_STAGE - 1) / SHARED_STAGE;
            const int lim = item.q_pos0 + first_tok + row / G;        // last visible key position of this row
            float m_used = -INFINITY, l = 0.f;
            // The group's half stages: of every stage, or of every second one; the item's last stage may have one half.
            const int first_k = both ? wg : 0, n_mine = both ? (n_st + 1 - wg) / 2 : two || item.mode == wg ? n_st : 0;
            const int last_k = both ? first_k + 2 * (n_mine - 1) : n_st - 1;
            const int mine = n_mine == 0 ? 0 : 2 * n_mine - (item.kv_end - item.kv_begin - last_k * SHARED_STAGE <= SHR_HALF ? 1 : 0);
            const Two scale2 = two_of(p.scale_log2, p.scale_log2);
            const int see = min(item.kv_end, lim + 1);                // the row sees keys below
            // largest score of a half stage (log2 units), keys that the row does not see taken out
            auto largest = [&](uint32_t (&s)[2][32], int kv0) {
                const int nvalid = see - kv0;
                if (nvalid < SHR_HALF) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int x = 0; x < 32; ++x)
                            if (32 * c + x >= nvalid) s[c][x] = 0xFF800000u;   // -inf
                }
                float mc[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t* x = &s[c >> 1][(c & 1) * 16];
                    mc[c] = __uint_as_float(x[0]);
#pragma unroll
                    for (int y = 1; y < 15; y += 2) mc[c] = max3(mc[c], __uint_as_float(x[y]), __uint_as_float(x[y + 1]));
                    mc[c] = fmaxf(mc[c], __uint_as_float(x[15]));
                }
                return fmaxf(max3(mc[0], mc[1], mc[2]), mc[3]) * p.scale_log2;
            };
            const int step = both ? 2 : 1;
            int kv0 = item.kv_begin + first_k * SHARED_STAGE;
            for (int i = 0; i < mine; ++i, ++use, kv0 += (i & 1) ? SHR_HALF : SHR_HALF + (step - 1) * SHARED_STAGE) {
                const uint32_t buf = use & 1u, s_tmem = t_lane + s_col, p_tmem = s_tmem + 64 + buf * 32;
                if (ok) ok = wait_all(&s_full[wg], use & 1u);
                uint32_t s[2][32];
                const bool work = wlive && ok;
                float base = 0.f;
                if (work) {
                    tc_fence_after();
                    tmem_ld32(s_tmem, s[0]);
                    tmem_ld32(s_tmem + 32, s[1]);
                    tmem_ld_wait();
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0 && ok) mbar_arrive(&s_empty[wg]);
                if (work) {
                    const float ms = largest(s, kv0);
                    if (i == 0) {
                        m_used = live ? ms : 0.f;
                    } else {
                        const bool grow = live && ms > m_used + ATT2_RESCALE_GAP;
                        if (__any_sync(0xFFFFFFFFu, grow)) {
                            // O is rescaled in tensor memory: the P V before must have completed.  (The one before that has, and with
                            // it P's buffer is free: these scores were issued behind it.)
                            ok = wait_all(&pv_done[2 * wg + (buf ^ 1u)], ((use - 1) >> 1) & 1u);
                            const float corr = grow ? ex2_approx(m_used - ms) : 1.f;
                            if (grow) {
                                m_used = ms;
                                l *= corr;
                            }
                            tc_fence_after();
#pragma unroll 1
                            for (int ch = 0; ok && ch < HD / 16; ++ch) {
                                uint32_t o[16];
                                tmem_ld16(t_lane + o_col + ch * 16, o);
                                tmem_ld_wait();
#pragma unroll
                                for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * corr);
                                tmem_st16(t_lane + o_col + ch * 16, o);
                            }
                        }
                    }
                    base = (m_used == -INFINITY ? 0.f : m_used) - SHR_P_SCALE_LOG2;
                }
                if (two) shr_turn(wg, wq);
                if (work) {
                    const Two base2 = two_of(-base, -base);
                    Two sum[2] = {two_of(0.f, 0.f), two_of(0.f, 0.f)};
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t pw[16];
#pragma unroll
                        for (int x = 0; x < 16; ++x) {
                            float a, b;
                            untwo(fma2(two_of(__uint_as_float(s[c][2 * x]), __uint_as_float(s[c][2 * x + 1])), scale2, base2), a, b);
                            a = ex2_approx(a);
                            b = ex2_approx(b);
                            sum[x & 1] = add2(sum[x & 1], two_of(a, b));
                            pw[x] = pack_op(a, b);   // (rows beyond the tile's hold garbage: they only meet themselves in the products)
                        }
                        tmem_st16(p_tmem + 16 * c, pw);
                    }
                    float u0, u1;
                    untwo(add2(sum[0], sum[1]), u0, u1);
                    l += u0 + u1;
                }
                if (two) shr_turn_over(wg, wq);
                if (work) {
                    tmem_st_wait();
                    tc_fence_before();
                }
                // Rows of the last page behind the item's keys: a weight of zero takes whatever is stale there out, unless that is no
                // number.  Every group that uses the stage clears them before its P V can start.
                if (i == mine - 1) {
                    // the V slots of the group's stages: their phases turn over
                    uint32_t& v_bits = two ? v_both : v_own;
                    uint32_t slot = (vs + (uint32_t)first_k) % VS;
                    for (int n = 1; n < n_mine; ++n) {
                        v_bits ^= 1u << slot;
                        slot += step;
                        if (slot >= (uint32_t)VS) slot -= VS;
                    }
                    const uint32_t parity = (v_bits >> slot) & 1u;
                    v_bits ^= 1u << slot;
                    if ((item.kv_end & 15) && last_k == n_st - 1 && ok) {
                        // (the phase before is over: the issuer has seen it before this stage's scores)
                        ok = wait_all(&v_full[(two ? 2 : wg) * VS + slot], parity);
                        uint8_t* box = vring + slot * SM::K_BYTES + ((item.kv_end - 1 - item.kv_begin) / 16 - last_k * SHR_PAGES) * SM::BOX_BYTES;
                        const int r0 = item.kv_end & 15;
                        for (int c = row; ok && c < (16 - r0) * HALVES * 8; c += 128) {
                            const int r = r0 + c / (HALVES * 8), half = (c >> 3) % HALVES;
                            *reinterpret_cast<uint4*>(box + (r >> 3) * SM::GROUP_BYTES + half * 1024 + (r & 7) * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                        }
                        fence_proxy_async_smem();
                    }
                }
                __syncwarp();
                if (lane == 0 && ok) mbar_arrive(&p_full[2 * wg + buf]);
            }
            vs = (vs + (uint32_t)n_st) % VS;
            const uint32_t q = qs + (two ? wg : 0);
            qs += two ? 2 : 1;
            if (mine == 0) continue;   // (the group's issuer has let the Q slot go)
            // ---- end of the item: the fp32 partial (m, l, O) of the group's rows.  A row is a thread's in tensor memory; written
            // like that, a store of 16 bytes would touch 32 lines a warp.  So the warp turns 32 rows x OUT_COLS columns at a time around in
            // the Q slot, which the products no longer read.
            if (ok) ok = wait_all(&o_full[wg], o_use & 1u);
            if (ok) ok = wait_all(&q_done[q & 1u], (q >> 1) & 1u);
            ++o_use;
            if (ok && wlive) {
                constexpr int C = SM::OUT_COLS, CHUNKS = C / 4, PER = 32 / CHUNKS;   // 16-byte chunks of a row; rows of a store
                tc_fence_after();
                const int row0 = wq * 32;   // of the tile
                float* out = p.part_o + ((int64_t)item.base + (two ? first_tok * G : both ? wg * item.n_tok * G : 0) + row0) * HD;
                uint8_t* turn = qbuf + (q & 1u) * SM::Q_BYTES + (both ? wg * (SM::Q_BYTES / 2) : 0) + wq * (32 * C * 4);
                const int r = lane / CHUNKS, c16 = lane % CHUNKS;
#pragma unroll 1
                for (int ch = 0; ch < HD / C; ++ch) {
                    uint32_t o[C];
                    if constexpr (C == 32) tmem_ld32(t_lane + o_col + ch * C, o);
                    else tmem_ld16(t_lane + o_col + ch * C, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c)
                        *reinterpret_cast<uint4*>(turn + lane * (C * 4) + ((c ^ (lane & (CHUNKS - 1))) << 4)) = make_uint4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 32 / PER; ++i) {
                        const int rr = i * PER + r;
                        const uint4 v = *reinterpret_cast<const uint4*>(turn + rr * (C * 4) + ((c16 ^ (rr & (CHUNKS - 1))) << 4));
                        if (row0 + rr < rows) *reinterpret_cast<uint4*>(out + (int64_t)rr * HD + ch * C + c16 * 4) = v;
                    }
                    __syncwarp();
                }
                tc_fence_before();
                if (live) p.part_ml[(int64_t)item.base + (two ? first_tok * G : both ? wg * item.n_tok * G : 0) + row] =
                    make_float2((m_used == -INFINITY ? 0.f : m_used) - SHR_P_SCALE_LOG2, l);
                fence_proxy_async_smem();
            }
            __syncwarp();
            if (lane == 0 && ok) {
                mbar_arrive(&o_empty[wg]);
                mbar_arrive(&q_empty[q & 1u]);
                if (two) mbar_arrive(&q_empty[(q ^ 1u) & 1u]);
            }
        }
    }
    // ---------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (warp == SHR_ALLOC_WARP) {
        tc_fence_after();
        tmem_dealloc(tmem_base, SM::TMEM_COLS);
    }
}

// Joins the partials of a (token, query head): WPR warps take its parts in turn.  The lanes of a warp read 32 parts' (m, l) at a
// time, then O part by part, four on their way at once (eight where a block has one row: there the parts are many and the warps few).
// Which rows belong together is the plan's, so it is looked up before the predecessor's results are waited for.  Measured: 37 us for 131 072
// partial rows of 128 (68 MB, 1.8 TB/s): latency, with 40 registers for 12 blocks an SM (and 40 bytes spilled) and four loads a warp.
constexpr int SHR_MERGE_SPLIT_ROWS = 16;   // rows an SM from which on a warp takes one alone
template <int HD, int WPR>
__global__ void __launch_bounds__(128, WPR > 1 ? 1 : 12)
shared_merge_kernel(SharedParams p, int n_rows_out) {
    constexpr int E = HD / 32;   // components of a lane
    __shared__ float part[WPR > 1 ? 4 : 1][WPR > 1 ? HD + 2 : 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r = WPR > 1 ? blockIdx.x : blockIdx.x * 4 + warp, w0 = WPR > 1 ? warp : 0;
    pdl_launch_dependents();
    int t = 0, hq = 0, off = 0, b = 0, e = 0;
    if (r < n_rows_out) {
        const int n_q_heads = p.n_kv_heads * p.group;
        t = r / n_q_heads;
        hq = r - t * n_q_heads;
        const int kvh = hq / p.group, seg = p.seg_of_token[t];
        off = (t - p.seg_first[seg]) * p.group + hq - kvh * p.group;
        const int* li = p.list_begin + seg * p.n_kv_heads + kvh;
        b = li[0];
        e = li[1];
    }
    int at = b + w0 + WPR * lane < e ? p.list[b + w0 + WPR * lane] + off : 0;
    pdl_wait();
    float m = -INFINITY, sum = 0.f, acc[E];
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] = 0.f;
    for (int k0 = b + w0; k0 < e; k0 += 32 * WPR) {
        const int n = min(32, (e - k0 + WPR - 1) / WPR);
        if (k0 != b + w0) at = lane < n ? p.list[k0 + WPR * lane] + off : 0;
        float2 ml = make_float2(-INFINITY, 0.f);
        if ((unsigned)at >= (unsigned)p.n_rows) {
            atomicExch(p.status, 2);
            at = 0;
        }
        if (lane < n) ml = __ldcg(&p.part_ml[at]);
        auto load = [&](int k, float (&v)[E]) {
            const int ak = __shfl_sync(0xFFFFFFFFu, at, k & 31);
            const float* src = p.part_o + (int64_t)ak * HD + lane * E;
            if constexpr (E == 4) {
                const float4 x = __ldcg(reinterpret_cast<const float4*>(src));
                v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
            } else {
                const float2 x = __ldcg(reinterpret_cast<const float2*>(src));
                v[0] = x.x; v[1] = x.y;
            }
        };
        constexpr int U = WPR > 1 ? 8 : 4;
        float v[U][E];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < n) load(u, v[u]);                         // on their way while the weights are made
        // A part in which the row sees nothing (its sum is zero) has no say: the weight of -1 tells.  Every other counts even where its
        // weight is zero: a sum or a result that is no number (maybe its reference exponent too) stays none.
        const bool say = ml.y != 0.f;
        const float mk = say ? ml.x : -INFINITY;
        float mn = mk;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xFFFFFFFFu, mn, o));
        mn = fmaxf(m, mn);
        const float bs = mn == -INFINITY ? 0.f : mn, corr = ex2_approx(m - bs);
        const float w = say ? ex2_approx(mk - bs) : -1.f;
        float ws = w * ml.y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) ws += __shfl_xor_sync(0xFFFFFFFFu, ws, o);
        sum = sum * corr + ws;
#pragma unroll
        for (int i = 0; i < E; ++i) acc[i] *= corr;
        m = mn;
        for (int k = 0;; ) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (k + u >= n) break;
                const float wk = __shfl_sync(0xFFFFFFFFu, w, (k + u) & 31);
#pragma unroll
                for (int i = 0; i < E; ++i) acc[i] = wk < 0.f ? acc[i] : fmaf(v[u][i], wk, acc[i]);
            }
            k += U;
            if (k >= n) break;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k + u < n) load(k + u, v[u]);
        }
    }
    if constexpr (WPR > 1) {
        // the warps' results, joined the same way by the first
#pragma unroll
        for (int i = 0; i < E; ++i) part[warp][lane * E + i] = acc[i];
        if (lane == 0) {
            part[warp][HD] = m;
            part[warp][HD + 1] = sum;
        }
        __syncthreads();
        if (warp > 0) return;
        float mn = -INFINITY;
#pragma unroll
        for (int k = 0; k < WPR; ++k) mn = fmaxf(mn, part[k][HD]);
        const float bs = mn == -INFINITY ? 0.f : mn;
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) acc[i] = 0.f;
#pragma unroll
        for (int k = 0; k < WPR; ++k) {
            const float w = ex2_approx(part[k][HD] - bs);
            if (part[k][HD + 1] != 0.f) {   // (as above)
                sum = fmaf(w, part[k][HD + 1], sum);
#pragma unroll
                for (int i = 0; i < E; ++i) acc[i] = fmaf(w, part[k][lane * E + i], acc[i]);
            }
        }
    }
    if (r >= n_rows_out) return;
    const float inv = 1.f / sum;
    uint32_t o[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) o[i] = pack_op(acc[2 * i] * inv, acc[2 * i + 1] * inv);
    op16* dst = p.out + (int64_t)t * p.q_dim + hq * HD + lane * E;
    if constexpr (E == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(o[0], o[1]);
    else *reinterpret_cast<uint32_t*>(dst) = o[0];
}

}  // namespace syn
