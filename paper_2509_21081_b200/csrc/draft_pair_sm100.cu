// Absorb attention of drafted tokens over the paged cache (16-bit, or E4M3 latent rows with a power of two per token): the S query
// tokens of a request are S * H rows that share its suffix, 128 of them per pair of CTAs.
//
// Work item (CTA pair) = (request, 128 of its rows, KV chunk), with the arrangement of the 128-row kernel (absorb_pair_sm100.cu):
//     S [128 rows, 128 tokens] = Q [128, 576] * K_tile [128, 576]^T       (K_tile = latent 512 | rope 64 of 128 tokens)
//     O [128 rows, 512]       += P [128, 128 tokens] * C_tile [128, 512]
// CTA r holds rows 64 r .. + 63, supplies tokens [64 r, + 64) as B of the first product and latent dims [256 r, + 256) as B of the
// second.  The suffix is read once per 128 rows, not once per drafted token: with H = 16 a tree of 8 is one tile.
//
// Masks.  The last n_b tokens of a suffix are the drafts; draft i is visible to a row where bit i of its 64-bit mask is set, all
// tokens before them are visible to every row.  A hidden logit becomes -inf, so whatever its token holds (NaN included) cannot
// reach the row through the softmax; through the second product it could (0 * NaN), so in the tiles that hold drafts the values
// that are not finite are zeroed in shared memory before it.  (A row that does see such a token has it in its logit.)  A row that
// sees nothing in a chunk gets weight zero there.
//
// 8-bit latent rows.  Widening codes to 16 bits on the way would take as much shared-memory traffic as the products themselves.
// Instead the products run on the codes (kind::f8f6f4, twice the rate of 16 bits) and the other operand is split into two E4M3
// numbers, the nearest one and the nearest one to the rest: 4 significant bits, a sign and 4 more, at least the 8 bits of bf16 (with
// m = the mantissa of a bf16 value as an integer in [128, 256) the nearest multiple of 16 and the rest, at most 8, are both exact;
// split from 32 bits the sum is off by 6e-4 of the value in the mean square, bf16 by 1.6e-3).  Two products at twice the rate: the
// time and the operand bytes of the 16-bit kernel, on half the cache bytes.  What is left of the range: a row of Q is scaled by a
// power of two to an amax in [224, 448], so an element loses bits only where it is 2^-10 of the row's largest (by 2^-18 of that at
// most); P is held to at most 2^8 with 2^4 at the reference, so a weight is good to 2^-14 of the row's largest contribution.
// The rope part (16-bit, unscaled) goes to an accumulator of its own, and a logit is S_lat * 2^(tau + e_t) + S_rope.  The token's power
// of two belongs to its values as well: with x the scaled logit in log2 units, P = 2^(x + e_t - n) against a reference n of the
// x + e_t, and the row sum is of 2^(x - m) against one of the x (per thread; any reference within 2^60 will do in 32 bits).
//
// (Query absorption splits Q, from 32 bits; the split of P is here, from 32 bits as well.)
//
// Warp roles (384 threads per CTA): warp 0 loads K tiles (and Q), warp 2 the second operand; warp 1 allocates tensor memory and in
// the even CTA issues both products; warp 3 lays out the tokens' powers of two; warps 4-11 softmax and epilogue.
#include <algorithm>
#include <cstddef>

#include "kernels.h"
#include "sm100.cuh"

namespace tmla {
namespace {

using namespace sm100;

constexpr int TOK = 128;
constexpr int SLAB = 64 * 128;                   // [64 rows][128 bytes], swizzled
constexpr float kLog2Off = 4.f, kLog2Room = 4.f; // 8 bits: P at the reference, and above it (2^8 at most)
constexpr float kRescale16 = 8.f;                // 16 bits: log2 above the reference

struct DraftParams {
    int B, S, H, rows;     // rows = S * H per request
    int row_tiles, chunk, n_chunks;
    int chunk0;            // partial slot of the first chunk
    int page_size, max_pages, num_pages;
    const int32_t* block_table;
    const int32_t* seq_lens;
    const int32_t* draft_lens;   // optional [B]
    const uint64_t* mask;        // optional [B, S]
    const int4* desc;      // optional, per launch position: {request, clamped suffix length, page 0, page 1}
    float scale_log2;
    float* lse_part;       // [slots][B * rows]
    __nv_bfloat16* o_lat_direct;   // single chunk: the merged result bf16 [B * rows][512], and its LSE
    float* lse_direct;
    int* status;
    const float* q_tau;            // 8 bits: power of two of a row of Q, [B * rows]
    const uint8_t* exponents;      // 8 bits: [num_pages][page_size]
    const char* l2_base;   // read by the kernel behind this one: requested into L2
    uint32_t l2_total, l2_bytes;
};

template <bool E8>
struct Shape {
    static constexpr int KS = E8 ? 2 : 1;                     // stages of K
    static constexpr int LAT = E8 ? 4 : 8;                    // latent slabs of 64 tokens
    static constexpr int K_BYTES = (LAT + 1) * SLAB;          // 64 tokens: latent slabs | rope slab
    static constexpr int NV = E8 ? 1 : 2;                     // copy groups of the second operand
    static constexpr int V_BYTES = (E8 ? 4 : 8) * SLAB;       // 128 tokens x 256 dims
    static constexpr int Q_BYTES = 9 * SLAB;                  // 8 bits: both terms of 4 slabs, and rope
    static constexpr int P_BYTES = 2 * SLAB;                  // 16 bits: [2 token halves][64 rows][64]; 8 bits: [2 terms][64 rows][128]
    static constexpr int GROUP = E8 ? 32 : 16;                // tokens of one MMA of the second product
};

template <bool E8>
struct Shared {
    uint64_t q_full;                  // these four groups count the copies of both CTAs, in the even CTA
    uint64_t k_full[Shape<E8>::KS][2];
    uint64_t v_full[2];
    uint64_t p_ready;                 // one arrival per softmax warp of both CTAs
    uint64_t k_empty[Shape<E8>::KS][2], v_empty[2];  // in both CTAs, by the commits of the even one
    uint64_t s_ready[2];
    uint64_t o_done[2];               // second product of tile j: o_done[j & 1]
    uint64_t v_tail;                  // own copies of the second operand of a tile whose values are gone through first
    uint64_t sc_full[4], sc_empty[4]; // 8 bits: powers of two of tile j in slot j & 3; one arrival per softmax warp when they are read
    uint32_t tmem_base;
    int abort_flag;
    float red[4][64];                 // [token quarter][row]
    float red2[E8 ? 4 : 1][E8 ? 64 : 1];
    alignas(16) float sc[E8 ? 4 : 1][E8 ? TOK : 4];      // of a token (times the softmax scale) ...
    alignas(16) float lg[E8 ? 4 : 1][E8 ? TOK : 4];      // ... its exponent
    alignas(16) float isc[E8 ? 4 : 1][E8 ? TOK : 4];     // ... and its inverse
    int wide[E8 ? 4 : 1];             // some token up to this tile has one outside 2^+-40
};

// (all of an SM's shared memory either way: no other kernel that allocates tensor memory fits beside a CTA)
constexpr int kDraftSmem = 232448;
template <bool E8>
constexpr int smem_used() {
    using X = Shape<E8>;
    return X::KS * X::K_BYTES + X::V_BYTES + X::Q_BYTES + X::P_BYTES + 1024 + (int)sizeof(Shared<E8>);
}
static_assert(smem_used<false>() <= kDraftSmem && smem_used<true>() <= kDraftSmem, "shared memory of one SM");

constexpr int kSoftmaxBar = 1;
__device__ __forceinline__ bool vote_or(bool pred) {   // over the 256 softmax threads
    uint32_t r;
    asm volatile(
        "{\n.reg .pred p, q;\nsetp.ne.b32 q, %2, 0;\n"
        "bar.red.or.pred p, %1, 256, q;\n"
        "selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(r) : "n"(kSoftmaxBar), "r"(pred ? 1u : 0u) : "memory");
    return r != 0;
}
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync %0, 256;\n" ::"n"(kSoftmaxBar) : "memory"); }

template <bool E8>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(384, 1)
draft_pair_sm100_kernel(const __grid_constant__ CUtensorMap tm_qa, const __grid_constant__ CUtensorMap tm_qp,
                        const __grid_constant__ CUtensorMap tm_ckv, const __grid_constant__ CUtensorMap tm_kpe,
                        const __grid_constant__ CUtensorMap tm_o, DraftParams p) {
    using X = Shape<E8>;
    constexpr int KS = X::KS, LAT = X::LAT, HALF = LAT / 2;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sK = smem;
    uint8_t* sV = sK + KS * X::K_BYTES;
    uint8_t* sQ = sV + X::V_BYTES;
    uint8_t* sP = sQ + X::Q_BYTES;
    auto* sh = reinterpret_cast<Shared<E8>*>(sP + X::P_BYTES);
    volatile int* abort_flag = &sh->abort_flag;

    const int warp = warp_index_uniform(), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_cta_rank();
    pdl_trigger();
    // Set-up touches no global memory: it runs before the wait for the preceding kernel.
    if (warp == 0) {
        uint64_t* all = &sh->q_full;
        constexpr int n_bars = (int)(offsetof(Shared<E8>, tmem_base) / sizeof(uint64_t));
        static_assert(n_bars <= 32, "one lane per barrier");
        if (lane < n_bars) mbar_init(all + lane, all + lane == &sh->p_ready ? 16 : all + lane >= &sh->sc_empty[0] ? 8 : 1);
        if (lane == 0) sh->abort_flag = 0;
        fence_mbar_init();
        __syncwarp();
    }
    if (warp == 1) tmem_alloc_pair(&sh->tmem_base, 512);
    if (warp == 2) {
        if (lane == 0) prefetch_tmap(&tm_qa);
        if (lane == 1) prefetch_tmap(&tm_qp);
        if (lane == 2) prefetch_tmap(&tm_ckv);
        if (lane == 3) prefetch_tmap(&tm_kpe);
    }
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, sh->tmem_base, 0);
    pdl_wait();

    // Work items in launch order: row tile fastest (they share the tokens), then chunk, then request in longest-first order.
    const int item = blockIdx.x >> 1;
    const int tile = item % p.row_tiles, chunk = (item / p.row_tiles) % p.n_chunks, z = item / (p.row_tiles * p.n_chunks);
    int b, len = -1, pg0 = -1, pg1 = -1;
    if (p.desc != nullptr) {
        const int4 d = p.desc[z];
        b = d.x; len = d.y; pg0 = d.z; pg1 = d.w;
    } else {
        b = z;
        len = min(max(p.seq_lens[b], 0), p.max_pages * p.page_size);
    }
    const int n_rows = min(128, p.rows - tile * 128);
    const int64_t row0 = (int64_t)b * p.rows + tile * 128;
    const int64_t all_rows = (int64_t)p.B * p.rows;
    const int tok_begin = chunk * p.chunk;
    // (through a shuffle: the role warps' loops are then known to be uniform)
    const int tok_end = __shfl_sync(0xffffffffu, min(len, tok_begin + p.chunk), 0);
    const int n_tiles = tok_end > tok_begin ? (tok_end - tok_begin + TOK - 1) / TOK : 0;
    const int n_last = tok_end - tok_begin - (n_tiles - 1) * TOK;      // tokens of the last tile
    // first draft (a single token that sees itself hides nothing: none)
    const int n_draft = p.draft_lens != nullptr ? min(max(p.draft_lens[b], 0), p.S) : p.S;
    const int draft0 = __shfl_sync(0xffffffffu, p.S == 1 && p.mask == nullptr ? len : len - n_draft, 0);
    // Tiles from `first_special` on: the second operand is gone through in shared memory before the product, values of drafts that
    // are not finite zeroed (see above), and the rest of the last group of tokens, which may hold anything.
    int first_special = draft0 >= tok_end ? n_tiles : max(draft0 - tok_begin, 0) / TOK;
    if (n_tiles > 0 && n_last % X::GROUP != 0) first_special = min(first_special, n_tiles - 1);

    const int32_t* bt = p.block_table + (int64_t)b * p.max_pages;
    bool bad_page = false;   // producer warps only: a page id of the caller's table was out of range
    auto page_at = [&](int t0) {   // physical page of token t0 < tok_end
        const int idx = t0 / p.page_size;
        int page = (p.desc != nullptr && idx < 2) ? (idx == 0 ? pg0 : pg1) : bt[idx];
        // The tensor maps end at num_pages: a coordinate at or past it reads as zeros instead of touching memory the caller does
        // not own.  The violation is reported through the status word.
        if ((unsigned)page >= (unsigned)p.num_pages) {
            bad_page = true;
            page = p.num_pages;
        }
        return page;
    };
    // physical page and slot of half `h` (64 tokens) of tile j; a half past the end reads as zeros
    auto page_of = [&](int j, int h, int& page, int& slot) {
        const int t0 = tok_begin + j * TOK + h * 64;
        slot = t0 % p.page_size;
        page = __shfl_sync(0xffffffffu, t0 < tok_end ? page_at(t0) : p.num_pages, 0);
    };

    int issued = 0;   // producer warps: tiles whose copies were issued, for the abort path
    if (n_tiles > 0) {
        if (warp == 0) {
            // ---------------- Q and K tiles
            const uint32_t ld = elect_one() ? 1u : 0u;
            const uint32_t ld_even = rank == 0 ? ld : 0u;
            auto prefetch_tile = [&](int j) {   // paged tiles are requested into L2 ahead of the load into a freed stage
                if (j >= n_tiles) return;
                int page, slot;
                page_of(j, (int)rank, page, slot);
#pragma unroll 1
                for (int i = 0; i < HALF; ++i) tma_prefetch_4d_if(ld, &tm_ckv, 0, slot, 2 * i, page);
                tma_prefetch_3d_if(ld, &tm_kpe, 0, slot, page);
            };
            bool ok = true;
            for (int j = 0; j < n_tiles && ok; ++j) {
                const int s = j % KS;
                uint8_t* dst = sK + s * X::K_BYTES;
                int page, slot;
                page_of(j, (int)rank, page, slot);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (j >= KS) ok = ok && mbar_wait_warp(&sh->k_empty[s][h], ((j / KS) & 1) ^ 1, abort_flag);
                    if (!ok) break;
                    const uint32_t kf = cluster_map(&sh->k_full[s][h], 0);
                    mbar_arrive_expect_tx_if(ld_even, &sh->k_full[s][h], 2 * (HALF + h) * SLAB);
#pragma unroll
                    for (int i = 0; i < HALF; i += 2)
                        tma_load_4d_pair_if(ld, dst + (HALF * h + i) * SLAB, &tm_ckv, kf, 0, slot, HALF * h + i, page);
                    if (h == 1) tma_load_3d_pair_if(ld, dst + LAT * SLAB, &tm_kpe, kf, 0, slot, page);
                }
                issued = j + 1;
                if (j == 0) {
                    const uint32_t qf = cluster_map(&sh->q_full, 0);
                    const int y = (int)row0 + 64 * (int)rank;
                    mbar_arrive_expect_tx_if(ld_even, &sh->q_full, 2 * X::Q_BYTES);
#pragma unroll 1
                    for (int sl = 0; sl < 8; ++sl) tma_load_2d_pair_if(ld, sQ + sl * SLAB, &tm_qa, qf, sl * 64, y);
                    tma_load_2d_pair_if(ld, sQ + 8 * SLAB, &tm_qp, qf, 0, y);
                    for (int i = 1; i < KS + 1; ++i) prefetch_tile(i);
                }
                prefetch_tile(j + KS + 1);
            }
        } else if (warp == 2) {
            // ---------------- second operand: latent dims [256 rank, + 256) of all 128 tokens
            const uint32_t ld = elect_one() ? 1u : 0u;
            const uint32_t ld_even = rank == 0 ? ld : 0u;
            const uint32_t vf[2] = {cluster_map(&sh->v_full[0], 0), cluster_map(&sh->v_full[1], 0)};
            const uint32_t vt = cluster_map(&sh->v_tail, rank);
            bool ok = true;
            for (int j = 0; j < n_tiles && ok; ++j) {
                int page[2], slot[2];
                page_of(j, 0, page[0], slot[0]);
                page_of(j, 1, page[1], slot[1]);
                const bool special = j >= first_special;     // counted by the CTA's own barrier: its threads go through the values
                if (special && j > 0) {                      // (the barrier's phases follow one another)
                    ok = mbar_wait_warp(&sh->v_empty[X::NV - 1], (j - 1) & 1, abort_flag);
                    if (!ok) break;
                }
                if (special) mbar_arrive_expect_tx_if(ld, &sh->v_tail, X::V_BYTES);
#pragma unroll
                for (int nb = 0; nb < X::NV; ++nb) {
                    if (j > 0) ok = ok && mbar_wait_warp(&sh->v_empty[nb], (j - 1) & 1, abort_flag);
                    if (!ok) break;
                    if (!special) mbar_arrive_expect_tx_if(ld_even, &sh->v_full[nb], 2 * X::V_BYTES / X::NV);
                    const uint32_t bar = special ? vt : vf[nb];
                    // 16 bits: blocks of 128 dims, [block][token half][2 slabs]; 8 bits: [token half][2 slabs = blocks]
                    const int slab = E8 ? 2 * (int)rank : 4 * (int)rank + 2 * nb;
                    tma_load_4d_pair_if(ld, sV + (4 * nb) * SLAB, &tm_ckv, bar, 0, slot[0], slab, page[0]);
                    tma_load_4d_pair_if(ld, sV + (4 * nb + 2) * SLAB, &tm_ckv, bar, 0, slot[1], slab, page[1]);
                }
                issued = j + 1;
            }
        } else if (warp == 1 && rank == 0) {
            // ---------------- both products (even CTA)
            constexpr uint32_t idesc_s = idesc_bf16(128, 128, false, false);
            constexpr uint32_t idesc_s8 = idesc_e4m3(128, 128, false, false);
            constexpr uint32_t idesc_o = E8 ? idesc_e4m3(128, 256, false, true) : idesc_bf16(128, 256, false, true);
            const uint32_t qa = smem_u32(sQ), va = smem_u32(sV), pa = smem_u32(sP);
            bool ok = mbar_wait_warp(&sh->q_full, 0, abort_flag);
            for (int j = 0; j <= n_tiles && ok; ++j) {
                if (j < n_tiles) {
                    // S(j) into buffer j & 1: the softmax of tile j - 2 has read it (p_ready of that tile, awaited below)
                    const int s = j % KS;
                    const uint32_t ka = smem_u32(sK) + s * X::K_BYTES;
                    const uint32_t d = tmem_base + 256u + (uint32_t)(j & 1) * (E8 ? 128u : 64u);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        ok = ok && mbar_wait_warp(&sh->k_full[s][h], (j / KS) & 1, abort_flag);
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_one()) {
                            if (E8) {
#pragma unroll
                                for (int sl = HALF * h; sl < HALF * (h + 1); ++sl)
#pragma unroll
                                    for (int t = 0; t < 2; ++t) {
                                        const uint64_t da = smem_desc_k_sw128(qa + (4 * t + sl) * SLAB);
                                        const uint64_t db = smem_desc_k_sw128(ka + sl * SLAB);
#pragma unroll
                                        for (int k = 0; k < 4; ++k) umma_pair_e4m3(d, da + 2 * k, db + 2 * k, idesc_s8, (sl | t | k) != 0);
                                    }
                                if (h == 1) {
                                    const uint64_t da = smem_desc_k_sw128(qa + 8 * SLAB), db = smem_desc_k_sw128(ka + LAT * SLAB);
#pragma unroll
                                    for (int k = 0; k < 4; ++k) umma_pair_ss(d + 64u, da + 2 * k, db + 2 * k, idesc_s, k != 0);
                                }
                            } else {
#pragma unroll
                                for (int sl = 4 * h; sl < (h == 0 ? 4 : 9); ++sl) {
                                    const uint64_t da = smem_desc_k_sw128(qa + sl * SLAB);
                                    const uint64_t db = smem_desc_k_sw128(ka + sl * SLAB);
#pragma unroll
                                    for (int k = 0; k < 4; ++k) umma_pair_ss(d, da + 2 * k, db + 2 * k, idesc_s, (sl | k) != 0);
                                }
                            }
                            umma_pair_commit(&sh->k_empty[s][h]);
                            if (h == 1) umma_pair_commit(&sh->s_ready[j & 1]);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                }
                if (j > 0) {
                    const int t = j - 1;
                    const bool last = t == n_tiles - 1;
                    const int n_k = last ? (n_last + X::GROUP - 1) / X::GROUP : TOK / X::GROUP;
                    ok = mbar_wait_warp(&sh->p_ready, t & 1, abort_flag);
                    if (!ok) break;
#pragma unroll
                    for (int nb = 0; nb < 2; ++nb) {
                        if (t < first_special && nb < X::NV) ok = ok && mbar_wait_warp(&sh->v_full[nb], t & 1, abort_flag);
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_one()) {
                            const uint32_t d = tmem_base + (uint32_t)nb * 128u;
                            if (E8) {
                                // a group of 32 tokens is 4 KB of the second operand and 32 bytes of P's rows
                                const uint64_t da0 = smem_desc_k_sw128(pa);
                                const uint64_t db0 = smem_desc_mn_sw128(va + nb * SLAB, SLAB, 1024);
#pragma unroll 1
                                for (int k = 0; k < n_k; ++k) {
                                    const uint64_t db = db0 + (k >> 1) * (2 * SLAB / 16) + (k & 1) * 256;
                                    umma_pair_e4m3(d, da0 + 2 * k, db, idesc_o, (t | k) != 0);
                                    umma_pair_e4m3(d, da0 + SLAB / 16 + 2 * k, db, idesc_o, 1);
                                }
                            } else {
                                const uint64_t da0 = smem_desc_k_sw128(pa);
                                const uint64_t db0 = smem_desc_mn_sw128(va + (4 * nb) * SLAB, SLAB, 1024);
                                auto product = [&](int k) {   // 16 tokens (descriptor addresses count 16-byte units)
                                    umma_pair_ss(d, da0 + (k >> 2) * (SLAB / 16) + 2 * (k & 3), db0 + (k >> 2) * (2 * SLAB / 16) + (k & 3) * 128,
                                                 idesc_o, (t | k) != 0);
                                };
                                if (n_k == 8) {
#pragma unroll
                                    for (int k = 0; k < 8; ++k) product(k);
                                } else {
#pragma unroll 1
                                    for (int k = 0; k < n_k; ++k) product(k);
                                }
                            }
                            if (nb >= 2 - X::NV) umma_pair_commit(&sh->v_empty[nb - (2 - X::NV)]);
                            if (nb == 1) umma_pair_commit(&sh->o_done[t & 1]);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                }
            }
        } else if (warp >= 4) {
            // ---------------- softmax: thread = (row, token quarter); the quarter's 32 tokens are half `half`, columns 32 w
            const int w = (warp - 4) >> 2, q = warp & 3;
            const int row = 32 * (q & 1) + lane, half = q >> 1;
            const int quarter = 2 * half + w;
            const uint32_t lane_base = (uint32_t)(32 * q) << 16;
            const uint32_t p_bar = cluster_map(&sh->p_ready, 0);
            const bool mine = 64 * (int)rank + row < n_rows;      // (else nobody's: sees nothing)
            uint64_t sees = 0;            // bit i: draft i
            if (mine) {
                const int j = (tile * 128 + 64 * (int)rank + row) / p.H;
                sees = p.mask != nullptr ? p.mask[(int64_t)b * p.S + j] : (2ull << j) - 1ull;
            }
            const float tau = E8 && mine ? p.q_tau[row0 + 64 * (int)rank + row] : 1.f;
            float m_ref = -INFINITY;      // log2 units; 8 bits: of the logits times the tokens' powers of two
            float m_sum = -INFINITY;      // 8 bits: reference of this thread's row sum, which is of the logits alone
            float l_part[2] = {0.f, 0.f};
            for (int j = 0; j < n_tiles; ++j) {
                const int n_valid = j == n_tiles - 1 ? n_last : TOK;
                bool ok = *abort_flag == 0 && mbar_wait(&sh->s_ready[j & 1], (j >> 1) & 1, abort_flag);
                if (E8) ok = ok && mbar_wait(&sh->sc_full[j & 3], (j >> 2) & 1, abort_flag);
                ok = __all_sync(0xffffffffu, ok);
                // bit c: token c of this quarter is there, and visible to this row
                const int t_rel = 32 * quarter, first = tok_begin + j * TOK + t_rel;
                uint32_t vis = !mine ? 0u : n_valid >= t_rel + 32 ? 0xffffffffu : n_valid > t_rel ? (1u << (n_valid - t_rel)) - 1u : 0u;
                if (first + 32 > draft0) {
                    const int at = first - draft0;      // > -32
                    vis &= at >= 64 ? 0u : at >= 0 ? (uint32_t)(sees >> at) : ((uint32_t)sees << -at) | ((1u << -at) - 1u);
                }
                // x[c]: the logit in log2 units, above the reference (8 bits: with the token's power of two, at the offset)
                float x[32], tsum = 0.f;
                uint32_t pk[16];
                float off = (E8 ? kLog2Off : 0.f) - (m_ref == -INFINITY ? 0.f : m_ref), top = -INFINITY;
                const float4* isc4 = reinterpret_cast<const float4*>(&sh->isc[E8 ? j & 3 : 0][E8 ? t_rel : 0]);
                const float4* lg4 = reinterpret_cast<const float4*>(&sh->lg[E8 ? j & 3 : 0][E8 ? t_rel : 0]);
                // P in the form of the product's operand, and (8 bits) its sum without the tokens' powers of two
                auto probabilities = [&] {
                    uint64_t sum = 0ull;      // two 32-bit zeros
#pragma unroll
                    for (int c = 0; c < 32; c += 4) {
                        const float p0 = fast_exp2(x[c]), p1 = fast_exp2(x[c + 1]), p2 = fast_exp2(x[c + 2]), p3 = fast_exp2(x[c + 3]);
                        if (E8) {
                            const float4 g = isc4[c / 4];
                            const uint64_t pa = pack_f32x2(p0, p1), pb = pack_f32x2(p2, p3);
                            sum = fma_f32x2(pa, pack_f32x2(g.x, g.y), sum);
                            sum = fma_f32x2(pb, pack_f32x2(g.z, g.w), sum);
                            split4_x2(pa, pb, pk[c / 4], pk[8 + c / 4]);
                        } else {
                            pk[c / 2] = pack_bf16(p0, p1);
                            pk[c / 2 + 1] = pack_bf16(p2, p3);
                        }
                    }
                    if (E8) {
                        float a, b2;
                        unpack_f32x2(sum, a, b2);
                        tsum = a + b2;
                    }
                };
                if (ok) {
                    tc_fence_after();
                    const uint32_t s_addr = tmem_base + lane_base + 256u + (uint32_t)((j & 1) * (E8 ? 128 : 64) + 32 * w);
                    uint32_t sr[32];
                    tmem_ld32(s_addr, sr);
                    const uint64_t off2 = pack_f32x2(off, off), scale2 = pack_f32x2(p.scale_log2, p.scale_log2);
                    if (E8) {
                        uint32_t rr[32];
                        tmem_ld32(s_addr + 64u, rr);
                        tmem_ld_wait();
                        const float4* sc4 = reinterpret_cast<const float4*>(&sh->sc[E8 ? j & 3 : 0][E8 ? t_rel : 0]);
                        const uint64_t tau2 = pack_f32x2(tau, tau);
#pragma unroll
                        for (int c = 0; c < 32; c += 4) {
                            const float4 g = sc4[c / 4], e = lg4[c / 4];
#pragma unroll
                            for (int i = 0; i < 4; i += 2) {
                                const uint64_t t1 = mul_f32x2(i == 0 ? pack_f32x2(g.x, g.y) : pack_f32x2(g.z, g.w), tau2);
                                const uint64_t t2 = add_f32x2(i == 0 ? pack_f32x2(e.x, e.y) : pack_f32x2(e.z, e.w), off2);
                                const uint64_t r2 = pack_f32x2(__uint_as_float(rr[c + i]), __uint_as_float(rr[c + i + 1]));
                                const uint64_t s2 = pack_f32x2(__uint_as_float(sr[c + i]), __uint_as_float(sr[c + i + 1]));
                                unpack_f32x2(fma_f32x2(s2, t1, fma_f32x2(r2, scale2, t2)), x[c + i], x[c + i + 1]);
                            }
                        }
                    } else {
                        tmem_ld_wait();
#pragma unroll
                        for (int c = 0; c < 32; c += 2)
                            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(sr[c]), __uint_as_float(sr[c + 1])), scale2, off2), x[c], x[c + 1]);
                    }
                    if (vis != 0xffffffffu) {
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (!((vis >> c) & 1u)) x[c] = -INFINITY;
                    }
                    // probabilities against the current reference: final unless the CTA votes for a rescale
                    probabilities();
                    float mx[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
                    for (int c = 4; c < 32; ++c) mx[c & 3] = fmaxf(mx[c & 3], x[c]);
                    top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                }
                // (a row without a reference: any logit exceeds it)
                if (vote_or(top > (m_ref == -INFINITY ? -INFINITY : E8 ? kLog2Off + kLog2Room : kRescale16))) {
                    sh->red[quarter][row] = top - off;
                    softmax_sync();
                    const float cm = fmaxf(fmaxf(sh->red[0][row], sh->red[1][row]), fmaxf(sh->red[2][row], sh->red[3][row]));
                    const float m_new = fmaxf(m_ref, cm);
                    const float f = (m_new == -INFINITY) ? 1.f : fast_exp2(m_ref - m_new);
                    m_ref = m_new;
                    if (!E8) {
                        l_part[0] *= f;
                        l_part[1] *= f;
                    }
                    if (j > 0) {
                        // this thread's lane of O (the same row), 128 of its 256 columns, once the previous tile's product has
                        // landed
                        if (*abort_flag == 0) mbar_wait(&sh->o_done[(j - 1) & 1], ((j - 1) >> 1) & 1, abort_flag);
                        __syncwarp();
                        tc_fence_after();
#pragma unroll 1
                        for (int i = 0; i < 4; ++i) {
                            uint32_t orr[32];
                            const uint32_t o_addr = tmem_base + lane_base + (uint32_t)(128 * w + 32 * i);
                            tmem_ld32(o_addr, orr);
                            tmem_ld_wait();
#pragma unroll
                            for (int c = 0; c < 32; ++c) orr[c] = __float_as_uint(__uint_as_float(orr[c]) * f);
                            tmem_st32(o_addr, orr);
                        }
                        tmem_st_wait();
                    }
                    if (ok) {
                        const float off_new = (E8 ? kLog2Off : 0.f) - (m_ref == -INFINITY ? 0.f : m_ref), d = off_new - off;
#pragma unroll
                        for (int c = 0; c < 32; ++c) x[c] += d;
                        off = off_new;
                        probabilities();
                    }
                }
                if (E8 && ok) {
                    // Row sum of 2^(logit - m_sum).  P holds the tokens' powers of two, so its sum without them is 2^off of that: exact as
                    // long as they are within 2^+-40 (nothing that counts is lost where P underflows); else from the logits themselves.
                    if (!sh->wide[E8 ? j & 3 : 0]) {
                        if (m_sum == -INFINITY || -off - m_sum > 40.f) {
                            l_part[0] = m_sum == -INFINITY ? 0.f : l_part[0] * fast_exp2(m_sum + off);
                            m_sum = -off;
                        }
                        l_part[0] = fmaf(tsum, fast_exp2(-off - m_sum), l_part[0]);
                    } else {
                        float mx = -INFINITY;
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            const float4 e = lg4[c];
                            const float y0 = x[4 * c] - e.x, y1 = x[4 * c + 1] - e.y, y2 = x[4 * c + 2] - e.z, y3 = x[4 * c + 3] - e.w;
                            mx = fmaxf(mx, fmaxf(fmaxf(y0, y1), fmaxf(y2, y3)));
                        }
                        mx -= off;
                        if (mx != -INFINITY && (m_sum == -INFINITY || mx - m_sum > 40.f)) {
                            l_part[0] = m_sum == -INFINITY ? 0.f : l_part[0] * fast_exp2(m_sum - mx);
                            m_sum = mx;
                        }
                        const float base = off + (m_sum == -INFINITY ? 0.f : m_sum);
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            const float4 e = lg4[c];
                            l_part[0] += (fast_exp2(x[4 * c] - e.x - base) + fast_exp2(x[4 * c + 1] - e.y - base)) +
                                         (fast_exp2(x[4 * c + 2] - e.z - base) + fast_exp2(x[4 * c + 3] - e.w - base));
                        }
                    }
                }
                if (ok) {
                    if (!E8) {
                        // row sums of the rounded values
#pragma unroll
                        for (int c = 0; c < 16; ++c) {
                            l_part[0] += __uint_as_float(pk[c] << 16);
                            l_part[1] += __uint_as_float(pk[c] & 0xffff0000u);
                        }
                    }
                    // P, once the previous tile's product has read its buffer
                    if (j > 0) mbar_wait(&sh->o_done[(j - 1) & 1], ((j - 1) >> 1) & 1, abort_flag);
                    if (E8) {
                        // row of 128 tokens, one byte each: this quarter is 16-byte pieces 2 * quarter and + 1, in both terms
                        uint8_t* p_row = sP + row * 128;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const int at = ((2 * quarter + c) ^ (row & 7)) * 16;
                            *reinterpret_cast<uint4*>(p_row + at) = make_uint4(pk[4 * c], pk[4 * c + 1], pk[4 * c + 2], pk[4 * c + 3]);
                            *reinterpret_cast<uint4*>(p_row + SLAB + at) = make_uint4(pk[8 + 4 * c], pk[9 + 4 * c], pk[10 + 4 * c], pk[11 + 4 * c]);
                        }
                    } else {
                        uint8_t* p_row = sP + half * SLAB + row * 128;
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            *reinterpret_cast<uint4*>(p_row + (((4 * w + c) ^ (row & 7)) * 16)) =
                                make_uint4(pk[4 * c], pk[4 * c + 1], pk[4 * c + 2], pk[4 * c + 3]);
                    }
                    if (j >= first_special) {
                        // own half of the second operand: drafts cleared of values that are not finite, token rows n_valid ..
                        // next multiple of a group zeroed
                        mbar_wait(&sh->v_tail, (j - first_special) & 1, abort_flag);
                        const int t_lo = min(max(draft0 - (tok_begin + j * TOK), 0), n_valid);
                        const int n_go = (n_valid + X::GROUP - 1) / X::GROUP * X::GROUP - t_lo;
                        constexpr int W = E8 ? 16 : 32;          // 16-byte pieces of a token's 256 dims
                        for (int i = threadIdx.x - 128; i < n_go * W; i += 256) {
                            const int t = t_lo + i / W, sl = (i >> 3) & (W / 8 - 1), c16 = i & 7;
                            uint8_t* at = sV + (E8 ? 2 * (t >> 6) + sl : 4 * (sl >> 1) + 2 * (t >> 6) + (sl & 1)) * SLAB + (t & 63) * 128 + c16 * 16;
                            uint4 v = *reinterpret_cast<const uint4*>(at);
                            uint32_t* vv = reinterpret_cast<uint32_t*>(&v);
                            uint32_t bad = 0;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                // bytes (16-bit halves) that are all ones where a value is not finite
                                const uint32_t f = E8 ? __vcmpeq4(vv[e] & 0x7f7f7f7fu, 0x7f7f7f7fu) : __vcmpgeu2(vv[e] & 0x7fff7fffu, 0x7f807f80u);
                                vv[e] &= ~f;
                                bad |= f;
                            }
                            if (t >= n_valid) v = make_uint4(0, 0, 0, 0);
                            if (t >= n_valid || bad) *reinterpret_cast<uint4*>(at) = v;
                        }
                    }
                }
                fence_proxy_async();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_cluster(p_bar);
                    if (E8) mbar_arrive(&sh->sc_empty[j & 3]);
                }
            }

            // ---------------- epilogue: row sums, normalised partial, LSE
            bool staged = false;
            if (!vote_or(*abort_flag != 0)) {
                sh->red[quarter][row] = l_part[0] + l_part[1];
                if (E8) sh->red2[E8 ? quarter : 0][E8 ? row : 0] = m_sum;
                softmax_sync();
                float l, m = m_ref;
                if (E8) {
                    m = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 4; ++i) m = fmaxf(m, sh->red2[E8 ? i : 0][E8 ? row : 0]);
                    l = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float mi = sh->red2[E8 ? i : 0][E8 ? row : 0], li = sh->red[i][row];
                        l += mi == -INFINITY ? li : li * fast_exp2(mi - m);
                    }
                } else {
                    l = sh->red[0][row] + sh->red[1][row] + sh->red[2][row] + sh->red[3][row];
                }
                // l = 0: nothing visible in this chunk.  l = NaN: some logit is not finite, and the row becomes NaN.
                const float inv = l == 0.f ? 0.f : (E8 ? fast_exp2(m_ref - kLog2Off - m) : 1.f) / l;
                const int r = 64 * (int)rank + row;
                const bool direct = p.o_lat_direct != nullptr;
                if (quarter == 0 && r < n_rows) {
                    const float lse = l == 0.f ? -INFINITY : l == l ? (m + log2f(l)) * kLn2 : kLseNotFinite;
                    if (direct) p.lse_direct[row0 + r] = lse;
                    else p.lse_part[(p.chunk0 + chunk) * all_rows + row0 + r] = lse;
                }
                const bool ok = __all_sync(0xffffffffu, mbar_wait(&sh->o_done[(n_tiles - 1) & 1], ((n_tiles - 1) >> 1) & 1, abort_flag));
                tc_fence_after();
                if (ok) {
                    // The normalised rows are staged over the K, V and Q tiles, which no product reads any more, as 128-byte
                    // swizzled boxes of 64 rows and leave with tiled stores (which cut off rows past the request's end).
                    // This thread's columns are latent dims 256 half + 128 w + 0 .. 127.
#pragma unroll 1
                    for (int i = 0; i < 4; ++i) {
                        uint32_t orr[32];
                        tmem_ld32(tmem_base + lane_base + (uint32_t)(128 * w + 32 * i), orr);
                        tmem_ld_wait();
                        if (direct) {
                            uint8_t* box = sK + (2 * quarter + (i >> 1)) * SLAB + row * 128;
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                uint4 v;
                                uint32_t* vv = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const uint32_t* x = orr + 8 * c + 2 * e;
                                    vv[e] = pack_bf16(__uint_as_float(x[0]) * inv, __uint_as_float(x[1]) * inv);
                                }
                                *reinterpret_cast<uint4*>(box + (((4 * (i & 1) + c) ^ (row & 7)) * 16)) = v;
                            }
                        } else {
                            uint8_t* box = sK + (4 * quarter + i) * SLAB + row * 128;
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                const float4 v = make_float4(__uint_as_float(orr[4 * c]) * inv, __uint_as_float(orr[4 * c + 1]) * inv,
                                                             __uint_as_float(orr[4 * c + 2]) * inv, __uint_as_float(orr[4 * c + 3]) * inv);
                                *reinterpret_cast<float4*>(box + ((c ^ (row & 7)) * 16)) = v;
                            }
                        }
                    }
                    fence_proxy_async();
                    staged = true;
                }
            }
            softmax_sync();
            // one thread issues the stores; a wait that gave up has set the flag, and nothing is stored
            if (threadIdx.x == 128 && staged && !*abort_flag && 64 * (int)rank < n_rows) {
                const int n_box = p.o_lat_direct != nullptr ? 8 : 16;
                const int slot = p.o_lat_direct != nullptr ? 0 : p.chunk0 + chunk;
                for (int i = 0; i < n_box; ++i) tma_store_4d(&tm_o, sK + i * SLAB, i * 64, tile * 128 + 64 * (int)rank, b, slot);
                bulk_commit();
                bulk_wait_read();   // the staging buffer must outlive the copy; the kernel end publishes the writes
            }
        } else if (E8 && warp == 3) {
            // ---------------- powers of two of a tile's tokens, 4 per lane
            auto load = [&](int j) {
                const int t0 = tok_begin + j * TOK + 4 * lane;
                if (j >= n_tiles || t0 >= tok_end) return 0x7f7f7f7fu;
                const int page = page_at(t0);
                return page >= p.num_pages ? 0x7f7f7f7fu
                                           : *reinterpret_cast<const uint32_t*>(p.exponents + (int64_t)page * p.page_size + t0 % p.page_size);
            };
            uint32_t next = load(0);
            bool wide = false;
            for (int j = 0; j < n_tiles; ++j) {
                const uint32_t bytes = next;
                next = load(j + 1);
                if (j >= 4 && !mbar_wait_warp(&sh->sc_empty[j & 3], ((j >> 2) & 1) ^ 1, abort_flag)) break;
                float sc[4], lg[4], isc[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t e = (bytes >> (8 * i)) & 0xffu;
                    sc[i] = (e == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(e << 23)) * p.scale_log2;    // (byte 0, 2^-127: zero)
                    lg[i] = (float)((int)e - 127);
                    isc[i] = e == 255u ? 1.f : __uint_as_float((254u - e) << 23);
                    wide = wide || (e != 255u && (e < 87u || e > 167u) && tok_begin + j * TOK + 4 * lane + i < tok_end);
                }
                wide = __any_sync(0xffffffffu, wide);
                *reinterpret_cast<float4*>(&sh->sc[E8 ? j & 3 : 0][E8 ? 4 * lane : 0]) = make_float4(sc[0], sc[1], sc[2], sc[3]);
                *reinterpret_cast<float4*>(&sh->lg[E8 ? j & 3 : 0][E8 ? 4 * lane : 0]) = make_float4(lg[0], lg[1], lg[2], lg[3]);
                *reinterpret_cast<float4*>(&sh->isc[E8 ? j & 3 : 0][E8 ? 4 * lane : 0]) = make_float4(isc[0], isc[1], isc[2], isc[3]);
                if (lane == 0) sh->wide[E8 ? j & 3 : 0] = wide;
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh->sc_full[j & 3]);
            }
        } else if (warp == 1) {
            // (odd CTA) The output projection behind this kernel reads W_UV: every pair requests its share into L2.
            const uint64_t at = ((uint64_t)item * 32u + (uint32_t)lane) * p.l2_bytes;
            if (at < p.l2_total)
                asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(p.l2_base + at),
                             "r"(min(p.l2_bytes, p.l2_total - (uint32_t)at)) : "memory");
        }
    } else {
        // empty chunk: weight zero in the merge (a request without any latent token: zero latent output)
        const int r = 64 * (int)rank + (int)threadIdx.x - 128;
        if (warp >= 4 && threadIdx.x < 192 && r < n_rows) {
            if (p.o_lat_direct) {
                p.lse_direct[row0 + r] = -INFINITY;
                for (int l = 0; l < 512; l += 8)
                    *reinterpret_cast<uint4*>(p.o_lat_direct + (row0 + r) * 512 + l) = make_uint4(0, 0, 0, 0);
            } else {
                p.lse_part[(p.chunk0 + chunk) * all_rows + row0 + r] = -INFINITY;
            }
        }
    }

    if (bad_page && p.status) atomicOr(p.status, TYPHOON_MLA_STATUS_BAD_PAGE);
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        // A wait gave up.  Before the shared memory is released the copies in flight are awaited (with a limit): the even CTA's
        // barriers count those of both CTAs, and neither CTA leaves before the other (the cluster barrier below).
        if ((warp == 0 || warp == 2) && issued > 0) {
            if (rank == 0 && warp == 0) {
                for (int s = 0; s < KS && s < issued; ++s) {
                    const int j = issued - 1 - (issued - 1 - s) % KS;      // last tile issued into stage s
                    for (int h = 0; h < 2; ++h) mbar_drain(&sh->k_full[s][h], (j / KS) & 1);
                }
                mbar_drain(&sh->q_full, 0);
            }
            if (rank == 0 && warp == 2 && first_special > 0)
                for (int nb = 0; nb < X::NV; ++nb) mbar_drain(&sh->v_full[nb], (min(issued, first_special) - 1) & 1);
            if (warp == 2 && issued > first_special) mbar_drain(&sh->v_tail, (issued - 1 - first_special) & 1);
        }
        if (threadIdx.x == 0 && p.status) atomicOr(p.status, 8);
    }
    __syncwarp();
    cluster_sync();
    if (warp == 1) tmem_dealloc_pair(tmem_base, 512);
}

// Rows of 512 bytes (codes) or 1 KB as [128 bytes | tokens of a page | slab | page], so that a box of two slabs is one copy
cudaError_t make_kv_tmaps(const typhoon_mla_cache_t& c, CUtensorMap* tm_ckv, CUtensorMap* tm_kpe) {
    const bool e8 = c.ckv_exponents != nullptr;
    const uint64_t row = (uint64_t)c.ckv_token_stride * (e8 ? 1 : 2), pages = (uint64_t)c.num_pages;
    {
        uint64_t dims[4] = {64, (uint64_t)c.page_size, e8 ? 4u : 8u, pages};
        uint64_t str[3] = {row, 128, (uint64_t)c.page_size * row};
        uint32_t box[4] = {64, 64, 2, 1};
        cudaError_t e = make_tmap_bf16(tm_ckv, c.ckv_pages, 4, dims, str, box);
        if (e != cudaSuccess) return e;
    }
    uint64_t dims[3] = {64, (uint64_t)c.page_size, pages};
    uint64_t str[2] = {(uint64_t)c.kpe_token_stride * 2, (uint64_t)c.page_size * c.kpe_token_stride * 2};
    uint32_t box[3] = {64, 64, 1};
    return make_tmap_bf16(tm_kpe, c.kpe_pages, 3, dims, str, box);
}

}  // namespace

cudaError_t set_attrs_draft_sm100() {
    cudaError_t e = cudaFuncSetAttribute(draft_pair_sm100_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kDraftSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(draft_pair_sm100_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kDraftSmem);
    return e;
}

cudaError_t launch_draft_sm100(const DraftAttn& a, void* o_lat_direct, float* lse_direct, int* status, cudaStream_t s) {
    if (a.B <= 0 || a.n_chunks <= 0) return cudaSuccess;
    if (a.chunk % TOK != 0 || a.S < 1 || a.S > 64 || a.H > 128) return cudaErrorInvalidValue;
    const bool e8 = a.cache->ckv_exponents != nullptr;
    const int rows = a.S * a.H;
    const int64_t all_rows = (int64_t)a.B * rows;
    const bool direct = o_lat_direct != nullptr;
    CUtensorMap tm_qa, tm_qp, tm_ckv, tm_kpe, tm_o;
    uint32_t box[2] = {64, 64};
    {   // the queries as one matrix of 1 KB rows (512 values, or both terms of 512); rows past the end read as zeros
        uint64_t dims[2] = {512, (uint64_t)all_rows};
        uint64_t str[1] = {512 * 2};
        cudaError_t e = make_tmap_bf16(&tm_qa, a.q_abs, 2, dims, str, box);
        if (e != cudaSuccess) return e;
        dims[0] = 64;
        str[0] = 64 * 2;
        e = make_tmap_bf16(&tm_qp, a.q_pe, 2, dims, str, box);
        if (e != cudaSuccess) return e;
    }
    cudaError_t e = make_kv_tmaps(*a.cache, &tm_ckv, &tm_kpe);
    if (e != cudaSuccess) return e;
    {   // output rows as [512 values | rows of a request | requests | slots]; fp32 values are described as pairs of 16-bit elements
        const uint64_t w = direct ? 512 : 1024;
        uint64_t dims[4] = {w, (uint64_t)rows, (uint64_t)a.B, direct ? 1u : (uint64_t)(a.chunk0 + a.n_chunks)};
        uint64_t str[3] = {w * 2, (uint64_t)rows * w * 2, (uint64_t)all_rows * w * 2};
        uint32_t obox[4] = {64, 64, 1, 1};
        e = make_tmap_bf16(&tm_o, direct ? o_lat_direct : a.o_part, 4, dims, str, obox);
        if (e != cudaSuccess) return e;
    }
    DraftParams p{};
    p.B = a.B; p.S = a.S; p.H = a.H; p.rows = rows;
    p.row_tiles = (rows + 127) / 128; p.chunk = a.chunk; p.n_chunks = a.n_chunks; p.chunk0 = a.chunk0;
    p.page_size = a.cache->page_size; p.max_pages = a.max_pages; p.num_pages = a.cache->num_pages;
    p.block_table = a.block_table; p.seq_lens = a.seq_lens; p.draft_lens = a.draft_lens; p.mask = a.mask;
    p.desc = reinterpret_cast<const int4*>(a.desc);
    p.scale_log2 = a.scale * kLog2e;
    p.lse_part = a.lse_part;
    p.o_lat_direct = static_cast<__nv_bfloat16*>(o_lat_direct); p.lse_direct = lse_direct; p.status = status;
    p.q_tau = a.q_tau; p.exponents = a.cache->ckv_exponents;
    const int64_t items = (int64_t)p.row_tiles * a.n_chunks * a.B;
    if (items > INT32_MAX / 2) return cudaErrorInvalidValue;
    p.l2_base = static_cast<const char*>(a.w_uv);
    p.l2_total = a.w_uv ? (uint32_t)a.H * 128u * 512u * 2u : 0u;
    p.l2_bytes = (uint32_t)(p.l2_total / (items * 32) / 16 + 1) * 16u;
    auto* kernel = e8 ? draft_pair_sm100_kernel<true> : draft_pair_sm100_kernel<false>;
    return launch_pdl(kernel, dim3((unsigned)(2 * items)), dim3(384), kDraftSmem, s, tm_qa, tm_qp, tm_ckv, tm_kpe, tm_o, p);
}

}  // namespace tmla
