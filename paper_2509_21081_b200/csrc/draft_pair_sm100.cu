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
// Instead the products run on the codes (kind::f8f6f4, twice the rate of 16 bits) and the other operand is split into 8-bit numbers.
//   Q: two E4M3 numbers, the nearest one and the nearest one to the rest: 4 significant bits, a sign and 4 more, at least the 8 bits of
//   bf16 (with m = the mantissa of a bf16 value as an integer in [128, 256) the nearest multiple of 16 and the rest, at most 8, are
//   both exact; split from 32 bits the sum is off by 6e-4 of the value in the mean square, bf16 by 1.6e-3).  A row is scaled by a
//   power of two to an amax in [224, 448], so an element loses bits only where it is 2^-10 of the row's largest (by 2^-18 of that at
//   most, in each of 512 dims).
//   P: three E5M2 numbers of 3 significant bits.  A weight may be small and still count, being one of many: what its rounding takes away
//   has to be small next to the weight itself, as with bf16, not next to the row's largest.  (Two E4M3 numbers end at 2^-9, 2^-14 of the
//   reference: 4096 equal tokens behind one with 0.8 of the weight vanished, 16 % of the output.)  With 2^11 at the reference and at most
//   2^15 a weight is good to 2^-8.6 of itself (5e-4 in the mean square) down to 2^-19 of the row's largest contribution, below that to
//   2^-27.8 of it: 2^19 tokens in an item could lose 2^-8.8 together.  Two E5M2 numbers would have 7 bits.
// Two and three products at twice the rate, on half the cache bytes.
// The rope part (16-bit, unscaled) goes to an accumulator of its own, and a logit is S_lat * 2^(tau + e_t) + S_rope.  The token's power
// of two belongs to its values as well: with x the scaled logit in log2 units P = 2^(x + e_t - n) against a reference n of the x + e_t,
// while the row sum is of 2^(x - m) against a reference m of the x (per thread; any within 2^40 will do in 32 bits):
// P = 2^(x - m) * 2^e_t * kappa with kappa = 2^(m - n) per thread and tile.  n is kept within 2^92 of the largest weight (and of the
// largest power of two), where kappa is a normal number: tokens whose values are under 2^-92 next to their weight count as zeros.
//
// (Query absorption splits Q, from 32 bits.  P is split here, from its rounding to fp16, 11 bits: the high byte of an fp16 number is an
// E5M2 number, so a term is a byte selection and the rest an exact subtraction.)
//
// Warp roles (12 warps per CTA): warp 0 loads K tiles (and Q), warp 2 the second operand; warp 1 allocates tensor memory and in
// the even CTA issues both products (in the odd one it requests W_UV into L2); warp 3 turns the tokens' exponent bytes into floats;
// warps 4-11: softmax and epilogue, a thread per row and 32 tokens of a tile.
//
// What bounds it (B200; 64 requests of 1024 rows over 2112 tokens each, 16 / 8 bits: 236 / 327 us, 1.27 / 0.92 PFLOP/s; 74 requests of
// 128 rows over 4096 tokens that nobody shares 75 / 96 us; 296 of 128 rows over 512 tokens 61 / 71; one tile per pair 12.8 / 14.5):
//   - 16 bits: a tile takes 2480 clocks, 2176 of them products; the rest is the reload of V, for which there is one stage (K, V, Q and P
//     fill shared memory; 136 KB come from L2 per CTA and tile).
//   - 8 bits: 3600 clocks for 2600 of products: the softmax warps' own chain (two per scheduler, in step by the vote).  Sixteen of them
//     with half the tokens each take as long; requesting the next logits earlier needs more registers than there are.  The third term
//     of P costs 12 % of the first shape above, half of it as products, half in the softmax warps (two terms of 3 bits would do without).
//   - an item costs 7000 clocks beside its tiles: result 3000, last product 1100, drafts' values read through 1000, first logits 1000.
//     Hence pairs that walk through items with loads one item ahead (one item per pair and launch: 10 us each).
#include <algorithm>
#include <cstddef>

#include "kernels.h"
#include "sm100.cuh"

namespace tmla {
namespace {

using namespace sm100;

constexpr int TOK = 128;
constexpr int SLAB = 64 * 128;                   // [64 rows][128 bytes], swizzled
constexpr float kLog2Off = 11.f, kMostP = 32768.f;  // 8 bits: P at the reference is 2^11, and at most 2^15 (fp16 and E5M2 end above that)
constexpr float kLog2Floor = 92.f;               // 8 bits: references are no further below the largest weight than this
constexpr float kRescale16 = 8.f;                // 16 bits: log2 above the reference

struct DraftParams {
    int B, S, H, rows;     // rows = S * H per request
    int row_tiles, chunk, n_chunks;
    int chunk0;            // partial slot of the first chunk
    int Ls, sh_chunk, n_sh_chunks, n_sh_items;   // prefix items: 128 rows of the stacked [B * rows] matrix and a chunk of the prefix
    int page_size, max_pages, num_pages;
    const int32_t* block_table;
    const int32_t* seq_lens;
    const int32_t* draft_lens;   // optional [B]
    const uint64_t* mask;        // optional [B, S]
    const int4* desc;      // optional, per launch position: {request, clamped suffix length, page 0, page 1}
    float scale_log2;
    float* o_part;         // [slots][B * rows][512]
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
    static constexpr int KS = E8 ? 2 : 1;                     // stages of K's first half of dims (its second half and the rope keys: one)
    static constexpr int VS = E8 ? 2 : 1;                     // stages of the second operand
    static constexpr int LAT = E8 ? 4 : 8;                    // latent slabs of 64 tokens
    static constexpr int K_BYTES = (LAT / 2 * KS + LAT / 2 + 1) * SLAB;   // 64 tokens: latent slabs | rope slab
    static constexpr int NV = E8 ? 1 : 2;                     // copy groups of the second operand
    static constexpr int V_BYTES = (E8 ? 4 : 8) * SLAB;       // a stage: 128 tokens x 256 dims
    static constexpr int Q_BYTES = 9 * SLAB;                  // 8 bits: both terms of 4 slabs, and rope
    static constexpr int P_BYTES = (E8 ? 3 : 2) * SLAB;       // 16 bits: [2 token halves][64 rows][64]; 8 bits: [3 terms][64 rows][128]
    static constexpr int GROUP = E8 ? 32 : 16;                // tokens of one MMA of the second product
    static constexpr int TPT = 32;                            // tokens of a tile per softmax thread
    static constexpr int PARTS = TOK / TPT;                   // softmax threads per row
    static constexpr int WARPS = 2 * PARTS;                   // softmax warps
    static constexpr int THREADS = 128 + 32 * WARPS;
};

template <bool E8>
struct Shared {
    uint64_t q_full;                  // these four groups count the copies of both CTAs, in the even CTA
    uint64_t k_full[Shape<E8>::KS][2];   // [stage][half of the dims] (the second half has stage 0 only)
    uint64_t v_full[2];               // 16 bits: block 0 | 1; 8 bits: stage
    uint64_t p_ready;                 // one arrival per softmax warp of both CTAs
    uint64_t k_empty[Shape<E8>::KS][2], v_empty[2];  // in both CTAs, by the commits of the even one
    uint64_t s_ready[2];
    uint64_t o_done[2];               // second product of tile j: o_done[j & 1]
    uint64_t v_tail[2];               // own copies of the second operand of a tile whose values are gone through first (8 bits: per stage)
    uint64_t q_empty;                 // the last logits of an item are there (both CTAs)
    uint64_t sc_full[4], sc_empty[4]; // 8 bits: powers of two of tile j in slot j & 3; one arrival per softmax warp when they are read
    uint32_t tmem_base;
    int abort_flag;
    float red[Shape<E8>::PARTS][64];  // [part of the tile's tokens][row]
    float red2[E8 ? Shape<E8>::PARTS : 1][E8 ? 64 : 1];
    alignas(16) float sigma[E8 ? 4 : 1][E8 ? TOK : 4];       // powers of two of a tile's tokens
};

// (all of an SM's shared memory either way: no other kernel that allocates tensor memory fits beside a CTA)
constexpr int kDraftSmem = 232448;
template <bool E8>
constexpr int smem_used() {
    using X = Shape<E8>;
    return X::K_BYTES + X::VS * X::V_BYTES + X::Q_BYTES + X::P_BYTES + 1024 + (int)sizeof(Shared<E8>);
}
static_assert(smem_used<false>() <= kDraftSmem && smem_used<true>() <= kDraftSmem, "shared memory of one SM");

constexpr int kSoftmaxBar = 1;
template <int N>
__device__ __forceinline__ bool vote_or(bool pred) {   // over the N softmax threads
    uint32_t r;
    asm volatile(
        "{\n.reg .pred p, q;\nsetp.ne.b32 q, %2, 0;\n"
        "bar.red.or.pred p, %1, %3, q;\n"
        "selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(r) : "n"(kSoftmaxBar), "r"(pred ? 1u : 0u), "n"(N) : "memory");
    return r != 0;
}
template <int N>
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync %0, %1;\n" ::"n"(kSoftmaxBar), "n"(N) : "memory"); }

// 32 bytes of one row
__device__ __forceinline__ void store_sector(void* p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                 "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
template <int N>
__device__ __forceinline__ float max_of(const float (&x)[N]) {
    static_assert(N % 4 == 0 || N == 1, "");
    if (N == 1) return x[0];
    float a = x[0], b = x[N / 2];
#pragma unroll
    for (int c = 1; c < N / 2 - 1; c += 2) {
        a = max3(a, x[c], x[c + 1]);
        b = max3(b, x[N / 2 + c], x[N / 2 + c + 1]);
    }
    return fmaxf(max3(a, b, x[N / 2 - 1]), x[N - 1]);
}

// 4 values as fp16 (two words, the lower half first): codes of three E5M2 terms, the value cut to 3 significant bits, the rest cut to 3, and the
// rest of that rounded to 3 (half up: its bits are a magnitude).  Not a number: the first term is not.
__device__ __forceinline__ void split4_e5m2(uint32_t a, uint32_t b, uint32_t& first, uint32_t& second, uint32_t& third) {
    auto cut_off = [](uint32_t x) {
        uint32_t d;
        asm("sub.rn.f16x2 %0, %1, %2;\n" : "=r"(d) : "r"(x), "r"(x & 0xff00ff00u));
        return d;
    };
    auto high_bytes = [](uint32_t x, uint32_t y) { return __byte_perm(x, y, 0x7531); };
    const uint32_t a1 = cut_off(a), b1 = cut_off(b);
    first = high_bytes(a, b);
    second = high_bytes(a1, b1);
    third = high_bytes(cut_off(a1) + 0x00800080u, cut_off(b1) + 0x00800080u);
}

template <bool E8>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Shape<E8>::THREADS, 1)
draft_pair_sm100_kernel(const __grid_constant__ CUtensorMap tm_qa, const __grid_constant__ CUtensorMap tm_qp,
                        const __grid_constant__ CUtensorMap tm_ckv, const __grid_constant__ CUtensorMap tm_kpe,
                        const __grid_constant__ CUtensorMap tm_ckv_sh, const __grid_constant__ CUtensorMap tm_kpe_sh, DraftParams p) {
    using X = Shape<E8>;
    constexpr int KS = X::KS, VS = X::VS, LAT = X::LAT, HALF = LAT / 2, TPT = X::TPT, PARTS = X::PARTS, SM = 32 * X::WARPS;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sK = smem;
    uint8_t* sV = sK + X::K_BYTES;
    uint8_t* sQ = sV + X::VS * X::V_BYTES;
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
        if (lane < n_bars) mbar_init(all + lane, all + lane == &sh->p_ready ? 2 * X::WARPS : all + lane >= &sh->sc_empty[0] ? X::WARPS : 1);
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

    // Work items: over the prefix (absorb-only steps of a 16-bit cache), chunk fastest, then 128 rows; over the suffixes, row tile
    // fastest (they share the tokens), then chunk, then request in longest-first order.  A pair takes every
    // n_pairs-th, in alternating direction; what it loads for the next item starts when the logits of the last tile are there, beside
    // that tile's softmax, product and the item's epilogue.
    const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const int n_items = p.n_sh_items + p.row_tiles * p.n_chunks * p.B;
    const int64_t all_rows = (int64_t)p.B * p.rows;
    struct Item {
        int b, pg0, pg1;          // request (prefix items: -1)
        int slot;                 // partial slot
        int row0, n_rows;         // rows of the stacked matrix (n_rows 0: no item)
        int tile;                 // ... of the request
        int tok_begin, tok_end, n_tiles, n_last;     // n_last: tokens of the last tile
        int draft0;               // first draft
        int first_special;        // tiles from this one on are gone through in shared memory before the second product
    };
    auto item_index = [&](int k) { return k * n_pairs + ((k & 1) ? n_pairs - 1 - pair : pair); };
    // {request, clamped suffix length, first two pages} of item k; length -1: no such item, request -1: over the prefix
    auto desc_of = [&](int k) {
        const int i = item_index(k);
        int4 d = make_int4(0, -1, -1, -1);
        if (i < p.n_sh_items) {
            d.x = -1;
            d.y = p.Ls;
        } else if (i < n_items) {
            const int z = (i - p.n_sh_items) / (p.row_tiles * p.n_chunks);
            if (p.desc != nullptr) d = p.desc[z];
            else d = make_int4(z, min(max(p.seq_lens[z], 0), p.max_pages * p.page_size), -1, -1);
        }
        return d;
    };
    auto item_at = [&](int k, int4 d) {
        Item it;
        // (through shuffles: the role warps' loops are then known to be uniform)
        const int len = __shfl_sync(0xffffffffu, d.y, 0);
        it.b = __shfl_sync(0xffffffffu, d.x, 0);
        it.pg0 = d.z;
        it.pg1 = d.w;
        const bool prefix = it.b < 0;
        const int i = item_index(k) - (prefix ? 0 : p.n_sh_items);
        const int tile = prefix ? i / p.n_sh_chunks : i % p.row_tiles;
        const int chunk = prefix ? i % p.n_sh_chunks : (i / p.row_tiles) % p.n_chunks;
        it.slot = prefix ? chunk : p.chunk0 + chunk;
        it.row0 = (prefix ? 0 : it.b * p.rows) + tile * 128;
        it.n_rows = len < 0 ? 0 : min(128, (prefix ? p.B * p.rows : p.rows) - tile * 128);
        it.tile = tile;
        it.tok_begin = chunk * (prefix ? p.sh_chunk : p.chunk);
        it.tok_end = min(max(len, 0), it.tok_begin + (prefix ? p.sh_chunk : p.chunk));
        it.n_tiles = it.tok_end > it.tok_begin ? (it.tok_end - it.tok_begin + TOK - 1) / TOK : 0;
        it.n_last = it.tok_end - it.tok_begin - (it.n_tiles - 1) * TOK;
        // (no drafts in the prefix; a single token that sees itself hides nothing)
        const int n_draft = p.draft_lens != nullptr && it.n_tiles > 0 && !prefix ? min(max(p.draft_lens[it.b], 0), p.S) : p.S;
        it.draft0 = __shfl_sync(0xffffffffu, prefix || (p.S == 1 && p.mask == nullptr) ? len : len - n_draft, 0);
        // values of drafts that are not finite are zeroed (see above), and the rest of the last group of tokens, which may hold anything
        // (the handle's copy of the prefix is padded with zeros)
        it.first_special = it.draft0 >= it.tok_end ? it.n_tiles : max(it.draft0 - it.tok_begin, 0) / TOK;
        if (it.n_tiles > 0 && it.n_last % X::GROUP != 0 && !prefix) it.first_special = min(it.first_special, it.n_tiles - 1);
        return it;
    };
    const int n_rounds = n_items > 0 ? (n_items + n_pairs - 1) / n_pairs : 0;
    pdl_wait();

    bool bad_page = false;   // loading warps only: a page id of the caller's table was out of range
    auto page_at = [&](const Item& it, int t0) {   // physical page of token t0 < tok_end
        const int idx = t0 / p.page_size;
        int page = (p.desc != nullptr && idx < 2) ? (idx == 0 ? it.pg0 : it.pg1) : p.block_table[(int64_t)it.b * p.max_pages + idx];
        // The tensor maps end at num_pages: a coordinate at or past it reads as zeros instead of touching memory the caller does
        // not own.  The violation is reported through the status word.
        if ((unsigned)page >= (unsigned)p.num_pages) {
            bad_page = true;
            page = p.num_pages;
        }
        return page;
    };
    // physical page and slot of half `h` (64 tokens) of tile j; a half past the end reads as zeros
    auto page_of = [&](const Item& it, int j, int h, int& page, int& slot) {
        const int t0 = it.tok_begin + j * TOK + h * 64;
        if (it.b < 0) {           // 64-token pages of the handle's copy
            page = t0 / 64;
            slot = 0;
            return;
        }
        slot = t0 % p.page_size;
        page = __shfl_sync(0xffffffffu, t0 < it.tok_end ? page_at(it, t0) : p.num_pages, 0);
    };

    // In every role g counts the tiles of all items so far (stages and phases go by it), n the items that have any.
    // loading warps, for the abort path: tiles, items, plain and special tiles per stage
    int issued = 0, issued_n = 0, issued_v[2] = {0, 0}, issued_t[2] = {0, 0};
    if (warp == 0) {
        // ---------------- Q and K tiles
        const uint32_t ld = elect_one() ? 1u : 0u;
        const uint32_t ld_even = rank == 0 ? ld : 0u;
        // tiles are requested into L2 KS + 1 ahead of the load into a freed stage, the next item's as well
        Item pf = item_at(0, desc_of(0));
        int pf_k = 0, pf_j = 0;
        auto prefetch_next = [&] {
            while (pf_k < n_rounds && pf_j >= pf.n_tiles) {
                ++pf_k;
                pf_j = 0;
                if (pf_k < n_rounds) pf = item_at(pf_k, desc_of(pf_k));
            }
            if (pf_k >= n_rounds) return;
            int page, slot;
            page_of(pf, pf_j, (int)rank, page, slot);
            const CUtensorMap* tc = pf.b < 0 ? &tm_ckv_sh : &tm_ckv;
#pragma unroll 1
            for (int i = 0; i < HALF; ++i) tma_prefetch_4d_if(ld, tc, 0, slot, 2 * i, page);
            tma_prefetch_3d_if(ld, pf.b < 0 ? &tm_kpe_sh : &tm_kpe, 0, slot, page);
            ++pf_j;
        };
        bool ok = true;
        int g = 0, n = 0;
        Item it = pf;
        for (int k = 0; k < n_rounds && ok; ++k) {
            if (k > 0) it = item_at(k, desc_of(k));
            const CUtensorMap* tc = it.b < 0 ? &tm_ckv_sh : &tm_ckv;
            for (int j = 0; j < it.n_tiles && ok; ++j, ++g) {
                int page, slot;
                page_of(it, j, (int)rank, page, slot);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int stages = h == 0 ? KS : 1, s = g % stages;
                    uint8_t* dst = sK + (h == 0 ? s * HALF : KS * HALF) * SLAB;
                    if (g >= stages) ok = ok && mbar_wait_warp(&sh->k_empty[s][h], ((g / stages) & 1) ^ 1, abort_flag);
                    if (!ok) break;
                    const uint32_t kf = cluster_map(&sh->k_full[s][h], 0);
                    mbar_arrive_expect_tx_if(ld_even, &sh->k_full[s][h], 2 * (HALF + h) * SLAB);
#pragma unroll
                    for (int i = 0; i < HALF; i += 2) tma_load_4d_pair_if(ld, dst + i * SLAB, tc, kf, 0, slot, HALF * h + i, page);
                    if (h == 1) tma_load_3d_pair_if(ld, dst + HALF * SLAB, it.b < 0 ? &tm_kpe_sh : &tm_kpe, kf, 0, slot, page);
                }
                issued = g + 1;
                if (j == 0 && ok) {
                    if (n > 0) ok = mbar_wait_warp(&sh->q_empty, (n - 1) & 1, abort_flag);
                    if (!ok) break;
                    const uint32_t qf = cluster_map(&sh->q_full, 0);
                    const int y = it.row0 + 64 * (int)rank;
                    mbar_arrive_expect_tx_if(ld_even, &sh->q_full, 2 * X::Q_BYTES);
#pragma unroll 1
                    for (int sl = 0; sl < 8; ++sl) tma_load_2d_pair_if(ld, sQ + sl * SLAB, &tm_qa, qf, sl * 64, y);
                    tma_load_2d_pair_if(ld, sQ + 8 * SLAB, &tm_qp, qf, 0, y);
                    issued_n = ++n;
                    if (n == 1) {
                        pf_j = 1;       // (this tile itself is on its way)
                        for (int i = 0; i < KS; ++i) prefetch_next();
                    }
                }
                prefetch_next();
            }
        }
    } else if (warp == 2) {
        // ---------------- second operand: latent dims [256 rank, + 256) of all 128 tokens
        const uint32_t ld = elect_one() ? 1u : 0u;
        const uint32_t ld_even = rank == 0 ? ld : 0u;
        const uint32_t vf[2] = {cluster_map(&sh->v_full[0], 0), cluster_map(&sh->v_full[1], 0)};
        const uint32_t vt[2] = {cluster_map(&sh->v_tail[0], rank), cluster_map(&sh->v_tail[1], rank)};
        bool ok = true;
        int g = 0;
        for (int k = 0; k < n_rounds && ok; ++k) {
            const Item it = item_at(k, desc_of(k));
            const CUtensorMap* tc = it.b < 0 ? &tm_ckv_sh : &tm_ckv;
            for (int j = 0; j < it.n_tiles && ok; ++j, ++g) {
                int page[2], slot[2];
                page_of(it, j, 0, page[0], slot[0]);
                page_of(it, j, 1, page[1], slot[1]);
                const bool special = j >= it.first_special;  // counted by the CTA's own barrier: its threads go through the values
                const int st = g % VS;
                uint8_t* dst = sV + st * X::V_BYTES;
#pragma unroll
                for (int nb = 0; nb < X::NV; ++nb) {
                    const int i = E8 ? st : nb;
                    if (g >= VS) ok = ok && mbar_wait_warp(&sh->v_empty[i], ((g / VS) & 1) ^ 1, abort_flag);
                    if (!ok) break;
                    // (v_empty of the first block: the softmax of the stage's previous tile is past its wait on v_tail)
                    if (special && nb == 0) mbar_arrive_expect_tx_if(ld, &sh->v_tail[st], X::V_BYTES);
                    if (!special) mbar_arrive_expect_tx_if(ld_even, &sh->v_full[i], 2 * X::V_BYTES / X::NV);
                    const uint32_t bar = special ? (st ? vt[1] : vt[0]) : (i ? vf[1] : vf[0]);
                    // 16 bits: blocks of 128 dims, [block][token half][2 slabs]; 8 bits: [token half][2 slabs = blocks]
                    const int slab = E8 ? 2 * (int)rank : 4 * (int)rank + 2 * nb;
                    tma_load_4d_pair_if(ld, dst + (4 * nb) * SLAB, tc, bar, 0, slot[0], slab, page[0]);
                    tma_load_4d_pair_if(ld, dst + (4 * nb + 2) * SLAB, tc, bar, 0, slot[1], slab, page[1]);
                }
                if (special) ++issued_t[st];
                else ++issued_v[st];
            }
        }
    } else if (warp == 1 && rank == 0) {
        // ---------------- both products (even CTA)
        constexpr uint32_t idesc_s = idesc_bf16(128, 128, false, false);
        constexpr uint32_t idesc_s8 = idesc_e4m3(128, 128, false, false);
        constexpr uint32_t idesc_o = E8 ? idesc_e5m2_e4m3(128, 256, false, true) : idesc_bf16(128, 256, false, true);
        const uint32_t qa = smem_u32(sQ), va = smem_u32(sV), pa = smem_u32(sP);
        bool ok = true;
        int g = 0, n = 0;
        uint32_t v_phase = 0;               // bit i: parity of the next phase of v_full[i] (per stage; only plain tiles have one)
        for (int k = 0; k < n_rounds && ok; ++k) {
            const Item it = item_at(k, desc_of(k));
            if (it.n_tiles == 0) continue;
            ok = mbar_wait_warp(&sh->q_full, n & 1, abort_flag);
            ++n;
            for (int j = 0; j <= it.n_tiles && ok; ++j) {
                if (j < it.n_tiles) {
                    // S of tile g into buffer g & 1: the softmax of tile g - 2 has read it (p_ready of that tile, awaited below)
                    const uint32_t d = tmem_base + 256u + (uint32_t)(g & 1) * (E8 ? 128u : 64u);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int stages = h == 0 ? KS : 1, s = g % stages;
                        const uint32_t ka = smem_u32(sK) + (h == 0 ? s * HALF : KS * HALF) * SLAB;      // slab HALF * h
                        ok = ok && mbar_wait_warp(&sh->k_full[s][h], (g / stages) & 1, abort_flag);
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_one()) {
                            if (E8) {
#pragma unroll
                                for (int sl = HALF * h; sl < HALF * (h + 1); ++sl)
#pragma unroll
                                    for (int t = 0; t < 2; ++t) {
                                        const uint64_t da = smem_desc_k_sw128(qa + (4 * t + sl) * SLAB);
                                        const uint64_t db = smem_desc_k_sw128(ka + (sl - HALF * h) * SLAB);
#pragma unroll
                                        for (int i = 0; i < 4; ++i) umma_pair_8bit(d, da + 2 * i, db + 2 * i, idesc_s8, (sl | t | i) != 0);
                                    }
                                if (h == 1) {
                                    const uint64_t da = smem_desc_k_sw128(qa + 8 * SLAB), db = smem_desc_k_sw128(ka + HALF * SLAB);
#pragma unroll
                                    for (int i = 0; i < 4; ++i) umma_pair_ss(d + 64u, da + 2 * i, db + 2 * i, idesc_s, i != 0);
                                }
                            } else {
#pragma unroll
                                for (int sl = 4 * h; sl < (h == 0 ? 4 : 9); ++sl) {
                                    const uint64_t da = smem_desc_k_sw128(qa + sl * SLAB);
                                    const uint64_t db = smem_desc_k_sw128(ka + (sl - 4 * h) * SLAB);
#pragma unroll
                                    for (int i = 0; i < 4; ++i) umma_pair_ss(d, da + 2 * i, db + 2 * i, idesc_s, (sl | i) != 0);
                                }
                            }
                            umma_pair_commit(&sh->k_empty[s][h]);
                            if (h == 1) umma_pair_commit(&sh->s_ready[g & 1]);
                            if (h == 1 && j == it.n_tiles - 1) umma_pair_commit(&sh->q_empty);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    ++g;
                }
                if (j > 0) {
                    const int t = j - 1, gt = j < it.n_tiles ? g - 2 : g - 1;    // its count over all items
                    const bool last = t == it.n_tiles - 1;
                    const int n_k = last ? (it.n_last + X::GROUP - 1) / X::GROUP : TOK / X::GROUP;
                    ok = mbar_wait_warp(&sh->p_ready, gt & 1, abort_flag);
                    if (!ok) break;
#pragma unroll
                    for (int nb = 0; nb < 2; ++nb) {
                        const int st = gt % VS;
                        if (t < it.first_special && nb < X::NV) {
                            const int i = E8 ? st : nb;
                            ok = ok && mbar_wait_warp(&sh->v_full[i], (v_phase >> i) & 1, abort_flag);
                            v_phase ^= 1u << i;
                        }
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_one()) {
                            const uint32_t d = tmem_base + (uint32_t)nb * 128u;
                            if (E8) {
                                // a group of 32 tokens is 4 KB of the second operand and 32 bytes of P's rows
                                const uint64_t da0 = smem_desc_k_sw128(pa);
                                const uint64_t db0 = smem_desc_mn_sw128(va + st * X::V_BYTES + nb * SLAB, SLAB, 1024);
                                auto product = [&](int i) {
                                    const uint64_t db = db0 + (i >> 1) * (2 * SLAB / 16) + (i & 1) * 256;
                                    umma_pair_8bit(d, da0 + 2 * i, db, idesc_o, (t | i) != 0);
                                    umma_pair_8bit(d, da0 + SLAB / 16 + 2 * i, db, idesc_o, 1);
                                    umma_pair_8bit(d, da0 + 2 * SLAB / 16 + 2 * i, db, idesc_o, 1);
                                };
                                if (n_k == 4) {
#pragma unroll
                                    for (int i = 0; i < 4; ++i) product(i);
                                } else {
#pragma unroll 1
                                    for (int i = 0; i < n_k; ++i) product(i);
                                }
                            } else {
                                const uint64_t da0 = smem_desc_k_sw128(pa);
                                const uint64_t db0 = smem_desc_mn_sw128(va + (4 * nb) * SLAB, SLAB, 1024);
                                auto product = [&](int i) {   // 16 tokens (descriptor addresses count 16-byte units)
                                    umma_pair_ss(d, da0 + (i >> 2) * (SLAB / 16) + 2 * (i & 3), db0 + (i >> 2) * (2 * SLAB / 16) + (i & 3) * 128,
                                                 idesc_o, (t | i) != 0);
                                };
                                if (n_k == 8) {
#pragma unroll
                                    for (int i = 0; i < 8; ++i) product(i);
                                } else {
#pragma unroll 1
                                    for (int i = 0; i < n_k; ++i) product(i);
                                }
                            }
                            if (nb >= 2 - X::NV) umma_pair_commit(&sh->v_empty[E8 ? st : nb]);
                            if (nb == 1) umma_pair_commit(&sh->o_done[gt & 1]);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                }
            }
        }
    } else if (warp >= 4) {
        // ---------------- softmax: thread = (row, part of the tile's tokens); the part's TPT tokens are half `half`, columns TPT * w
        const int w = (warp - 4) >> 2, q = warp & 3;
        const int row = 32 * (q & 1) + lane, half = q >> 1;
        const int part = half * (PARTS / 2) + w;
        const uint32_t lane_base = (uint32_t)(32 * q) << 16;
        const uint32_t p_bar = cluster_map(&sh->p_ready, 0);
        const bool direct = p.o_lat_direct != nullptr;
        int g = 0;
        uint32_t t_phase = 0;               // bit i: parity of the next phase of v_tail[i]
        int4 next = desc_of(0);
        for (int k = 0; k < n_rounds; ++k) {
            const Item it = item_at(k, next);
            next = desc_of(k + 1);        // (asked for an item ahead)
            if (it.n_rows == 0) continue;
            const int n_rows = it.n_rows;
            const int64_t row0 = it.row0;
            if (it.n_tiles == 0) {
                // empty chunk: weight zero in the merge (a request without any latent token: zero latent output)
                const int tid = (int)threadIdx.x - 128, own = min(max(n_rows - 64 * (int)rank, 0), 64);
                const int64_t r0 = row0 + 64 * (int)rank;
                if (tid < own) {
                    if (direct) p.lse_direct[r0 + tid] = -INFINITY;
                    else p.lse_part[(int64_t)it.slot * all_rows + r0 + tid] = -INFINITY;
                }
                if (direct)
                    for (int i = tid; i < own * 64; i += SM) reinterpret_cast<uint4*>(p.o_lat_direct + r0 * 512)[i] = make_uint4(0, 0, 0, 0);
                continue;
            }
            const bool mine = 64 * (int)rank + row < n_rows;      // (else nobody's: sees nothing)
            uint64_t sees = 0;            // bit i: draft i
            if (mine) {
                const int j = (it.tile * 128 + 64 * (int)rank + row) / p.H;      // (unused over the prefix)
                sees = it.b >= 0 && p.mask != nullptr ? p.mask[(int64_t)it.b * p.S + j] : (2ull << (j & 63)) - 1ull;
            }
            const float tau = E8 && mine ? p.q_tau[row0 + 64 * (int)rank + row] : 1.f;
            float m_ref = -INFINITY;      // log2 units; 8 bits: of the logits times the tokens' powers of two
            float m_sum = -INFINITY;      // 8 bits: reference of this thread's row sum, which is of the logits alone
            float l_part[2] = {0.f, 0.f};
            // Powers of two of this part's tokens, loaded a tile ahead: the products keep the shared memory busy, and loads from it are
            // slow beside them.
            float sigma[E8 ? TPT : 1];
            auto load_sigma = [&](int tile_g) {
#pragma unroll
                for (int i = 0; i < TPT / 4; ++i) {
                    const float4 v = *reinterpret_cast<const float4*>(&sh->sigma[E8 ? tile_g & 3 : 0][E8 ? TPT * part + 4 * i : 0]);
                    sigma[E8 ? 4 * i : 0] = v.x; sigma[E8 ? 4 * i + 1 : 0] = v.y; sigma[E8 ? 4 * i + 2 : 0] = v.z; sigma[E8 ? 4 * i + 3 : 0] = v.w;
                }
            };
            if (E8 && *abort_flag == 0 && mbar_wait(&sh->sc_full[g & 3], (g >> 2) & 1, abort_flag)) load_sigma(g);
            for (int j = 0; j < it.n_tiles; ++j, ++g) {
                const int n_valid = j == it.n_tiles - 1 ? it.n_last : TOK;
                bool ok = *abort_flag == 0;
                if (!E8 || j == it.n_tiles - 1) ok = ok && mbar_wait(&sh->s_ready[g & 1], (g >> 1) & 1, abort_flag);
                else if (!mbar_try_wait2(&sh->s_ready[g & 1], (g >> 1) & 1, &sh->sc_full[(g + 1) & 3], ((g + 1) >> 2) & 1))
                    ok = ok && mbar_wait(&sh->s_ready[g & 1], (g >> 1) & 1, abort_flag) &&
                         mbar_wait(&sh->sc_full[(g + 1) & 3], ((g + 1) >> 2) & 1, abort_flag);
                ok = __all_sync(0xffffffffu, ok);
                // bit c: token c of this part is there, and visible to this row
                constexpr uint32_t all_bits = (uint32_t)((1ull << TPT) - 1);
                const int t_rel = TPT * part, first = it.tok_begin + j * TOK + t_rel;
                uint32_t vis = !mine ? 0u : n_valid >= t_rel + TPT ? all_bits : n_valid > t_rel ? (1u << (n_valid - t_rel)) - 1u : 0u;
                if (first + TPT > it.draft0) {
                    const int at = first - it.draft0;      // > -TPT
                    vis &= at >= 64 ? 0u : at >= 0 ? (uint32_t)(sees >> at) : ((uint32_t)sees << -at) | ((1u << -at) - 1u);
                }
                // x[c]: the logit in log2 units above a reference: 16 bits, the row's; 8 bits, this thread's (its row sum's)
                float x[TPT], kappa = 0.f, top = -INFINITY, tsum = 0.f;
                uint32_t pk[TPT / 2];                  // pairs, 16 bits: bf16; 8 bits: fp16
                const float base = E8 ? (m_sum == -INFINITY ? 0.f : m_sum) : (m_ref == -INFINITY ? 0.f : m_ref);
                bool exceed = false;
                // P in the form of the product's operand: 16 bits, 2^x; 8 bits, 2^x sigma kappa, and the sum of 2^x
                auto probabilities = [&] {
                    uint64_t sum = 0ull;      // two 32-bit zeros
                    const uint64_t kappa2 = pack_f32x2(kappa, kappa);
#pragma unroll
                    for (int c = 0; c < TPT; c += 4) {
                        const float p0 = fast_exp2(x[c]), p1 = fast_exp2(x[c + 1]), p2 = fast_exp2(x[c + 2]), p3 = fast_exp2(x[c + 3]);
                        if (E8) {
                            const uint64_t pa = pack_f32x2(p0, p1), pb = pack_f32x2(p2, p3);
                            sum = add_f32x2(add_f32x2(pa, pb), sum);
                            pk[c / 2] = pack_f16_x2(mul_f32x2(pa, mul_f32x2(pack_f32x2(sigma[E8 ? c : 0], sigma[E8 ? c + 1 : 0]), kappa2)));
                            pk[c / 2 + 1] = pack_f16_x2(mul_f32x2(pb, mul_f32x2(pack_f32x2(sigma[E8 ? c + 2 : 0], sigma[E8 ? c + 3 : 0]), kappa2)));
                        } else {
                            pk[c / 2] = pack_bf16(p0, p1);
                            pk[c / 2 + 1] = pack_bf16(p2, p3);
                        }
                    }
                    float s0, s1;
                    unpack_f32x2(sum, s0, s1);
                    tsum = s0 + s1;
                };
                if (ok) {
                    tc_fence_after();
                    const uint32_t s_addr = tmem_base + lane_base + 256u + (uint32_t)((g & 1) * (E8 ? 128 : 64) + TPT * w);
                    uint32_t sr[TPT];
                    tmem_ld32(s_addr, sr);
                    const uint64_t off2 = pack_f32x2(-base, -base), scale2 = pack_f32x2(p.scale_log2, p.scale_log2);
                    if (E8) {
                        uint32_t rr[TPT];
                        tmem_ld32(s_addr + 64u, rr);
                        const uint64_t tau2 = pack_f32x2(tau * p.scale_log2, tau * p.scale_log2);
                        tmem_ld_wait();
#pragma unroll
                        for (int c = 0; c < TPT; c += 2) {
                            const uint64_t s2 = pack_f32x2(__uint_as_float(sr[c]), __uint_as_float(sr[c + 1]));
                            const uint64_t r2 = pack_f32x2(__uint_as_float(rr[c]), __uint_as_float(rr[c + 1]));
                            const uint64_t f2 = mul_f32x2(pack_f32x2(sigma[E8 ? c : 0], sigma[E8 ? c + 1 : 0]), tau2);
                            unpack_f32x2(fma_f32x2(s2, f2, fma_f32x2(r2, scale2, off2)), x[c], x[c + 1]);
                        }
                    } else {
                        tmem_ld_wait();
#pragma unroll
                        for (int c = 0; c < TPT; c += 2)
                            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(sr[c]), __uint_as_float(sr[c + 1])), scale2, off2), x[c], x[c + 1]);
                    }
                    if (vis != all_bits) {
#pragma unroll
                        for (int c = 0; c < TPT; ++c)
                            if (!((vis >> c) & 1u)) {
                                x[c] = -INFINITY;
                                if (E8) sigma[E8 ? c : 0] = 0.f;      // (a hidden token may hold any exponent)
                            }
                    }
                    top = max_of(x);
                    if (E8) {
                        // the reference of this thread's row sum: raised where the sum could leave 32 bits
                        if (top != -INFINITY && (m_sum == -INFINITY || top > 40.f)) {
                            l_part[0] *= m_sum == -INFINITY ? 0.f : fast_exp2(-top);
                            m_sum = base + top;
#pragma unroll
                            for (int c = 0; c < TPT; ++c) x[c] -= top;
                            top = 0.f;
                        }
                        kappa = m_ref == -INFINITY ? 0.f : fast_exp2(fminf(m_sum - m_ref + kLog2Off, 120.f));
                        // some 2^x sigma kappa above its limit?  First by the largest of both factors.  (And kappa, with or without a
                        // power of two, stays far from what 32 bits hold.)
                        const float most_k = max_of(sigma) * kappa;
                        exceed = m_ref == -INFINITY ? top != -INFINITY : fast_exp2(top) * most_k > kMostP;
                        if (exceed && m_ref != -INFINITY) {
                            float most = 0.f;
#pragma unroll
                            for (int c = 0; c < TPT; ++c) most = fmaxf(most, fast_exp2(x[c]) * (sigma[E8 ? c : 0] * kappa));
                            exceed = most > kMostP;
                        }
                        exceed |= fmaxf(most_k, kappa) > 0x1p105f;
                    } else {
                        // (a row without a reference: any logit exceeds it)
                        exceed = top > (m_ref == -INFINITY ? -INFINITY : kRescale16);
                    }
                }
                // (an item's first tile has no reference yet, and does not vote)
                if (j == 0 || vote_or<SM>(exceed)) {
                    // the row's largest logit (8 bits: times the token's power of two)
                    if (E8 && ok) {
                        float most = -INFINITY;
#pragma unroll
                        for (int c = 0; c < TPT; ++c)
                            if (sigma[E8 ? c : 0] > 0.f) most = fmaxf(most, x[c] + (float)((int)(__float_as_uint(sigma[E8 ? c : 0]) >> 23) - 127));
                        // (at least 2^-kLog2Floor of the largest weight and of the largest power of two seen beside it: what is below
                        // counts as nothing)
                        const float sum_ref = m_sum == -INFINITY ? 0.f : m_sum, most_s = max_of(sigma);
                        if (top != -INFINITY)
                            most = fmaxf(most, fmaxf(top, 0.f) - kLog2Floor + (most_s > 1.f ? (float)((int)(__float_as_uint(most_s) >> 23) - 127) : 0.f));
                        top = most + sum_ref;
                    } else {
                        top += base;
                    }
                    sh->red[part][row] = top;
                    softmax_sync<SM>();
                    float cm = sh->red[0][row];
#pragma unroll
                    for (int i = 1; i < PARTS; ++i) cm = fmaxf(cm, sh->red[i][row]);
                    const float m_new = fmaxf(m_ref, cm);
                    const float f = (m_new == -INFINITY) ? 1.f : fast_exp2(m_ref - m_new);
                    m_ref = m_new;
                    if (!E8) {
                        l_part[0] *= f;
                        l_part[1] *= f;
                    }
                    if (j > 0) {
                        // this thread's lane of O (the same row), its part of the 256 columns, once the previous tile's product has
                        // landed
                        if (*abort_flag == 0) mbar_wait(&sh->o_done[(g - 1) & 1], ((g - 1) >> 1) & 1, abort_flag);
                        __syncwarp();
                        tc_fence_after();
#pragma unroll 1
                        for (int i = 0; i < TPT / 8; ++i) {
                            uint32_t orr[32];
                            const uint32_t o_addr = tmem_base + lane_base + (uint32_t)(4 * TPT * w + 32 * i);
                            tmem_ld32(o_addr, orr);
                            tmem_ld_wait();
#pragma unroll
                            for (int c = 0; c < 32; ++c) orr[c] = __float_as_uint(__uint_as_float(orr[c]) * f);
                            tmem_st32(o_addr, orr);
                        }
                        tmem_st_wait();
                    }
                    if (ok) {
                        if (E8) {
                            kappa = m_ref == -INFINITY ? 0.f : fast_exp2(fminf(m_sum - m_ref + kLog2Off, 120.f));
                        } else {
                            const float d = base - (m_ref == -INFINITY ? 0.f : m_ref);
#pragma unroll
                            for (int c = 0; c < TPT; ++c) x[c] += d;
                        }
                    }
                }
                if (ok) probabilities();
                if (E8 && ok) {
                    l_part[0] += tsum;
                    if (j < it.n_tiles - 1) load_sigma(g + 1);
                }
                if (ok) {
                    if (!E8) {
                        // row sums of the rounded values
#pragma unroll
                        for (int c = 0; c < TPT / 2; ++c) {
                            l_part[0] += __uint_as_float(pk[c] << 16);
                            l_part[1] += __uint_as_float(pk[c] & 0xffff0000u);
                        }
                    }
                    // P, once the previous tile's product has read its buffer (the previous item's last: awaited in its epilogue)
                    if (j > 0) mbar_wait(&sh->o_done[(g - 1) & 1], ((g - 1) >> 1) & 1, abort_flag);
                    if (E8) {
                        // row of 128 tokens, one byte each, in all three terms
#pragma unroll
                        for (int c = 0; c < TPT / 16; ++c) {
                            uint8_t* at = sP + row * 128 + (((part * (TPT / 16) + c) ^ (row & 7)) * 16);
                            uint32_t t[3][4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) split4_e5m2(pk[8 * c + 2 * i], pk[8 * c + 2 * i + 1], t[0][i], t[1][i], t[2][i]);
#pragma unroll
                            for (int i = 0; i < 3; ++i) *reinterpret_cast<uint4*>(at + i * SLAB) = make_uint4(t[i][0], t[i][1], t[i][2], t[i][3]);
                        }
                    } else {
                        uint8_t* p_row = sP + half * SLAB + row * 128;
#pragma unroll
                        for (int c = 0; c < TPT / 8; ++c)
                            *reinterpret_cast<uint4*>(p_row + (((4 * w + c) ^ (row & 7)) * 16)) =
                                make_uint4(pk[4 * c], pk[4 * c + 1], pk[4 * c + 2], pk[4 * c + 3]);
                    }
                    if (j >= it.first_special) {
                        // own half of the second operand: drafts cleared of values that are not finite, token rows n_valid ..
                        // next multiple of a group zeroed
                        uint8_t* v_at = sV + (g % VS) * X::V_BYTES;
                        mbar_wait(&sh->v_tail[g % VS], (t_phase >> (g % VS)) & 1, abort_flag);
                        const int t_lo = min(max(it.draft0 - (it.tok_begin + j * TOK), 0), n_valid);
                        const int n_go = (n_valid + X::GROUP - 1) / X::GROUP * X::GROUP - t_lo;
                        constexpr int W = E8 ? 16 : 32;          // 16-byte pieces of a token's 256 dims
                        for (int i = threadIdx.x - 128; i < n_go * W; i += SM) {
                            const int t = t_lo + i / W, sl = (i >> 3) & (W / 8 - 1), c16 = i & 7;
                            uint8_t* at = v_at + (E8 ? 2 * (t >> 6) + sl : 4 * (sl >> 1) + 2 * (t >> 6) + (sl & 1)) * SLAB + (t & 63) * 128 + c16 * 16;
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
                if (j >= it.first_special) t_phase ^= 1u << (g % VS);
                fence_proxy_async();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_cluster(p_bar);
                    if (E8) mbar_arrive(&sh->sc_empty[g & 3]);
                }
            }

            // ---------------- epilogue: row sums, normalised partial, LSE
            softmax_sync<SM>();     // (the last tile may have had a new reference: its maxima are read before the sums take their place)
            sh->red[part][row] = l_part[0] + l_part[1];
            if (E8) sh->red2[E8 ? part : 0][E8 ? row : 0] = m_sum;
            softmax_sync<SM>();
            float l, m = m_ref;
            if (E8) {
                m = -INFINITY;
#pragma unroll
                for (int i = 0; i < PARTS; ++i) m = fmaxf(m, sh->red2[E8 ? i : 0][E8 ? row : 0]);
                l = 0.f;
#pragma unroll
                for (int i = 0; i < PARTS; ++i) {
                    const float mi = sh->red2[E8 ? i : 0][E8 ? row : 0], li = sh->red[i][row];
                    l += mi == -INFINITY ? li : li * fast_exp2(mi - m);
                }
            } else {
                l = 0.f;
#pragma unroll
                for (int i = 0; i < PARTS; ++i) l += sh->red[i][row];
            }
            // l = 0: nothing visible in this chunk.  l = NaN: some logit is not finite, and the row becomes NaN.
            const float inv = l == 0.f ? 0.f : (E8 ? fast_exp2((m_ref - m) - kLog2Off) : 1.f) / l;
            if (part == 0 && mine) {
                const float lse = l == 0.f ? -INFINITY : l == l ? (m + log2f(l)) * kLn2 : kLseNotFinite;
                const int64_t r = row0 + 64 * (int)rank + row;
                if (direct) p.lse_direct[r] = lse;
                else p.lse_part[(int64_t)it.slot * all_rows + r] = lse;
            }
            if (vote_or<SM>(*abort_flag != 0 || !mbar_wait(&sh->o_done[(g - 1) & 1], ((g - 1) >> 1) & 1, abort_flag))) break;
            tc_fence_after();
            // The normalised rows go straight from tensor memory to the workspace, a thread its row's 32-byte sectors: through shared memory
            // and tiled stores the next item's second operand would wait for the space (3500 clocks per item against 1000).  This
            // thread's columns are latent dims 256 half + 128 w + 0 .. 127.
            const int64_t r = row0 + 64 * (int)rank + row;
            const int col0 = 128 * part;
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
                uint32_t orr[32];
                tmem_ld32(tmem_base + lane_base + (uint32_t)(128 * w + 32 * i), orr);
                tmem_ld_wait();
                if (!mine) continue;
                if (direct) {
                    __nv_bfloat16* dst = p.o_lat_direct + r * 512 + col0 + 32 * i;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t v[8];
#pragma unroll
                        for (int f = 0; f < 8; ++f)
                            v[f] = pack_bf16(__uint_as_float(orr[16 * c + 2 * f]) * inv, __uint_as_float(orr[16 * c + 2 * f + 1]) * inv);
                        store_sector(dst + 16 * c, v);
                    }
                } else {
                    float* dst = p.o_part + ((int64_t)it.slot * all_rows + r) * 512 + col0 + 32 * i;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t v[8];
#pragma unroll
                        for (int f = 0; f < 8; ++f) v[f] = __float_as_uint(__uint_as_float(orr[8 * c + f]) * inv);
                        store_sector(dst + 8 * c, v);
                    }
                }
            }
            tc_fence_before();
        }
    } else if (E8 && warp == 3) {
        // ---------------- powers of two of a tile's tokens, 4 per lane
        auto load = [&](const Item& it, int j) {
            const int t0 = it.tok_begin + j * TOK + 4 * lane;
            if (j >= it.n_tiles || t0 >= it.tok_end) return 0x7f7f7f7fu;
            const int page = page_at(it, t0);
            return page >= p.num_pages ? 0x7f7f7f7fu
                                       : *reinterpret_cast<const uint32_t*>(p.exponents + (int64_t)page * p.page_size + t0 % p.page_size);
        };
        int g = 0;
        bool ok = true;
        for (int k = 0; k < n_rounds && ok; ++k) {
            const Item it = item_at(k, desc_of(k));
            uint32_t next = load(it, 0);
            for (int j = 0; j < it.n_tiles; ++j, ++g) {
                const uint32_t bytes = next;
                next = load(it, j + 1);
                if (g >= 4) ok = mbar_wait_warp(&sh->sc_empty[g & 3], ((g >> 2) & 1) ^ 1, abort_flag);
                if (!ok) break;
                float4 v;     // byte 0 (2^-127) is taken as zero; 255: every value NaN, whatever the codes
                float* f = &v.x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t e = (bytes >> (8 * i)) & 0xffu;
                    f[i] = __uint_as_float(e == 255u ? 0x7fc00000u : e << 23);
                }
                *reinterpret_cast<float4*>(&sh->sigma[E8 ? g & 3 : 0][E8 ? 4 * lane : 0]) = v;
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh->sc_full[g & 3]);
            }
        }
    } else if (warp == 1) {
        // (odd CTA) The output projection behind this kernel reads W_UV: every pair requests its share into L2.
        const uint64_t at = ((uint64_t)pair * 32u + (uint32_t)lane) * p.l2_bytes;
        if (at < p.l2_total)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(p.l2_base + at),
                         "r"(min(p.l2_bytes, p.l2_total - (uint32_t)at)) : "memory");
    }

    if (bad_page && p.status) atomicOr(p.status, TYPHOON_MLA_STATUS_BAD_PAGE);
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        // A wait gave up.  Before the shared memory is released the copies in flight are awaited (with a limit): the even CTA's
        // barriers count those of both CTAs, and neither CTA leaves before the other (the cluster barrier below).
        if (rank == 0 && warp == 0 && issued > 0) {
            for (int s = 0; s < KS && s < issued; ++s)      // last tile issued into stage s
                mbar_drain(&sh->k_full[s][0], ((issued - 1 - (issued - 1 - s) % KS) / KS) & 1);
            mbar_drain(&sh->k_full[0][1], (issued - 1) & 1);
            if (issued_n > 0) mbar_drain(&sh->q_full, (issued_n - 1) & 1);
        }
        if (warp == 2)
            for (int i = 0; i < VS; ++i) {
                if (rank == 0 && issued_v[i] > 0)
                    for (int nb = 0; nb < X::NV; ++nb) mbar_drain(&sh->v_full[E8 ? i : nb], (issued_v[i] - 1) & 1);
                if (issued_t[i] > 0) mbar_drain(&sh->v_tail[i], (issued_t[i] - 1) & 1);
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
    if (a.n_sh_chunks > 0 && (e8 || a.sh_chunk % TOK != 0)) return cudaErrorInvalidValue;
    CUtensorMap tm_qa, tm_qp, tm_ckv, tm_kpe, tm_ckv_sh, tm_kpe_sh;
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
    tm_ckv_sh = tm_ckv;
    tm_kpe_sh = tm_kpe;
    if (a.n_sh_chunks > 0) {
        const typhoon_mla_cache_t prefix{const_cast<void*>(a.ckv_shared), const_cast<void*>(a.kpe_shared), nullptr, 512, 64, 64,
                                         (int32_t)(a.Ls_pad / 64)};
        e = make_kv_tmaps(prefix, &tm_ckv_sh, &tm_kpe_sh);
        if (e != cudaSuccess) return e;
    }
    DraftParams p{};
    p.B = a.B; p.S = a.S; p.H = a.H; p.rows = rows;
    p.row_tiles = (rows + 127) / 128; p.chunk = a.chunk; p.n_chunks = a.n_chunks; p.chunk0 = a.chunk0;
    p.page_size = a.cache->page_size; p.max_pages = a.max_pages; p.num_pages = a.cache->num_pages;
    p.block_table = a.block_table; p.seq_lens = a.seq_lens; p.draft_lens = a.draft_lens; p.mask = a.mask;
    p.desc = reinterpret_cast<const int4*>(a.desc);
    p.scale_log2 = a.scale * kLog2e;
    p.o_part = a.o_part; p.lse_part = a.lse_part;
    p.o_lat_direct = static_cast<__nv_bfloat16*>(o_lat_direct); p.lse_direct = lse_direct; p.status = status;
    p.q_tau = a.q_tau; p.exponents = a.cache->ckv_exponents;
    p.Ls = a.Ls; p.sh_chunk = a.sh_chunk; p.n_sh_chunks = a.n_sh_chunks;
    const int64_t sh_items = a.n_sh_chunks * ((all_rows + 127) / 128);
    const int64_t items = sh_items + (int64_t)p.row_tiles * a.n_chunks * a.B;
    if (items > INT32_MAX / 2) return cudaErrorInvalidValue;
    p.n_sh_items = (int)sh_items;
    p.l2_base = static_cast<const char*>(a.w_uv);
    const int pairs = (int)std::min<int64_t>(items, std::max(a.n_sm / 2, 1));
    // (4 KB per lane at most: a few pairs that ask for all of it would wait behind it themselves; 1 request x 128 heads 63 -> 47 us a step)
    p.l2_total = a.w_uv ? (uint32_t)std::min<int64_t>((int64_t)a.H * 128 * 512 * 2, (int64_t)pairs * 32 * 4096) : 0u;
    p.l2_bytes = (p.l2_total / (pairs * 32u) / 16u + 1u) * 16u;
    auto* kernel = e8 ? draft_pair_sm100_kernel<true> : draft_pair_sm100_kernel<false>;
    const dim3 block(e8 ? Shape<true>::THREADS : Shape<false>::THREADS);
    return launch_pdl(kernel, dim3((unsigned)(2 * pairs)), block, kDraftSmem, s, tm_qa, tm_qp, tm_ckv, tm_kpe, tm_ckv_sh, tm_kpe_sh, p);
}

}  // namespace tmla
