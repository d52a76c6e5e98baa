// Rotary positions of query rows, writing tokens into the paged latent cache (16-bit, or 8-bit codes) and reading them back.
//
// All three move bytes and are bound by them: one pass, 16-byte accesses, nothing in between.
//
// Angles.  pos * f radians in 32 bits is wrong by 0.06 at position 10^6, so the tables hold every frequency as turns per position in
// units of 2^-64 of a turn: the 64-bit product with the integer position, modulo 2^64, is the fraction of a turn to 2^-64 * pos, its top
// 32 bits are the angle within +-pi.  No 64-bit floating point, no argument reduction.
#include <algorithm>
#include <cmath>

#include "../../include/typhoon_mla.h"
#include "kernels.h"
#include "sm100.cuh"

namespace tmla {
namespace {

using sm100::pdl_trigger;
using sm100::pdl_wait;

__device__ __forceinline__ float2 cos_sin_of(uint64_t turns, int pos, float scale) {
    const uint64_t frac = turns * (uint64_t)(int64_t)pos;
    // 2^32 of the top word is one turn; within +-pi the fast sine and cosine are off by at most 2^-21.2, far below bf16's 2^-9 (the
    // accurate pair costs 40 instructions more for each of a token's 32 pairs: 10 % of the time of an 8-bit append)
    float s, c;
    __sincosf((float)(int32_t)(frac >> 32) * (3.14159265358979f * 0x1p-31f), &s, &c);
    return make_float2(c * scale, s * scale);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// Products of this file's 8-bit path keep subnormal numbers (the library is compiled with flush-to-zero arithmetic).
__device__ __forceinline__ float mul_keep(float a, float b) {
    float d;
    asm("mul.rn.f32 %0, %1, %2;\n" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// ---------------------------------------------------------------- rotary positions of query rows
// Rows are (token, head) pairs in order.  A block takes ROWS of them: 8 threads carry a row's 64 rope dims, 16 bytes each, 16 threads
// its 128 other dims, and all of a thread's loads (12 with 128 rows) go out before anything waits.  Meanwhile the cosines and sines of
// the tokens among the rows go to shared memory once: a row of 128 heads shares its token's 32 pairs; computed per row they would
// take as long as the copy.  With the half layout the other element of a pair is in another thread of the row: a shuffle.  Every row
// is read by the block that writes it, before it writes, so rows may be rotated in place.
// (B200, 4759 tokens x 128 heads, 468 MB in and out: 71 us, the rate of a plain copy; 64 tokens 3.1 us.)
constexpr int kRopeThreads = 256;
struct RopeQParams {
    const __nv_bfloat16* nope; int64_t nope_t, nope_h;
    const __nv_bfloat16* pe; int64_t pe_t, pe_h;
    const int32_t* positions;
    __nv_bfloat16 *nope_out, *pe_out;
    int64_t n_rows;
    int H;
    typhoon_mla_rope_t rope;
};

template <bool HALF, int ROWS>
__global__ void __launch_bounds__(kRopeThreads) rope_queries_kernel(const __grid_constant__ RopeQParams p) {
    extern __shared__ float4 cs4[];   // [tokens of this block][pairs] of (cos, sin)
    float2* cs = reinterpret_cast<float2*>(cs4);
    constexpr int NP = ROWS / 32, NN = ROWS / 16;
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x, pairs = p.rope.d_rot / 2;
    const int64_t r0 = (int64_t)blockIdx.x * ROWS;
    const int n = (int)min((int64_t)ROWS, p.n_rows - r0);
    const int64_t t0 = r0 / p.H;
    const int h0 = (int)(r0 - t0 * p.H);
    uint4 pe[NP], no[NN];
    int tok[NP];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        const int r = min((tid >> 3) + 32 * k, n - 1);   // (whole warps take part in the shuffles)
        tok[k] = (h0 + r) / p.H;
        pe[k] = *reinterpret_cast<const uint4*>(p.pe + (t0 + tok[k]) * p.pe_t + (h0 + r - tok[k] * p.H) * p.pe_h + (tid & 7) * 8);
    }
    if (p.nope_out != nullptr) {
#pragma unroll
        for (int k = 0; k < NN; ++k) {
            const int r = min((tid >> 4) + 16 * k, n - 1), t = (h0 + r) / p.H;
            no[k] = *reinterpret_cast<const uint4*>(p.nope + (t0 + t) * p.nope_t + (h0 + r - t * p.H) * p.nope_h + (tid & 15) * 8);
        }
    }
    const int n_tok = (h0 + n - 1) / p.H + 1;
    for (int i = tid; i < n_tok * pairs; i += kRopeThreads) {
        const int t = i / pairs, k = i - t * pairs;
        cs[i] = cos_sin_of(p.rope.turns[k], p.positions[t0 + t], p.rope.scale);
    }
    __syncthreads();
    const int c = tid & 7;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        const uint32_t a[4] = {pe[k].x, pe[k].y, pe[k].z, pe[k].w};
        uint32_t o[4] = {a[0], a[1], a[2], a[3]};
        const float2* ct = cs + tok[k] * pairs;
        if (HALF) {
            const int step = pairs >> 3;          // 16-byte pieces between the two elements of a pair
            const bool turned = c < 2 * step, second = c >= step;
            const int lane = tid & 31, from = turned ? (second ? lane - step : lane + step) : lane;
            uint32_t b[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) b[e] = __shfl_sync(0xffffffffu, a[e], from);
            if (turned) {
                const float2* cc = ct + (second ? c - step : c) * 8;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float4 f = *reinterpret_cast<const float4*>(cc + 2 * e);    // cos, sin, cos, sin
                    const float s0 = second ? f.y : -f.y, s1 = second ? f.w : -f.w;
                    o[e] = pack_bf16(bf16_lo(a[e]) * f.x + bf16_lo(b[e]) * s0, bf16_hi(a[e]) * f.z + bf16_hi(b[e]) * s1);
                }
            }
        } else if (c * 4 < pairs) {
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const float4 f = *reinterpret_cast<const float4*>(ct + c * 4 + e);
                const float x0 = bf16_lo(a[e]), x1 = bf16_hi(a[e]), x2 = bf16_lo(a[e + 1]), x3 = bf16_hi(a[e + 1]);
                o[e] = pack_bf16(x0 * f.x - x1 * f.y, x0 * f.y + x1 * f.x);
                o[e + 1] = pack_bf16(x2 * f.z - x3 * f.w, x2 * f.w + x3 * f.z);
            }
        }
        const int r = (tid >> 3) + 32 * k;
        if (r < n) *reinterpret_cast<uint4*>(p.pe_out + (r0 + r) * 64 + c * 8) = make_uint4(o[0], o[1], o[2], o[3]);
    }
    if (p.nope_out != nullptr) {
#pragma unroll
        for (int k = 0; k < NN; ++k) {
            const int r = (tid >> 4) + 16 * k;
            if (r < n) *reinterpret_cast<uint4*>(p.nope_out + (r0 + r) * 128 + (tid & 15) * 8) = no[k];
        }
    }
}

// ---------------------------------------------------------------- the paged cache
struct CacheView {
    uint8_t* ckv; int64_t ckv_stride;     // bytes per token
    uint8_t* kpe; int64_t kpe_stride;     // bytes per token
    uint8_t* exponents;                   // null: 16-bit latent rows
    int64_t n_slots;
    int* status;
};
CacheView view_of(const typhoon_mla_cache_t& c, int* status) {
    const int64_t width = c.ckv_exponents ? 1 : 2;
    return CacheView{static_cast<uint8_t*>(c.ckv_pages), c.ckv_token_stride * width, static_cast<uint8_t*>(c.kpe_pages), c.kpe_token_stride * 2,
                     c.ckv_exponents, (int64_t)c.num_pages * c.page_size, status};
}

// A warp takes a token at a time: 1 KB of latent values in two 16-byte loads per lane, the rope key one pair per lane.  With more
// tokens than resident warps a warp goes on to further ones and requests the next before it works on the one it has: one token per
// warp and a block per 8 tokens left the memory idle while warps started and ended.
// (B200, 70001 tokens into an 8-bit cache, 126 MB: one token per warp 29.6 us, this 26.9, with the fast sine and no clamp before
// the conversions (the instructions counted for as much as the bytes) 22.0; 16-bit, 162 MB: 29.5.)
constexpr int kCacheWarps = 8, kCacheBlocksPerSm = 5, kCacheSms = 148;
int cache_blocks(int64_t T) { return (int)std::min<int64_t>((T + kCacheWarps - 1) / kCacheWarps, kCacheSms * kCacheBlocksPerSm); }

__global__ void __launch_bounds__(32 * kCacheWarps, kCacheBlocksPerSm)
cache_append_kernel(const __nv_bfloat16* __restrict__ ckv, int64_t ld_ckv, const __nv_bfloat16* __restrict__ kpe, int64_t ld_kpe,
                    const int32_t* __restrict__ positions, const int64_t* __restrict__ slots, int64_t T, CacheView c,
                    const __grid_constant__ typhoon_mla_rope_t rope) {
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int64_t step = (int64_t)gridDim.x * kCacheWarps;
    // pair of this lane: the rotated pairs first, then the dims that are copied, two at a time
    const int pairs = rope.d_rot / 2;
    const bool half = rope.layout == TYPHOON_MLA_ROPE_HALF && lane < pairs;
    const bool turned = positions != nullptr && lane < pairs;
    const int i0 = half ? lane : 2 * lane, i1 = half ? lane + pairs : 2 * lane + 1;
    const uint64_t turns = turned ? rope.turns[lane] : 0;
    struct Token {
        uint4 v[2];
        uint32_t key;     // both elements of the pair
        int pos;
        int64_t slot;
    };
    auto load = [&](int64_t t) {
        Token x;
        x.slot = slots[t];
        const uint4* src = reinterpret_cast<const uint4*>(ckv + t * ld_ckv) + 2 * lane;
        x.v[0] = src[0];
        x.v[1] = src[1];
        const uint16_t* kr = reinterpret_cast<const uint16_t*>(kpe + t * ld_kpe);
        x.key = half ? (uint32_t)kr[i0] | ((uint32_t)kr[i1] << 16) : *reinterpret_cast<const uint32_t*>(kr + i0);
        x.pos = turned ? positions[t] : 0;
        return x;
    };
    auto write = [&](const Token& x) {
        if (x.slot < 0) return;                       // a padding token
        if (x.slot >= c.n_slots) {                    // never dereferenced
            if (lane == 0 && c.status) atomicOr(c.status, TYPHOON_MLA_STATUS_BAD_PAGE);
            return;
        }
        uint8_t* dst = c.ckv + x.slot * c.ckv_stride;
        if (c.exponents == nullptr) {
            reinterpret_cast<uint4*>(dst)[2 * lane] = x.v[0];
            reinterpret_cast<uint4*>(dst)[2 * lane + 1] = x.v[1];
        } else {
            // largest magnitude of the row, as 16-bit patterns (ordered like the magnitudes; >= 0x7f80: not finite)
            const uint32_t w[8] = {x.v[0].x, x.v[0].y, x.v[0].z, x.v[0].w, x.v[1].x, x.v[1].y, x.v[1].z, x.v[1].w};
            uint32_t m2 = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m2 = __vmaxu2(m2, w[i] & 0x7fff7fffu);
            const uint32_t m = __reduce_max_sync(0xffffffffu, max(m2 & 0xffffu, m2 >> 16));
            // Smallest power of two under which the row fits E4M3's +-448 = 1.75 * 2^8: with m = 1.f * 2^x it is 2^(x - 8), or
            // 2^(x - 7) for 1.f above 1.75 (7 bits: 0x60).  Exponents below 2^-126 are taken as that; a row that is not finite
            // has no codes: exponent byte 255, which reads back as NaN.  (A magnitude above 1.875 * 2^127 would round to 2^128,
            // which bf16 does not hold: it takes the code below, 240 * 2^120.)
            const bool finite = m < 0x7f80u;
            const int byte = finite ? max(1, (int)(m >> 7) - 8 + ((m & 0x7fu) > 0x60u ? 1 : 0)) : 255;
            const float inv = __uint_as_float((uint32_t)(254 - min(byte, 253)) << 23);
            auto scaled = [&](float y) { return mul_keep(y, inv); };
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint16_t lo, hi;
                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(lo) : "f"(scaled(bf16_hi(w[2 * i]))), "f"(scaled(bf16_lo(w[2 * i]))));
                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n"
                    : "=h"(hi) : "f"(scaled(bf16_hi(w[2 * i + 1]))), "f"(scaled(bf16_lo(w[2 * i + 1]))));
                o[i] = finite ? (uint32_t)lo | ((uint32_t)hi << 16) : 0u;
            }
            if (byte == 247) {       // (code magnitude 0x78 stands for 256, 0x77 for 240; per byte)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = (o[i] & 0x80808080u) | __vminu4(o[i] & 0x7f7f7f7fu, 0x77777777u);
            }
            reinterpret_cast<uint4*>(dst)[lane] = make_uint4(o[0], o[1], o[2], o[3]);
            if (lane == 0) c.exponents[x.slot] = (uint8_t)byte;
        }
        uint16_t* kd = reinterpret_cast<uint16_t*>(c.kpe + x.slot * c.kpe_stride);
        uint32_t key = x.key;
        if (turned) {
            const float2 f = cos_sin_of(turns, x.pos, rope.scale);
            const float x0 = bf16_lo(key), x1 = bf16_hi(key);
            key = pack_bf16(x0 * f.x - x1 * f.y, x0 * f.y + x1 * f.x);
        }
        if (half) {
            kd[i0] = (uint16_t)key;
            kd[i1] = (uint16_t)(key >> 16);
        } else {
            *reinterpret_cast<uint32_t*>(kd + i0) = key;
        }
    };
    int64_t t = (int64_t)blockIdx.x * kCacheWarps + (threadIdx.x >> 5);
    if (t >= T) return;
    Token cur = load(t);
    while (true) {
        const int64_t next = t + step;
        if (next >= T) break;
        const Token ahead = load(next);
        write(cur);
        cur = ahead;
        t = next;
    }
    write(cur);
}

// One token per warp: its rows wait for the slot, and 64 warps per SM hide that better than 40 that look ahead.  (B200, 16384 tokens of
// an 8-bit cache 5.5 us, looking ahead 6.6; 70001 tokens 22.2.)
__global__ void __launch_bounds__(32 * kCacheWarps)
cache_read_kernel(CacheView c, const int64_t* __restrict__ slots, int64_t T, __nv_bfloat16* __restrict__ ckv_out, int64_t ld_ckv,
                  __nv_bfloat16* __restrict__ kpe_out, int64_t ld_kpe) {
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    struct Token {
        uint4 v[2];      // 16-bit values, or (in v[0]) codes
        uint32_t key, byte;
    };
    auto load = [&](int64_t slot) {
        Token x{{zero, zero}, 0, 127};
        if (slot >= c.n_slots && lane == 0 && c.status) atomicOr(c.status, TYPHOON_MLA_STATUS_BAD_PAGE);
        if (slot < 0 || slot >= c.n_slots) return x;
        const uint4* src = reinterpret_cast<const uint4*>(c.ckv + slot * c.ckv_stride);
        x.key = reinterpret_cast<const uint32_t*>(c.kpe + slot * c.kpe_stride)[lane];
        if (c.exponents == nullptr) {
            x.v[0] = src[2 * lane];
            x.v[1] = src[2 * lane + 1];
        } else {
            x.v[0] = src[lane];
            x.byte = c.exponents[slot];
        }
        return x;
    };
    auto write = [&](int64_t t, const Token& x) {
        uint4* dst = reinterpret_cast<uint4*>(ckv_out + t * ld_ckv);
        reinterpret_cast<uint32_t*>(kpe_out + t * ld_kpe)[lane] = x.key;
        if (c.exponents == nullptr) {
            dst[2 * lane] = x.v[0];
            dst[2 * lane + 1] = x.v[1];
            return;
        }
        const float scale = x.byte == 255u ? __uint_as_float(0x7fc00000u) : x.byte == 0u ? 0x1p-127f : __uint_as_float(x.byte << 23);
        const uint32_t w[4] = {x.v[0].x, x.v[0].y, x.v[0].z, x.v[0].w};
        uint32_t o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t h2;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(h2) : "h"((uint16_t)(w[i >> 1] >> (16 * (i & 1)))));
            const float2 f = __half22float2(*reinterpret_cast<__half2*>(&h2));
            o[i] = pack_bf16(mul_keep(f.x, scale), mul_keep(f.y, scale));   // 4 significant bits: exact (down to 2^-133)
        }
        dst[2 * lane] = make_uint4(o[0], o[1], o[2], o[3]);
        dst[2 * lane + 1] = make_uint4(o[4], o[5], o[6], o[7]);
    };
    const int64_t t = (int64_t)blockIdx.x * kCacheWarps + (threadIdx.x >> 5);
    if (t < T) write(t, load(slots[t]));
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

bool rope_valid(const typhoon_mla_rope_t* r) {
    return r && r->d_rot >= 16 && r->d_rot <= 64 && r->d_rot % 16 == 0 && r->layout >= TYPHOON_MLA_ROPE_INTERLEAVED &&
           r->layout <= TYPHOON_MLA_ROPE_HALF && std::isfinite(r->scale);
}

}  // namespace

bool cache_valid(const typhoon_mla_cache_t* c) {
    if (!c || !c->ckv_pages || !c->kpe_pages || (c->page_size != 64 && c->page_size != 128) || c->num_pages < 1) return false;
    const int64_t unit = c->ckv_exponents ? 16 : 8;   // 16 bytes
    return aligned(c->ckv_pages, 16) && aligned(c->kpe_pages, 16) && (c->ckv_exponents == nullptr || aligned(c->ckv_exponents, 16)) &&
           c->ckv_token_stride >= 512 && c->ckv_token_stride % unit == 0 && c->kpe_token_stride >= 64 && c->kpe_token_stride % 8 == 0;
}

}  // namespace tmla

using namespace tmla;

extern "C" {

int typhoon_mla_rope_init(typhoon_mla_rope_t* rope, int32_t d_rot, int32_t layout, double base, int32_t scaling, double factor,
                          double original_length, double beta_fast, double beta_slow, double scale) {
    if (!rope || d_rot < 16 || d_rot > 64 || d_rot % 16) return TYPHOON_MLA_ERR_INVALID_ARG;
    if (layout != TYPHOON_MLA_ROPE_INTERLEAVED && layout != TYPHOON_MLA_ROPE_HALF) return TYPHOON_MLA_ERR_INVALID_ARG;
    if (scaling < TYPHOON_MLA_ROPE_SCALE_NONE || scaling > TYPHOON_MLA_ROPE_SCALE_YARN) return TYPHOON_MLA_ERR_INVALID_ARG;
    if (!(base > 1.0) || !std::isfinite(base) || !std::isfinite((float)scale)) return TYPHOON_MLA_ERR_INVALID_ARG;
    if (scaling != TYPHOON_MLA_ROPE_SCALE_NONE && (!(factor >= 1.0) || !std::isfinite(factor))) return TYPHOON_MLA_ERR_INVALID_ARG;
    const double pi = 3.14159265358979323846, d = d_rot;
    double low = 0.0, high = 0.0;
    if (scaling == TYPHOON_MLA_ROPE_SCALE_YARN) {
        if (!(original_length >= 1.0) || !std::isfinite(original_length) || !(beta_slow > 0.0) || !(beta_fast >= beta_slow) ||
            !std::isfinite(beta_fast))
            return TYPHOON_MLA_ERR_INVALID_ARG;
        // pair whose angle turns `beta` times over the original length
        auto pair_of = [&](double beta) { return d * std::log(original_length / (beta * 2.0 * pi)) / (2.0 * std::log(base)); };
        low = std::max(std::floor(pair_of(beta_fast)), 0.0);
        high = std::min(std::ceil(pair_of(beta_slow)), d - 1.0);
    }
    if (scaling == TYPHOON_MLA_ROPE_SCALE_NTK) base *= std::pow(factor, d / (d - 2.0));
    if (!std::isfinite(base)) return TYPHOON_MLA_ERR_INVALID_ARG;
    typhoon_mla_rope_t r{};
    r.d_rot = d_rot;
    r.layout = layout;
    r.scale = (float)scale;
    for (int i = 0; i < d_rot / 2; ++i) {
        double f = std::pow(base, -2.0 * i / d);
        if (scaling == TYPHOON_MLA_ROPE_SCALE_LINEAR) f /= factor;
        if (scaling == TYPHOON_MLA_ROPE_SCALE_YARN) {
            const double ramp = std::min(std::max((i - low) / std::max(high - low, 0.001), 0.0), 1.0);
            f = f / factor * ramp + f * (1.0 - ramp);
        }
        // radians per position (at most 1) -> turns, in units of 2^-64
        r.turns[i] = (uint64_t)(std::ldexp((long double)f / (2.0L * 3.14159265358979323846264338327950288L), 64));
    }
    *rope = r;
    return TYPHOON_MLA_OK;
}

int typhoon_mla_rope_queries(const typhoon_mla_rope_t* rope, const void* q_nope, int64_t nope_token_stride, int64_t nope_head_stride,
                             const void* q_pe, int64_t pe_token_stride, int64_t pe_head_stride, const int32_t* positions, int64_t T,
                             int32_t H, void* q_nope_out, void* q_pe_out, void* stream) {
    api_set_last_launches(0);
    if (!rope_valid(rope) || T < 0 || H < 1 || H > 65536) return TYPHOON_MLA_ERR_INVALID_ARG;
    if ((q_nope == nullptr) != (q_nope_out == nullptr)) return TYPHOON_MLA_ERR_INVALID_ARG;
    if (T == 0) return TYPHOON_MLA_OK;
    if (!q_pe || !q_pe_out || !positions || T > (int64_t)1 << 40) return TYPHOON_MLA_ERR_INVALID_ARG;
    if (!aligned(q_pe, 16) || !aligned(q_pe_out, 16) || !aligned(q_nope, 16) || !aligned(q_nope_out, 16) || !aligned(positions, 4))
        return TYPHOON_MLA_ERR_INVALID_ARG;
    if (pe_token_stride % 8 || pe_head_stride % 8 || (q_nope && (nope_token_stride % 8 || nope_head_stride % 8))) return TYPHOON_MLA_ERR_INVALID_ARG;
    const int64_t n_rows = T * H;
    // 128 rows per block carry 12 16-byte pieces per thread; below four blocks per SM 32 rows spread a small call over the GPU
    const int rows = n_rows >= (int64_t)128 * 4 * 148 ? 128 : 32;
    const int64_t blocks = (n_rows + rows - 1) / rows;
    if (blocks > INT32_MAX) return TYPHOON_MLA_ERR_INVALID_ARG;
    const RopeQParams p{static_cast<const __nv_bfloat16*>(q_nope), nope_token_stride, nope_head_stride, static_cast<const __nv_bfloat16*>(q_pe),
                        pe_token_stride, pe_head_stride, positions, static_cast<__nv_bfloat16*>(q_nope_out),
                        static_cast<__nv_bfloat16*>(q_pe_out), n_rows, H, *rope};
    const int tokens = (rows + H - 2) / H + 1;   // at most, of one block
    const size_t smem = (size_t)tokens * (rope->d_rot / 2) * sizeof(float2);
    api_adopt_settings();
    const bool half = rope->layout == TYPHOON_MLA_ROPE_HALF;
    auto* kernel = rows == 128 ? (half ? rope_queries_kernel<true, 128> : rope_queries_kernel<false, 128>)
                               : (half ? rope_queries_kernel<true, 32> : rope_queries_kernel<false, 32>);
    const cudaError_t e = launch_pdl(kernel, dim3((unsigned)blocks), dim3(kRopeThreads), smem, static_cast<cudaStream_t>(stream), p);
    if (e != cudaSuccess) return api_cuda_fail(e);
    api_set_last_launches(1);
    return TYPHOON_MLA_OK;
}

int typhoon_mla_cache_append(const typhoon_mla_cache_t* cache, const void* ckv, int64_t ld_ckv, const void* kpe, int64_t ld_kpe,
                             const typhoon_mla_rope_t* rope, const int32_t* positions, const int64_t* slots, int64_t T, int32_t* status,
                             void* stream) {
    api_set_last_launches(0);
    if (!cache_valid(cache) || T < 0 || (rope && !rope_valid(rope))) return TYPHOON_MLA_ERR_INVALID_ARG;
    if (T == 0) return TYPHOON_MLA_OK;      // (no tokens: an empty array of positions may have no address)
    if ((rope == nullptr) != (positions == nullptr)) return TYPHOON_MLA_ERR_INVALID_ARG;
    if (!ckv || !kpe || !slots || !aligned(ckv, 16) || !aligned(kpe, 16) || !aligned(positions, 4) || !aligned(slots, 8) || !aligned(status, 4))
        return TYPHOON_MLA_ERR_INVALID_ARG;
    if (ld_ckv < 512 || ld_ckv % 8 || ld_kpe < 64 || ld_kpe % 8) return TYPHOON_MLA_ERR_INVALID_ARG;
    api_adopt_settings();
    const typhoon_mla_rope_t none{};
    const cudaError_t e = launch_pdl(cache_append_kernel, dim3(cache_blocks(T)), dim3(32 * kCacheWarps), 0,
                                     static_cast<cudaStream_t>(stream), static_cast<const __nv_bfloat16*>(ckv), ld_ckv,
                                     static_cast<const __nv_bfloat16*>(kpe), ld_kpe, positions, slots, T, view_of(*cache, status),
                                     rope ? *rope : none);
    if (e != cudaSuccess) return api_cuda_fail(e);
    api_set_last_launches(1);
    return TYPHOON_MLA_OK;
}

int typhoon_mla_cache_read(const typhoon_mla_cache_t* cache, const int64_t* slots, int64_t T, void* ckv_out, int64_t ld_ckv, void* kpe_out,
                           int64_t ld_kpe, int32_t* status, void* stream) {
    api_set_last_launches(0);
    if (!cache_valid(cache) || T < 0) return TYPHOON_MLA_ERR_INVALID_ARG;
    if (T == 0) return TYPHOON_MLA_OK;
    if (!slots || !ckv_out || !kpe_out || !aligned(ckv_out, 16) || !aligned(kpe_out, 16) || !aligned(slots, 8) || !aligned(status, 4))
        return TYPHOON_MLA_ERR_INVALID_ARG;
    if (ld_ckv < 512 || ld_ckv % 8 || ld_kpe < 64 || ld_kpe % 8 || T > (int64_t)INT32_MAX * kCacheWarps) return TYPHOON_MLA_ERR_INVALID_ARG;
    api_adopt_settings();
    const cudaError_t e = launch_pdl(cache_read_kernel, dim3((unsigned)((T + kCacheWarps - 1) / kCacheWarps)), dim3(32 * kCacheWarps), 0,
                                     static_cast<cudaStream_t>(stream), view_of(*cache, status), slots, T, static_cast<__nv_bfloat16*>(ckv_out),
                                     ld_ckv, static_cast<__nv_bfloat16*>(kpe_out), ld_kpe);
    if (e != cudaSuccess) return api_cuda_fail(e);
    api_set_last_launches(1);
    return TYPHOON_MLA_OK;
}

}  // extern "C"
