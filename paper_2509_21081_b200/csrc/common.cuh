// Small device helpers shared by the kernels of this library (sm_100a).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace tmla {

constexpr int kDn = 128;   // D_n  nope head dim
constexpr int kDr = 64;    // D_r  rope head dim
constexpr int kDv = 128;   // D_v  value head dim
constexpr int kDl = 512;   // D_l  latent width
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// LSE by which a partial of drafted tokens says that some logit of the row is not finite: its weight in any merge is 1 and its values
// are NaN, so the row becomes NaN.
constexpr float kLseNotFinite = 3.2e38f;
// (a kernel's own LSE of such a row may also be a NaN: the merges take it as this)
__device__ __forceinline__ float partial_lse(float l) { return l == l ? l : kLseNotFinite; }
// LSE of a row from the largest of its partials' and the sum of their weights (m > -inf).
__device__ __forceinline__ float merged_lse(float m, float z) { return m < kLseNotFinite ? m + __logf(z) : __int_as_float(0x7fc00000); }

__device__ __forceinline__ uint32_t smem_u32(const void* p) {
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

// 16-byte asynchronous copy global -> shared; pred == false writes zeros.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool pred) {
    int sz = pred ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(sz) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory");
}

__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}

// D(16x8, fp32) += A(16x16, bf16, row) * B(16x8, bf16, col)
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ float bf16_round(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }

__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}

// Block-wide sort used for the longest-first launch order of ragged suffixes: perm[] = request
// indices by descending length, ties by ascending index.  `keys` is shared memory for the next
// power of two >= B (<= 4096) 64-bit keys.  Called by every thread of the block.
__device__ __forceinline__ void block_order_by_length(const int32_t* __restrict__ seq_lens, int B,
                                                      int32_t* __restrict__ perm, unsigned long long* keys) {
    const int nt = blockDim.x, tid = threadIdx.x;
    int n = 1;
    while (n < B) n <<= 1;
    for (int i = tid; i < n; i += nt) {
        unsigned long long k = ~0ull;   // padding sorts last
        if (i < B) k = ((unsigned long long)(0x7fffffffu - (unsigned)max(seq_lens[i], 0)) << 32) | (unsigned)i;
        keys[i] = k;
    }
    __syncthreads();
    for (int size = 2; size <= n; size <<= 1) {
        for (int stride = size >> 1; stride > 0; stride >>= 1) {
            for (int i = tid; i < n / 2; i += nt) {
                const int lo = (i / stride) * 2 * stride + (i % stride), hi = lo + stride;
                const bool up = ((lo & size) == 0);
                const unsigned long long a = keys[lo], b = keys[hi];
                if ((a > b) == up) { keys[lo] = b; keys[hi] = a; }
            }
            __syncthreads();
        }
    }
    for (int i = tid; i < B; i += nt) perm[i] = (int32_t)(keys[i] & 0xffffffffu);
}

}  // namespace tmla
