// What the kernels have in common that multiply 4-bit words of the cache with m16n8k16 products: the products, codes as f16 operands,
// copies to shared memory and the rows of q that a lane takes.
#pragma once
#include "kv_attention.cuh"

namespace lce {

// d = A B + c
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, float c0, float c1,
                                    float c2, float c3)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    mma(d, a0, a1, a2, a3, b0, b1, d[0], d[1], d[2], d[3]);
}
// A pair of codes on the mantissa of 1024, 1024 + 4 n or 1024 + 64 n, as f16 numbers c = n - 8.
__device__ __forceinline__ uint32_t half_fma(uint32_t w, unsigned short by, unsigned short plus)
{
    const __half2 v = __hfma2(*reinterpret_cast<const __half2 *>(&w), __half2half2(__ushort_as_half(by)), __half2half2(__ushort_as_half(plus)));
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t signed_even(uint32_t w) { return half_fma(w, 0x3400, 0xdc20); }  // / 4 - 264
__device__ __forceinline__ uint32_t signed_odd(uint32_t w) { return half_fma(w, 0x2400, 0xce00); }   // / 64 - 24

// W words of a lane from shared memory.
template <int W>
__device__ __forceinline__ void load_words(const uint32_t *p, uint32_t (&w)[W])
{
    if (W == 4) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        w[0] = v.x; w[W > 1 ? 1 : 0] = v.y; w[W > 2 ? 2 : 0] = v.z; w[W > 3 ? 3 : 0] = v.w;
    } else if (W == 2) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        w[0] = v.x; w[W > 1 ? 1 : 0] = v.y;
    } else {
        w[0] = *p;
    }
}

__device__ __forceinline__ void cp_async16(uint32_t smem, const void *g)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(g) : "memory");
}

// The lane's channels of its columns as they come from memory.
template <int B, int NT, typename T>
struct Queries {
    Eight<T> e[NT][B];
    template <bool VEC>
    __device__ __forceinline__ void load(const AttnParams &p, const Unit &u, int head)
    {
        const int lane = threadIdx.x & 31, n = lane >> 2, quarter = lane & 3;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int column = u.column0 + 8 * nt + n, row = column / p.group;
            const int64_t at = (u.row0 + row) * p.q_token + ((int64_t)head * p.group + (column - row * p.group)) * p.q_head + 8 * quarter;
#pragma unroll
            for (int b = 0; b < B; ++b) e[nt][b] = load_eight<T, VEC>(static_cast<const T *>(p.q) + at + 32 * b, row < u.rows ? p.g.dim - 32 * b - 8 * quarter : 0);
        }
    }
};

}  // namespace lce
