// The 4-bit key/value cache: its layout, the element types of its callers and the quantiser's arithmetic.
//
// A tile is 16 tokens of one head: with B = ceil(head_dim / 32) blocks, uint32 K[64 B], V[64 B], scales[16 B].  Its blocks come
// in planes of 4, then 2, then 1 (6 = 4 + 2), W blocks each, so that a lane's words of a plane are one vector load:
//   K       word (half h, lane l, block w) at (32 h + l) W + w: the 8 codes of token 8 h + l / 4, channels 8 (l % 4) .. + 7 of
//           block w, lowest channel in the lowest nibble;
//   V       word (h, l, w), same place: tokens 8 h + 2 (l % 4) in the low and the one behind it in the high half, channels
//           4 (l / 4) .. + 3 of block w;
//   scales  word (token, w) at W token + w: bf16 of the key in the low, of the value in the high half.
// Lane l of a warp finds there exactly its part of the A operands of m16n8k16 products, 16 tokens x channels for the keys
// and channels x 16 tokens for the values: no transposition, and shared memory is read lane by lane without bank conflicts.
// Codes are stored as n = c + 8, in either half of a word rotated left by two bits: bits 2 .. 5 and 6 .. 9 of a half, and of one with
// its bytes exchanged, are then codes as high in the ten mantissa bits of an f16 number as two of them can stand.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"

namespace lce {

constexpr int kKvTile = 16;     // tokens of a tile
constexpr int kKvMaxDim = 256;

__host__ __device__ __forceinline__ constexpr int kv_tile_words(int blocks) { return 144 * blocks; }

struct KvGeom {
    int32_t pages, page_size, heads, dim, blocks;
    int32_t slots;
};

inline lce_status make_kv_geom(const lce_kv_desc *d, KvGeom *g)
{
    if (!d || d->pages <= 0 || d->page_size <= 0 || d->kv_heads <= 0 || d->head_dim <= 0) return LCE_ERR_INVALID_ARG;
    if (d->page_size % kKvTile != 0) return LCE_ERR_INVALID_ARG;
    if (d->head_dim > kKvMaxDim || d->kv_heads > 65535 || (int64_t)d->pages * d->page_size >= (1ll << 31)) return LCE_ERR_UNSUPPORTED;
    g->pages = d->pages; g->page_size = d->page_size; g->heads = d->kv_heads; g->dim = d->head_dim;
    g->blocks = (d->head_dim + 31) / 32;
    g->slots = d->pages * d->page_size;
    return LCE_OK;
}

inline bool type_known(int32_t t) { return t >= LCE_TYPE_FLOAT32 && t <= LCE_TYPE_BFLOAT16; }
inline size_t type_size(int32_t t) { return t == LCE_TYPE_FLOAT32 ? 4 : 2; }

// Where block `b` lies in a tile of `blocks`: its plane's first block and width.
__host__ __device__ __forceinline__ void kv_plane(int blocks, int b, int *first, int *width)
{
    const int quads = blocks & ~3;
    if (b < quads) { *first = b & ~3; *width = 4; }
    else if ((blocks & 2) && b < quads + 2) { *first = quads; *width = 2; }
    else { *first = blocks - 1; *width = 1; }
}
// Words of a tile: the keys' of (token, block, quarter of its channels), the values' of (token pair, block, eighth), the scales'.
__host__ __device__ __forceinline__ int kv_key_word(int blocks, int token, int b, int quarter)
{
    int first, width;
    kv_plane(blocks, b, &first, &width);
    return 64 * first + ((token >> 3) * 32 + (token & 7) * 4 + quarter) * width + (b - first);
}
__host__ __device__ __forceinline__ int kv_value_word(int blocks, int pair, int b, int eighth)
{
    int first, width;
    kv_plane(blocks, b, &first, &width);
    return 64 * blocks + 64 * first + ((pair >> 2) * 32 + eighth * 4 + (pair & 3)) * width + (b - first);
}
__host__ __device__ __forceinline__ int kv_scale_word(int blocks, int token, int b)
{
    int first, width;
    kv_plane(blocks, b, &first, &width);
    return 128 * blocks + 16 * first + token * width + (b - first);
}

// --- elements of the callers' tensors ---------------------------------------------------------------

template <typename T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Eight consecutive elements as they come from memory, in one access where VEC (the address is then a multiple of their size, 16 or 32
// bytes, and either all eight exist or none; fp32 in two accesses of 16 bytes asks for every sector twice); `count` of them exist, zeros
// stand for the others.  Nothing is done to them here, so that many loads can be on their way at once.
template <typename T>
struct alignas(8 * sizeof(T)) Eight {
    T e[8];
    __device__ __forceinline__ void expand(float (&v)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_float(e[i]);
    }
};
template <typename T, bool VEC>
__device__ __forceinline__ Eight<T> load_eight(const T *p, int count)
{
    Eight<T> r;
    if (VEC && sizeof(T) == 4) {
        uint32_t q[8] = {};
        if (count > 0)
            asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                         : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]), "=r"(q[4]), "=r"(q[5]), "=r"(q[6]), "=r"(q[7])
                         : "l"(p)
                         : "memory");
#pragma unroll
        for (int i = 0; i < 8; ++i) reinterpret_cast<uint32_t *>(r.e)[i] = q[i];
    } else if (VEC) {
        uint4 q = make_uint4(0, 0, 0, 0);
        if (count > 0) q = *reinterpret_cast<const uint4 *>(p);
        *reinterpret_cast<uint4 *>(r.e) = q;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            r.e[i] = from_float<T>(0.0f);
            if (i < count) r.e[i] = p[i];
        }
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void store_eight(T *p, const Eight<T> &r)
{
    const uint32_t *const q = reinterpret_cast<const uint32_t *>(r.e);
    if (sizeof(T) == 4)
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(q[0]), "r"(q[1]), "r"(q[2]), "r"(q[3]), "r"(q[sizeof(T)]), "r"(q[sizeof(T) + 1]),
                     "r"(q[2 * sizeof(T) - 2]), "r"(q[2 * sizeof(T) - 1])
                     : "memory");
    else
        *reinterpret_cast<uint4 *>(p) = make_uint4(q[0], q[1], q[2], q[3]);
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T *p, int count, const float (&v)[8])
{
    if (VEC) {
        if (count <= 0) return;
        Eight<T> r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r.e[i] = from_float<T>(v[i]);
        store_eight(p, r);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = from_float<T>(v[i]);
    }
}

// --- the quantiser ------------------------------------------------------------------------------

// The smallest bf16 s with 7 s >= a, a finite and not negative.  7 s is exact (3 + 8 bits).  The product with a seventh lies within two
// units of a / 7, so cut to bf16 it is that s or one of its neighbours.
__device__ __forceinline__ float kv_scale(float a)
{
    const uint32_t cut = __float_as_uint(__fmul_rn(a, 1.0f / 7.0f)) & 0xffff0000u;
    if (7.0f * __uint_as_float(cut) < a) return __uint_as_float(cut + 0x10000u);
    return cut != 0 && 7.0f * __uint_as_float(cut - 0x10000u) >= a ? __uint_as_float(cut - 0x10000u) : __uint_as_float(cut);
}

// round-half-even(x / s) for 0 <= x <= 7 s.  The product with the reciprocal is off by a few units of its last place, so the
// code is the right one or, next to a tie, its neighbour; the remainder e = x - c s (exact: one rounding of a number of at most
// 24 bits) tells.  s and 1 / s are normal numbers (kv_codes sees to it).
__device__ __forceinline__ float kv_code(float x, float s, float r)
{
    float c = rintf(x * r);
    const float e = fmaf(-c, s, x), twice = e + e;
    const bool odd = (int)c & 1;
    if (twice > s || (twice == s && odd)) c += 1.0f;
    if (-twice > s || (-twice == s && odd)) c -= 1.0f;
    return c;
}

__device__ __forceinline__ uint32_t kv_rotate(uint32_t w) { return (w & 0x3fff3fffu) << 2 | (w >> 14 & 0x00030003u); }
__device__ __forceinline__ uint32_t kv_rotate_back(uint32_t w) { return (w >> 2 & 0x3fff3fffu) | (w & 0x00030003u) << 14; }

// Codes of eight channels as a word holds them, for the block's scale.
__device__ __noinline__ static uint32_t kv_codes_any(float v0, float v1, float v2, float v3, float v4, float v5, float v6, float v7, float s)
{
    const float v[8] = {v0, v1, v2, v3, v4, v5, v6, v7};
    const float up = s < 0x1p-100f ? 0x1p80f : 1.0f;  // away from subnormal numbers, exactly
    const float t = s * up, r = __frcp_rn(t);
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float c = kv_code(fabsf(v[i]) * up, t, r);
        word |= (uint32_t)(8 + (int)(v[i] < 0.0f ? -c : c)) << (4 * i);
    }
    return word;
}

// Two fp32 numbers in one operation
__device__ __forceinline__ uint64_t pair_of(float x, float y)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
    return v;
}
__device__ __forceinline__ void of_pair(uint64_t v, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t v;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
    return v;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b)
{
    uint64_t v;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b)
{
    uint64_t v;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}

// The same of f16 or bf16 values: x and s have 11 and 8 significant bits, so a quotient that is no tie is 2^-13 away from one at least.
// The product with a reciprocal that is off by a unit or two is off by less than 2^-18; its remainder x - q s is exact to 2^-24 of
// itself, and what the correction by it leaves is below 2^-40, so that a tie is hit and nothing else comes near one.  The sum with
// 1.5 * 2^23 + 8 rounds half to even and leaves n in its lowest bits; what stands above them adds up to a constant.  Three operations
// a value where the general form takes twelve.
__device__ __forceinline__ uint32_t kv_codes_short(float (&v)[8], float s, bool small)
{
    if (small && s < 0x1p-100f) {  // away from subnormal numbers, exactly
        s *= 0x1p80f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= 0x1p80f;
    }
    float reciprocal;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(reciprocal) : "f"(s));
    const uint64_t r = pair_of(reciprocal, reciprocal), less = pair_of(-s, -s), add = pair_of(12582920.0f, 12582920.0f);
    uint32_t word = 0;
#pragma unroll
    for (int i = 6; i >= 0; i -= 2) {
        const uint64_t x = pair_of(v[i], v[i + 1]), q = mul_pair(x, r), n = add_pair(fma_pair(fma_pair(q, less, x), r, q), add);
        word = (word * 16 + (uint32_t)(n >> 32)) * 16 + (uint32_t)n;
    }
    return word - 0x4b400000u * 0x11111111u;
}

enum { KV_ANY, KV_SHORT, KV_HALF };  // any fp32 numbers; f16 or bf16 ones; f16 ones, whose scales are above 2^-28
template <int VALUES>
__device__ __forceinline__ uint32_t kv_codes(float (&v)[8], float s)
{
    if (!(s > 0.0f)) return kv_rotate(0x88888888u);  // all zeros, or NaN
    if (VALUES != KV_ANY) return kv_rotate(kv_codes_short(v, s, VALUES == KV_SHORT));
    return kv_rotate(kv_codes_any(v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], s));
}

}  // namespace lce
