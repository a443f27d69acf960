// Quantising keys and values into the 4-bit cache as they are written, and reading them back.
//
// Both kernels move memory: a thread takes eight channels of the key and of the value of one (token, head), four threads a
// block of 32 channels, whose largest value they find with two shuffles; no value is read twice.
#include "kv_common.cuh"

namespace lce {
namespace {

constexpr int kThreads = 256;

struct KvRows {
    KvGeom g;
    int64_t items;            // (token, head, block, quarter), the quarter fastest
    int64_t k_token, k_head, v_token, v_head;
    const int32_t *slots;
    uint32_t *cache;
};

struct KvItem {
    int64_t token;
    int head, block, quarter, slot;
};

__device__ __forceinline__ KvItem kv_item(const KvRows &p, int64_t at)
{
    KvItem it;
    it.quarter = (int)(at & 3);
    const int64_t row = (at >> 2) / p.g.blocks;
    it.block = (int)((at >> 2) - row * p.g.blocks);
    it.token = row / p.g.heads;
    it.head = (int)(row - it.token * p.g.heads);
    it.slot = __ldg(p.slots + it.token);
    return it;
}

__device__ __forceinline__ uint32_t *kv_tile_of(const KvRows &p, const KvItem &it)
{
    const int page = it.slot / p.g.page_size, in_page = it.slot - page * p.g.page_size;
    const int64_t tile = ((int64_t)page * p.g.heads + it.head) * (p.g.page_size / kKvTile) + in_page / kKvTile;
    return p.cache + tile * kv_tile_words(p.g.blocks);
}

// Scale of the block that four neighbouring lanes hold, NaN where a value is not finite.
__device__ __forceinline__ float block_scale(const float (&v)[8])
{
    uint32_t a = 0;  // magnitudes compare like integers, NaN and infinity above all others
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(v[i]) & 0x7fffffffu);
    a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
    a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
    return a >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : kv_scale(__uint_as_float(a));
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) kv_quantize_kernel(const __grid_constant__ KvRows p, const T *k, const T *v)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t step = (int64_t)gridDim.x * kThreads;
    // whole warps go round together: the shuffles need every lane
    for (int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x; at - (threadIdx.x & 31) < p.items; at += step) {
        const bool there = at < p.items;
        const KvItem it = kv_item(p, there ? at : p.items - 1);
        const int channel = it.block * 32 + it.quarter * 8;
        float kx[8], vx[8];
        load8<T, VEC>(k + it.token * p.k_token + it.head * p.k_head + channel, p.g.dim - channel, kx);
        load8<T, VEC>(v + it.token * p.v_token + it.head * p.v_head + channel, p.g.dim - channel, vx);
        const float ks = block_scale(kx), vs = block_scale(vx);
        if (!there || it.slot < 0 || it.slot >= p.g.slots) continue;
        uint32_t *const tile = kv_tile_of(p, it);
        const int token = it.slot % kKvTile;
        tile[kv_key_word(p.g.blocks, token, it.block, it.quarter)] = kv_codes(kx, ks);
        const uint32_t codes = kv_codes(vx, vs);
        uint16_t *const halves = reinterpret_cast<uint16_t *>(tile) + (token & 1);
        halves[2 * kv_value_word(p.g.blocks, token >> 1, it.block, 2 * it.quarter)] = (uint16_t)codes;
        halves[2 * kv_value_word(p.g.blocks, token >> 1, it.block, 2 * it.quarter + 1)] = (uint16_t)(codes >> 16);
        if (it.quarter == 0) tile[kv_scale_word(p.g.blocks, token, it.block)] = (__float_as_uint(ks) >> 16) | (__float_as_uint(vs) & 0xffff0000u);
    }
}

__device__ __forceinline__ void kv_values(uint32_t word, float s, float (&v)[8])
{
    word = kv_rotate_back(word);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)((int)((word >> (4 * i)) & 15u) - 8) * s;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) kv_dequantize_kernel(const __grid_constant__ KvRows p, T *k, T *v)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t step = (int64_t)gridDim.x * kThreads;
    for (int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x; at < p.items; at += step) {
        const KvItem it = kv_item(p, at);
        const int channel = it.block * 32 + it.quarter * 8;
        if (channel >= p.g.dim) continue;
        float kx[8] = {}, vx[8] = {};
        if (it.slot >= 0 && it.slot < p.g.slots) {
            const uint32_t *const tile = kv_tile_of(p, it);
            const int token = it.slot % kKvTile;
            const uint32_t s = __ldg(tile + kv_scale_word(p.g.blocks, token, it.block));
            if (k) kv_values(__ldg(tile + kv_key_word(p.g.blocks, token, it.block, it.quarter)), __uint_as_float(s << 16), kx);
            if (v) {
                const uint16_t *const halves = reinterpret_cast<const uint16_t *>(tile) + (token & 1);
                const uint32_t lo = __ldg(halves + 2 * kv_value_word(p.g.blocks, token >> 1, it.block, 2 * it.quarter));
                const uint32_t hi = __ldg(halves + 2 * kv_value_word(p.g.blocks, token >> 1, it.block, 2 * it.quarter + 1));
                kv_values(lo | hi << 16, __uint_as_float(s & 0xffff0000u), vx);
            }
        }
        const int64_t out = (it.token * p.g.heads + it.head) * p.g.dim + channel;
        if (k) store8<T, VEC>(k + out, p.g.dim - channel, kx);
        if (v) store8<T, VEC>(v + out, p.g.dim - channel, vx);
    }
}

int grid_for(int64_t items)
{
    const int64_t blocks = (items + kThreads - 1) / kThreads;
    return (int)(blocks < 148 * 8 ? blocks : 148 * 8);
}

bool stride_ok(int64_t s) { return s >= 0 && s < (1ll << 40); }

// 16-byte accesses: whole groups of eight channels, rows on 16 bytes
bool rows_on_16(const void *p, int64_t token_stride, int64_t head_stride, size_t size)
{
    return aligned(p, 16) && token_stride * size % 16 == 0 && head_stride * size % 16 == 0;
}

template <typename T>
lce_status quantize(const KvRows &p, const void *k, const void *v, cudaStream_t s)
{
    const bool vec = p.g.dim % 8 == 0 && rows_on_16(k, p.k_token, p.k_head, sizeof(T)) && rows_on_16(v, p.v_token, p.v_head, sizeof(T));
    return launch_dependent(vec ? kv_quantize_kernel<T, true> : kv_quantize_kernel<T, false>, dim3(grid_for(p.items)), kThreads, 0, s, p,
                            static_cast<const T *>(k), static_cast<const T *>(v));
}

template <typename T>
lce_status dequantize(const KvRows &p, void *k, void *v, cudaStream_t s)
{
    const bool vec = p.g.dim % 8 == 0 && aligned(k, 16) && aligned(v, 16);
    return launch_dependent(vec ? kv_dequantize_kernel<T, true> : kv_dequantize_kernel<T, false>, dim3(grid_for(p.items)), kThreads, 0, s, p,
                            static_cast<T *>(k), static_cast<T *>(v));
}

}  // namespace
}  // namespace lce

extern "C" size_t lce_kv_cache_bytes(const lce_kv_desc *desc)
{
    using namespace lce;
    KvGeom g;
    if (make_kv_geom(desc, &g) != LCE_OK) return 0;
    return (size_t)(g.slots / kKvTile) * g.heads * kv_tile_words(g.blocks) * 4;
}

extern "C" lce_status lce_kv_quantize(const lce_kv_desc *desc, const void *k, const void *v, int32_t type, int64_t tokens, int64_t k_token_stride,
                                      int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride, const int32_t *slots, void *cache,
                                      void *stream)
{
    using namespace lce;
    KvRows p{};
    const lce_status st = make_kv_geom(desc, &p.g);
    if (st != LCE_OK) return st;
    if (!type_known(type) || tokens < 0 || !stride_ok(k_token_stride) || !stride_ok(k_head_stride) || !stride_ok(v_token_stride) || !stride_ok(v_head_stride))
        return LCE_ERR_INVALID_ARG;
    if (tokens >= (1ll << 31)) return LCE_ERR_UNSUPPORTED;
    if (tokens == 0) return LCE_OK;
    if (!k || !v || !slots || !cache) return LCE_ERR_INVALID_ARG;
    if (!aligned(k, type_size(type)) || !aligned(v, type_size(type)) || !aligned(slots, 4) || !aligned(cache, 16)) return LCE_ERR_ALIGNMENT;
    p.items = tokens * p.g.heads * p.g.blocks * 4;
    p.k_token = k_token_stride; p.k_head = k_head_stride; p.v_token = v_token_stride; p.v_head = v_head_stride;
    p.slots = slots;
    p.cache = static_cast<uint32_t *>(cache);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (type) {
        case LCE_TYPE_FLOAT32: return quantize<float>(p, k, v, s);
        case LCE_TYPE_FLOAT16: return quantize<__half>(p, k, v, s);
        default: return quantize<__nv_bfloat16>(p, k, v, s);
    }
}

extern "C" lce_status lce_kv_dequantize(const lce_kv_desc *desc, const void *cache, const int32_t *slots, int64_t tokens, int32_t type, void *k, void *v,
                                        void *stream)
{
    using namespace lce;
    KvRows p{};
    const lce_status st = make_kv_geom(desc, &p.g);
    if (st != LCE_OK) return st;
    if (!type_known(type) || tokens < 0) return LCE_ERR_INVALID_ARG;
    if (tokens >= (1ll << 31)) return LCE_ERR_UNSUPPORTED;
    if (tokens == 0) return LCE_OK;
    if ((!k && !v) || !slots || !cache) return LCE_ERR_INVALID_ARG;
    if (!aligned(k, type_size(type)) || !aligned(v, type_size(type)) || !aligned(slots, 4) || !aligned(cache, 16)) return LCE_ERR_ALIGNMENT;
    p.items = tokens * p.g.heads * p.g.blocks * 4;
    p.slots = slots;
    p.cache = static_cast<uint32_t *>(const_cast<void *>(cache));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (type) {
        case LCE_TYPE_FLOAT32: return dequantize<float>(p, k, v, s);
        case LCE_TYPE_FLOAT16: return dequantize<__half>(p, k, v, s);
        default: return dequantize<__nv_bfloat16>(p, k, v, s);
    }
}
