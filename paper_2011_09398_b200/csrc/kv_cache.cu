// Quantising keys and values into the 4-bit cache as they are written, and reading them back.
//
// Both kernels move memory.  A thread takes eight channels of the key and of the value of one (token, head), four threads a block of
// 32 channels, whose largest value they find with two shuffles; no value is read twice.  A block of threads works on sixteen
// consecutive tokens of a head, because that is what shares the cache's sectors: a token's values lie in two bytes each all over
// its tile.  Where the sixteen are a whole tile (a prompt) they are put together in shared memory and leave in 16-byte stores.
// 16384 tokens of 8 heads of 128 channels in bf16 (67 MB) are stored in 28 us and read back in 15; what bounds storing is the
// quantiser's instructions (73 % of the issue slots), reading the stores (32768 tokens: 36 us, 4.7 TB/s).
#include "kv_common.cuh"

#include <type_traits>

namespace lce {
namespace {

constexpr int kThreads = 256;

struct KvRows {
    KvGeom g;
    int64_t tokens;
    int32_t groups;           // of sixteen tokens
    FastDiv by_heads, by_page;
    int64_t k_token, k_head, v_token, v_head;
    const int32_t *slots;
    uint32_t *cache;
};

// The tile that a slot of the pool lies in.
__device__ __forceinline__ uint32_t *kv_tile_of(const KvRows &p, int slot, int head)
{
    const int page = p.by_page(slot), in_page = slot - page * p.g.page_size;
    const int64_t tile = ((int64_t)page * p.g.heads + head) * (p.g.page_size / kKvTile) + in_page / kKvTile;
    return p.cache + tile * kv_tile_words(p.g.blocks);
}

__device__ __forceinline__ float max_or_nan(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

__device__ __forceinline__ float scale_or_nan(float a) { return a < __uint_as_float(0x7f800000u) ? kv_scale(a) : __uint_as_float(0x7fc00000u); }

// Scales of the blocks of keys and of values that four neighbouring lanes hold, NaN where a value is not finite.
template <typename T>
struct BlockScales {  // fp32
    static __device__ __forceinline__ void find(const Eight<T> &k, const Eight<T> &v, float &ks, float &vs)
    {
        float a = fabsf(k.e[0]), b = fabsf(v.e[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) {
            a = max_or_nan(a, fabsf(k.e[i]));
            b = max_or_nan(b, fabsf(v.e[i]));
        }
#pragma unroll
        for (int d = 1; d <= 2; ++d) {
            a = max_or_nan(a, __shfl_xor_sync(0xffffffffu, a, d));
            b = max_or_nan(b, __shfl_xor_sync(0xffffffffu, b, d));
        }
        ks = scale_or_nan(a);
        vs = scale_or_nan(b);
    }
};
// 16 bits: two values at a time, then the key's and the value's largest in one word
template <typename T, typename T2>
struct PairScales {
    static __device__ __forceinline__ T2 largest(const Eight<T> &x)
    {
        const uint32_t *const w = reinterpret_cast<const uint32_t *>(x.e);
        T2 m[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t a = w[i] & 0x7fff7fffu;
            m[i] = *reinterpret_cast<const T2 *>(&a);
        }
        return __hmax2_nan(__hmax2_nan(m[0], m[1]), __hmax2_nan(m[2], m[3]));
    }
    static __device__ __forceinline__ void find(const Eight<T> &k, const Eight<T> &v, float &ks, float &vs)
    {
        const T2 a = largest(k), b = largest(v);
        const uint32_t x = *reinterpret_cast<const uint32_t *>(&a), y = *reinterpret_cast<const uint32_t *>(&b);
        const uint32_t low = __byte_perm(x, y, 0x5410), high = __byte_perm(x, y, 0x7632);  // (key, value)
        T2 m = __hmax2_nan(*reinterpret_cast<const T2 *>(&low), *reinterpret_cast<const T2 *>(&high));
#pragma unroll
        for (int d = 1; d <= 2; ++d) {
            const uint32_t o = __shfl_xor_sync(0xffffffffu, *reinterpret_cast<const uint32_t *>(&m), d);
            m = __hmax2_nan(m, *reinterpret_cast<const T2 *>(&o));
        }
        ks = scale_or_nan(to_float(m.x));
        vs = scale_or_nan(to_float(m.y));
    }
};
template <>
struct BlockScales<__half> : PairScales<__half, __half2> {};
template <>
struct BlockScales<__nv_bfloat16> : PairScales<__nv_bfloat16, __nv_bfloat162> {};

template <typename T>
constexpr int kValues = sizeof(T) == 4 ? KV_ANY : std::is_same<T, __half>::value ? KV_HALF : KV_SHORT;

// BLOCKS of 32 channels; 0: p.g.blocks.  16-bit values fit 40 registers and six blocks to an SM (16384 tokens in bf16 stored and read
// back: five 44.6 us, six 43.1); fp32 would spill.
template <typename T, bool VEC, int BLOCKS>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 6 : 5) kv_quantize_kernel(const __grid_constant__ KvRows p, const T *k, const T *v)
{
    __shared__ __align__(16) uint32_t staged[kv_tile_words(kKvMaxDim / 32)];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int blocks = BLOCKS ? BLOCKS : p.g.blocks;
    const int group = p.by_heads((int)blockIdx.x), head = blockIdx.x - group * p.g.heads;
    const int64_t token0 = (int64_t)group * kKvTile;
    const int tokens = (int)min(p.tokens - token0, (int64_t)kKvTile);
    const int threads_per_token = 4 * blocks, items = tokens * threads_per_token;
    // the block's part of an address once, in 64 bits
    const T *const key_rows = k + (token0 * p.k_token + head * p.k_head), *const value_rows = v + (token0 * p.v_token + head * p.v_head);
    Eight<T> ke, ve;
    const auto load = [&](int at) {
        const int token = at / threads_per_token, channel = 8 * (at - token * threads_per_token);
        ke = load_eight<T, VEC>(key_rows + (token * p.k_token + channel), p.g.dim - channel);
        ve = load_eight<T, VEC>(value_rows + (token * p.v_token + channel), p.g.dim - channel);
    };
    load(min((int)threadIdx.x, items - 1));  // on their way while the slots are
    // A whole tile, in order?  Every warp reads the sixteen slots for itself, which takes no barrier.
    const int first = __ldg(p.slots + token0);
    bool whole = false;
    if (tokens == kKvTile) {
        const int sixteenth = threadIdx.x % kKvTile;
        whole = __all_sync(0xffffffffu, first >= 0 && (first & 15) == 0 && first < p.g.slots && __ldg(p.slots + token0 + sixteenth) == first + sixteenth);
    }
    // whole warps go round together: the shuffles need every lane
    const auto items_to = [&](int items, auto tile_of) {
        for (int at = threadIdx.x; at - (int)(threadIdx.x & 31) < items; at += kThreads) {
            const bool there = at < items;
            const int token = (uint32_t)min(at, items - 1) / (uint32_t)threads_per_token, in_row = min(at, items - 1) - token * threads_per_token;
            const int block = in_row >> 2, quarter = in_row & 3;
            __builtin_assume(block >= 0 && block < blocks);
            if (at >= kThreads) load(min(at, items - 1));
            float kx[8], vx[8];
            ke.expand(kx);
            ve.expand(vx);
            float ks, vs;
            BlockScales<T>::find(ke, ve, ks, vs);
            int in_tile;
            uint32_t *const tile = tile_of(token, in_tile);
            if (!there || !tile) continue;
            tile[kv_key_word(blocks, in_tile, block, quarter)] = kv_codes<kValues<T>>(kx, ks);
            const uint32_t codes = kv_codes<kValues<T>>(vx, vs);
            uint16_t *const halves = reinterpret_cast<uint16_t *>(tile) + (in_tile & 1);
            halves[2 * kv_value_word(blocks, in_tile >> 1, block, 2 * quarter)] = (uint16_t)codes;
            halves[2 * kv_value_word(blocks, in_tile >> 1, block, 2 * quarter + 1)] = (uint16_t)(codes >> 16);
            if (quarter == 0) tile[kv_scale_word(blocks, in_tile, block)] = (__float_as_uint(ks) >> 16) | (__float_as_uint(vs) & 0xffff0000u);
        }
    };
    if (!whole) {
        items_to(items, [&](int token, int &in_tile) -> uint32_t * {
            const int slot = __ldg(p.slots + token0 + token);
            in_tile = slot % kKvTile;
            return slot >= 0 && slot < p.g.slots ? kv_tile_of(p, slot, head) : nullptr;
        });
        return;
    }
    items_to(kKvTile * threads_per_token, [&](int token, int &in_tile) {
        in_tile = token;
        return staged;
    });
    __syncthreads();
    uint4 *const to = reinterpret_cast<uint4 *>(kv_tile_of(p, first, head));
    for (int i = threadIdx.x; i < kv_tile_words(blocks) / 4; i += kThreads) to[i] = reinterpret_cast<const uint4 *>(staged)[i];
}

// Eight values c * s, rounded to T once; the product itself is exact in fp32.
template <typename T>
struct Values {
    T e[8];
    __device__ __forceinline__ void set(uint32_t word, uint32_t scale)  // a bf16 number in the high half
    {
        word = kv_rotate_back(word);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = from_float<T>((__uint_as_float((word >> (4 * i) & 15u) | 0x4b400000u) - 12582920.0f) * __uint_as_float(scale));
    }
};
template <>
struct Values<__nv_bfloat16> {
    // two at a time: 128 + n by one AND-OR, less 136, times s in bf16, which is the one rounding
    __nv_bfloat16 e[8];
    __device__ __forceinline__ void set(uint32_t word, uint32_t scale)
    {
        word = kv_rotate_back(word);
        const __nv_bfloat162 s = __bfloat162bfloat162(__ushort_as_bfloat16((unsigned short)(scale >> 16))), less = __bfloat162bfloat162(__ushort_as_bfloat16(0x4308));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t n = (word >> (4 * i) & 0x000f000fu) | 0x43004300u;
            const __nv_bfloat162 v = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&n), less), s);
            e[i] = v.x;
            e[i + 4] = v.y;
        }
    }
};

template <typename T, bool VEC>
__device__ __forceinline__ void store_values(T *p, int count, const Values<T> &v)
{
    if (VEC) {
        Eight<T> e;
#pragma unroll
        for (int i = 0; i < 8; ++i) e.e[i] = v.e[i];
        store_eight(p, e);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = v.e[i];
    }
}

template <typename T, bool VEC, int BLOCKS>
__global__ void __launch_bounds__(kThreads) kv_dequantize_kernel(const __grid_constant__ KvRows p, T *k, T *v)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int blocks = BLOCKS ? BLOCKS : p.g.blocks;
    const int group = p.by_heads((int)blockIdx.x), head = blockIdx.x - group * p.g.heads;
    const int64_t token0 = (int64_t)group * kKvTile;
    const int tokens = (int)min(p.tokens - token0, (int64_t)kKvTile);
    const int threads_per_token = 4 * blocks, items = tokens * threads_per_token;
    for (int at = threadIdx.x; at < items; at += kThreads) {
        const int token = at / threads_per_token, in_row = at - token * threads_per_token;
        const int block = in_row >> 2, quarter = in_row & 3, channel = in_row * 8, slot = __ldg(p.slots + token0 + token);
        if (channel >= p.g.dim) continue;
        uint32_t kw = kv_rotate(0x88888888u), vw = kw, s = 0;  // zeros for a slot outside the pool
        if (slot >= 0 && slot < p.g.slots) {
            const uint32_t *const tile = kv_tile_of(p, slot, head);
            const int in_tile = slot % kKvTile;
            s = __ldg(tile + kv_scale_word(blocks, in_tile, block));
            if (k) kw = __ldg(tile + kv_key_word(blocks, in_tile, block, quarter));
            if (v) {
                const uint16_t *const halves = reinterpret_cast<const uint16_t *>(tile) + (in_tile & 1);
                vw = __ldg(halves + 2 * kv_value_word(blocks, in_tile >> 1, block, 2 * quarter)) |
                     (uint32_t)__ldg(halves + 2 * kv_value_word(blocks, in_tile >> 1, block, 2 * quarter + 1)) << 16;
            }
        }
        const int64_t out = ((token0 + token) * p.g.heads + head) * p.g.dim + channel;
        Values<T> x;
        if (k) {
            x.set(kw, s << 16);
            store_values<T, VEC>(k + out, p.g.dim - channel, x);
        }
        if (v) {
            x.set(vw, s & 0xffff0000u);
            store_values<T, VEC>(v + out, p.g.dim - channel, x);
        }
    }
}

// A block to a head of sixteen tokens.
lce_status set_rows(KvRows *p, int64_t tokens, const int32_t *slots, const void *cache)
{
    const int64_t groups = (tokens + kKvTile - 1) / kKvTile;
    if (groups * p->g.heads >= (1ll << 31)) return LCE_ERR_UNSUPPORTED;
    p->tokens = tokens;
    p->groups = (int32_t)groups;
    fast_div_constants((uint32_t)p->g.heads, &p->by_heads.mul, &p->by_heads.sh);
    fast_div_constants((uint32_t)p->g.page_size, &p->by_page.mul, &p->by_page.sh);
    p->slots = slots;
    p->cache = static_cast<uint32_t *>(const_cast<void *>(cache));
    return LCE_OK;
}

// The kernel for so many blocks.
template <typename Kernel>
auto with_blocks(int blocks, Kernel kernel) -> decltype(kernel(std::integral_constant<int, 1>()))
{
    switch (blocks) {
        case 1: return kernel(std::integral_constant<int, 1>());
        case 2: return kernel(std::integral_constant<int, 2>());
        case 3: return kernel(std::integral_constant<int, 3>());
        case 4: return kernel(std::integral_constant<int, 4>());
        case 5: return kernel(std::integral_constant<int, 5>());
        case 6: return kernel(std::integral_constant<int, 6>());
        case 7: return kernel(std::integral_constant<int, 7>());
        default: return kernel(std::integral_constant<int, 8>());
    }
}

bool stride_ok(int64_t s) { return s >= 0 && s < (1ll << 40); }

// Whole groups of eight channels in one access: rows on 16 bytes, fp32 rows on 32
bool rows_aligned(const void *p, int64_t token_stride, int64_t head_stride, size_t size)
{
    return aligned(p, 8 * size) && token_stride % 8 == 0 && head_stride % 8 == 0;
}

template <typename T>
lce_status quantize(const KvRows &p, const void *k, const void *v, cudaStream_t s)
{
    const bool vec = p.g.dim % 8 == 0 && rows_aligned(k, p.k_token, p.k_head, sizeof(T)) && rows_aligned(v, p.v_token, p.v_head, sizeof(T));
    return launch_dependent(vec ? with_blocks(p.g.blocks, [](auto b) { return kv_quantize_kernel<T, true, b.value>; }) : kv_quantize_kernel<T, false, 0>, dim3((unsigned)(p.groups * p.g.heads)), kThreads, 0, s, p,
                            static_cast<const T *>(k), static_cast<const T *>(v));
}

template <typename T>
lce_status dequantize(const KvRows &p, void *k, void *v, cudaStream_t s)
{
    const bool vec = p.g.dim % 8 == 0 && aligned(k, 8 * sizeof(T)) && aligned(v, 8 * sizeof(T));
    return launch_dependent(vec ? with_blocks(p.g.blocks, [](auto b) { return kv_dequantize_kernel<T, true, b.value>; }) : kv_dequantize_kernel<T, false, 0>, dim3((unsigned)(p.groups * p.g.heads)), kThreads, 0, s, p,
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
    if (set_rows(&p, tokens, slots, cache) != LCE_OK) return LCE_ERR_UNSUPPORTED;
    p.k_token = k_token_stride; p.k_head = k_head_stride; p.v_token = v_token_stride; p.v_head = v_head_stride;
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
    if (set_rows(&p, tokens, slots, cache) != LCE_OK) return LCE_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (type) {
        case LCE_TYPE_FLOAT32: return dequantize<float>(p, k, v, s);
        case LCE_TYPE_FLOAT16: return dequantize<__half>(p, k, v, s);
        default: return dequantize<__nv_bfloat16>(p, k, v, s);
    }
}
