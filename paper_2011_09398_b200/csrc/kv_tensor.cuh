// What the kernels have in common that multiply keys of the 4-bit cache on the 5th-generation tensor cores: products of f16 operands in
// shared memory, accumulators read from TMEM, 4-bit words decoded to f16, the four producer warps' meetings, bounded waits.
#pragma once
#include "kv_attention.cuh"
#include "mx_common.cuh"

namespace lce {

constexpr int kTokens = 128;  // of a tile there: eight tiles of the cache

__device__ __forceinline__ void mma_shared(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
// Operand in shared memory without swizzle: 8 rows x 16 bytes are 128 bytes in a row, those of the next eight k behind them, those of the next
// eight rows `rows8` bytes on.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t rows8)
{
    return (uint64_t)(at >> 4) | (uint64_t)(128 >> 4) << 16 | (uint64_t)(rows8 >> 4) << 32 | 1ull << 46;
}

// 128 columns
__device__ __forceinline__ void tmem_load128(uint32_t at, uint32_t (&r)[128])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31"
        "}, [%128];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63"
        "}, [%129];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%64,%65,%66,%67,%68,%69,%70,%71,%72,%73,%74,%75,%76,%77,%78,%79,%80,%81,%82,%83,%84,%85,%86,%87,%88,%89,%90,%91,%92,%93,%94,%95"
        "}, [%130];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%96,%97,%98,%99,%100,%101,%102,%103,%104,%105,%106,%107,%108,%109,%110,%111,%112,%113,%114,%115,%116,%117,%118,%119,%120,%121,%122,%123,%124,%125,"
        "%126,%127"
        "}, [%131];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), 
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), 
          "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), 
          "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), 
          "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]), 
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63]), "=r"(r[64]), "=r"(r[65]), "=r"(r[66]), 
          "=r"(r[67]), "=r"(r[68]), "=r"(r[69]), "=r"(r[70]), "=r"(r[71]), "=r"(r[72]), "=r"(r[73]), "=r"(r[74]), "=r"(r[75]), "=r"(r[76]), "=r"(r[77]), 
          "=r"(r[78]), "=r"(r[79]), "=r"(r[80]), "=r"(r[81]), "=r"(r[82]), "=r"(r[83]), "=r"(r[84]), "=r"(r[85]), "=r"(r[86]), "=r"(r[87]), "=r"(r[88]), 
          "=r"(r[89]), "=r"(r[90]), "=r"(r[91]), "=r"(r[92]), "=r"(r[93]), "=r"(r[94]), "=r"(r[95]), "=r"(r[96]), "=r"(r[97]), "=r"(r[98]), "=r"(r[99]), 
          "=r"(r[100]), "=r"(r[101]), "=r"(r[102]), "=r"(r[103]), "=r"(r[104]), "=r"(r[105]), "=r"(r[106]), "=r"(r[107]), "=r"(r[108]), "=r"(r[109]), 
          "=r"(r[110]), "=r"(r[111]), "=r"(r[112]), "=r"(r[113]), "=r"(r[114]), "=r"(r[115]), "=r"(r[116]), "=r"(r[117]), "=r"(r[118]), "=r"(r[119]), 
          "=r"(r[120]), "=r"(r[121]), "=r"(r[122]), "=r"(r[123]), "=r"(r[124]), "=r"(r[125]), "=r"(r[126]), "=r"(r[127])
        : "r"(at), "r"(at + 32), "r"(at + 64), "r"(at + 96)
        : "memory");
}
// 32 columns on their way, and there.
__device__ __forceinline__ void tmem_begin32(uint32_t at, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31"
        "}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
          "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at)
        : "memory");
}
__device__ __forceinline__ void tmem_end32(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
          "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]),
          "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}

// The B words of a place (a lane's of ROWS = 64 places, a token's of 16), plane by plane.
template <int B, int ROWS>
__device__ __forceinline__ void load_planes(const uint32_t *base, int place, uint32_t (&w)[B])
{
    if (B == 4) {
        const uint4 v = __ldg(reinterpret_cast<const uint4 *>(base) + place);
        w[0] = v.x; w[B > 1 ? 1 : 0] = v.y; w[B > 2 ? 2 : 0] = v.z; w[B > 3 ? 3 : 0] = v.w;
    } else {
        if (B & 2) {
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(base) + place);
            w[0] = v.x; w[B > 1 ? 1 : 0] = v.y;
        }
        if (B & 1) w[B - 1] = __ldg(base + ROWS * (B - 1) + place);
    }
}

__device__ __forceinline__ uint32_t half2_bits(__half2 v) { return *reinterpret_cast<const uint32_t *>(&v); }
__device__ __forceinline__ __half2 as_half2(uint32_t v) { return *reinterpret_cast<const __half2 *>(&v); }
// c s of the eight codes of a word, pair by pair: codes 0 and 4 (of the low and the high half), 1 and 5, 2 and 6, 3 and 7.
__device__ __forceinline__ uint4 decode(uint32_t word, __half2 scale)
{
    constexpr uint32_t kEven = 0x003c003cu, kOdd = 0x03c003c0u, kBase = 0x64006400u;
    const __half2 quarter = as_half2(0x34003400u), less264 = as_half2(0xdc20dc20u), part64 = as_half2(0x24002400u), less24 = as_half2(0xce00ce00u);
    const uint32_t other = swap_bytes(word);
    return make_uint4(half2_bits(__hmul2(__hfma2(as_half2(and_or(word, kEven, kBase)), quarter, less264), scale)),
                      half2_bits(__hmul2(__hfma2(as_half2(and_or(word, kOdd, kBase)), part64, less24), scale)),
                      half2_bits(__hmul2(__hfma2(as_half2(and_or(other, kEven, kBase)), quarter, less264), scale)),
                      half2_bits(__hmul2(__hfma2(as_half2(and_or(other, kOdd, kBase)), part64, less24), scale)));
}

__device__ __forceinline__ uint32_t key_scale(uint32_t word) { return word << 16; }  // as fp32 bits
__device__ __forceinline__ void producers_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
// The same, and whether all of them are well: where one's wait gave up, all leave together.
__device__ __forceinline__ bool producers_sync_and(bool ok)
{
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\t"
        "bar.red.and.pred p, 1, 128, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(all)
        : "r"((uint32_t)ok)
        : "memory");
    return all != 0;
}

// mbar_wait_bounded in place: a kernel that calls a function cannot share its registers out.
__device__ __forceinline__ bool wait_bounded(uint64_t *bar, uint32_t parity)
{
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = globaltimer_ns();
    do {
#pragma unroll 1
        for (int i = 0; i < 32; ++i)
            if (mbar_try_wait(bar, parity)) return true;
    } while (globaltimer_ns() - t0 < kWaitLimitNs);
    return false;
}

// The page that lane l's tile of the cache, the l-th of eight, lies on; negative behind the sequence.  Only loaded here: what is done with
// it comes a tile later.
__device__ __forceinline__ int32_t find_page(const AttnParams &p, const int32_t *table, int length, int tile, int lane)
{
    const int32_t t = tile * 8 + lane;
    if (lane >= 8 || t >= (length + kKvTile - 1) / kKvTile) return -1;
    return __ldg(table + t / (p.g.page_size / kKvTile));
}

}  // namespace lce
