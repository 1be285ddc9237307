// Attention of trees of drafted tokens over the 4-bit paged cache (wide_attn_tree): every new row sees the prefix of its sequence and, of the
// new tokens, those that its bits name.
//
// A tree of 8 to 64 tokens and 4 query heads a KV head has 32 to 256 query rows that share every key, many more than the 8 to 24 that
// wide_attn_cache keeps in registers, so here the codes become 16-bit tiles in shared memory once and the products run on
// tcgen05, 64 or 128 query rows a pass.  Keys are the 128-row operand, so what a tile costs follows the rows there are:
//     S^T [128 keys (TMEM lanes)][rows]      = K [128 x D]   Q^T
//     P^T = exp2(S^T scale - ref)              a thread has one key; written to shared memory as [key][row]
//     O^T [D channels (lanes)][rows]        += V^T [D x 128] P^T   (V as unpacked, [key][channel], is the MN-major operand)
// The reference `ref` of a row is raised (and its O rescaled in TMEM) only when a logit passes it by 2^kSlack; the sums of P over the keys
// are a second product, with ones in V's place.
//
// Everything 16-bit is fp16 where that holds it well, else bf16 (2^-11 against 2^-8: with bf16 for K, V and P the 2-norm of the error was 0.0033,
// twice that of the output's own rounding, which is what is left now).  P is up to 2^15 (a row's largest is 2^7 when its reference is set), so that what fp16
// loses at its lower end is 2^-32 of the largest.  A value's type goes by its block of 16 keys, a step of the product; queries' and keys' by the item; a
// key out of the type's range is taken times a power of two, which its thread of the softmax puts into the logit.
//
// Roles: a warp that walks the items and brings 16-key blocks by bulk copies, eight warps that unpack them, sixteen that make P and
// the outputs, in two streams, and a warp for each of the two products.  K is unpacked for the next tile while the softmax has this
// one.  Unpacking takes 3.25 instructions for two values: a code n in the low bits of the fp16 number 1024 is 1024 + n, four bits further up 1024 + 16 n;
// taking 1024 off is exact, and one fma rounds m + s n, or m + (s / 16) 16 n, once.  With the fragment order in which
// the codes lie, keys go out as 16-byte rows and values through transposing 8x8 stores; O's channels come out permuted within 32.
//
// What bounds it: instructions and hand-overs.  In long items a tile of 128 keys is 8.5 thousand warp instructions with 64 rows and 11.3 with 128, and takes 3700 and 4800 clocks (57 and
// 59 % of the issue slots; over a whole call 56 %).  So 64 rows' probabilities are 2.8 thousand, and 5.6 are the unpacking: 1.7 of them the arithmetic above, the rest parameters and
// their words, addresses, stores, waits.  61 nodes on 32768 tokens, 32 heads on 8: 98 us in a stream of calls; 32 sequences of 17 to
// 8192 tokens with 16 nodes each: 175 us.  What did not help: moving registers between the
// warpgroups, unpacking K and V by warps of their own (eight left for the softmax: 117 against 100 us), packed fp32 arithmetic.
//
// Items are cut into equal pieces for the CTAs and joined as in wide_attn_cache (attn_plan.cuh).
#include <cuda_fp16.h>

#include <atomic>
#include <type_traits>

#include "cache.cuh"

namespace {

constexpr int kItemCost = 40;      // units that an item counts on top of its blocks: queries in, results out
// One CTA takes an item alone where cutting it would take longer.  us alone / cut: 8 items of 32 blocks 23.8 / 20.5, of 94 38.7 / 22.4; 40 items of 32 blocks 25.2 / 26.2, of 44
// 28.9 / 26.3, of 94 39.6 / 31.0; 96 items of 44 blocks 28.6 / 32.3, of 94 39.9 / 42.5: joining is 10 to 17 blocks.  A launch that knows that nothing is
// cut saves the joining kernel, 2.5 us, so where page tables have room for kItemShort blocks nothing is (8 items of 19 blocks 21.5 / 20.3, 96 items 22.6 / 26.5).
constexpr int kItemAlone = 96, kItemJoin = 14, kItemShort = 24;

}  // namespace

#include "attn_plan.cuh"

namespace {

constexpr int kTile = 8;            // blocks of a tile: 128 keys
constexpr int kKeys = 16 * kTile;
constexpr int kMostRing = 3;        // tiles of codes on their way
// A part of an item longer than this is taken in portions, whose results are joined in the workspace like those of CTAs.  The tensor cores cut a sum off at
// every addition, a step of 16 keys, always towards zero: up to 2^-24 of the sum on average, so 4096 steps lose 2.4e-4.  In one portion, the 2-norm of the error over a
// million keys was 0.0029 (64 rows, two streams) and 0.0055 (128 rows), and grew with the length (the sums of P lose more than outputs of both signs do): 0.0017 in portions.
constexpr int kPortion = 512;       // tiles
constexpr int kDescs = 8;           // tiles that are known: the ring's, and at most three behind it whose softmax is not done
constexpr int kUnpackWarps = 8, kSoftWarps = 16, kGroups = kSoftWarps / 4;
constexpr int kLoadWarp = kUnpackWarps + kSoftWarps, kScoreWarp = kLoadWarp + 1, kValueWarp = kLoadWarp + 2, kWarps = kLoadWarp + 3;
constexpr float kSlack = 8.f;
constexpr float kHigh = 7.f;         // log2 of a row's largest probability when its reference is set
constexpr int kOnes = 1280, kOnesWide = 512;    // bytes of ones in fp16, in bf16
constexpr float kNothing = 1e38f;    // minus the reference of a row that has seen nothing yet: a logit of any size passes it
constexpr int kHalf = 16384;        // bytes of [128 keys][64 channels or rows]

struct TreeArgs : AttnArgs {
    const uint32_t* tree;
    int tree_words;
    int* timeout;                   // takes WIDE_ERR_TIMEOUT
    unsigned long long wait_ns;
};

struct Tile {                       // what the roles are told of a tile
    int blk, nb;                    // first block, blocks
    uint32_t present;               // bit b: block b has a page
    int first;                      // of a portion of the item's part in this CTA
    int index, left, item;          // tiles of the portion before this one (2: two or more); behind it; the portion's number in the CTA
    int masked;                     // not all rows see all 128 keys
    int kvh, rb, row0, n_rows, len;
    int item_rows, rows_a_block;    // query rows of the item; of a whole one
    int begins, ends;               // whether the part has the item's first, last block
    int goes_on, more;              // the portion is not the part's first, last one
    int final;                      // the CTA's last tile
};

struct alignas(16) Shared {
    uint64_t ring_full[kMostRing], ring_empty[kMostRing], k_full, k_free, v_full[2], v_free[2], s_full[2], s_free[2], p_full[2], pv_done[2], read[2], meet[kGroups], q_meet;
    uint32_t tmem;
    int abort;
    int n_tiles;                    // of this CTA, once it is known
    int ref_at[kGroups];            // which reference a group used in its last tile of an item
    Cursor start;
    Tile tiles[kDescs];
    alignas(16) float minus_ref[2][128];        // of a stream's row, twice: the one in use and the next
    float most[4][128];             // of a stream's row, per warp of a group: the largest logit
    alignas(16) int flag[4][kGroups][4];        // [tile of the stream][group][warp]: a logit passed its reference
    float key_by[4][kKeys];         // of a tile's key: what its products with q are taken times to be logits, in powers of two
    uint8_t odd[4][kKeys];          // sub-groups of a new token's values that are not finite (their values are 0 in the tile)
    alignas(8) uint8_t wide[4][kUnpackWarps];     // of a tile: whether a block's values (and probabilities) are bf16, not fp16
    alignas(8) uint8_t q_wide[4][kUnpackWarps];   // of an item: whether queries that the warp brought do not fit fp16 (queries and keys are bf16 then)
    uint32_t spoilt[256];           // of a row: such sub-groups that it sees (for two items of 128 rows, or four of 64)
};

template <int D, int G, int NB>
struct Layout {
    static constexpr int kRows = 64 * NB, kNS = D / G, kSB = 16 * D + 128 * kNS, kStage = kTile * kSB, kBlocks = D / 64;
    static constexpr int kTileBytes = kBlocks * kHalf;                 // of unpacked keys, or values
    static constexpr int kRing = D == 128 && NB == 2 && G == 32 ? 2 : kMostRing;     // (no room for three)
    static constexpr int kQ = 0, kK = kQ + kBlocks * kRows * 128, kV = kK + kTileBytes, kP = kV + 2 * kTileBytes, kCodes = kP + 2 * kHalf,
                         kOnesAt = kCodes + kRing * kStage, kPlan = kOnesAt + kOnes + kOnesWide;
    static constexpr int kPlanRoom = 227 * 1024 - 1024 - kPlan - static_cast<int>(sizeof(Shared)) - 512 < 16384
                                         ? (227 * 1024 - 1024 - kPlan - static_cast<int>(sizeof(Shared)) - 512) / 256 * 256 : 16384;
    static constexpr int kSmem = kPlan + kPlanRoom + 1024;
    static constexpr uint32_t kCols = 512, kO = 2 * kRows, kSum = kO + 128;     // two buffers of scores, two streams' outputs and sums of P
    static __device__ __forceinline__ int spoilt_at(int item, int row) { return NB == 1 ? (item & 3) * 64 + row : (item & 1) * 128 + row; }
    static_assert(kPlanRoom >= 1024 && kSmem + sizeof(Shared) <= 227 * 1024, "shared memory");
};

// MN-major operand in the 128-byte swizzle: rows of 64 elements, one per step of K; blocks of 64 elements `lbo` bytes apart
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr, uint32_t lbo) {
    return umma_desc_sw128(addr & ~0u) & ~(static_cast<uint64_t>(0x3FFF) << 16) | static_cast<uint64_t>(lbo >> 4) << 16;
}
// the same where all elements are one number: groups of 8 rows 128 bytes apart
__device__ __forceinline__ uint64_t desc_ones(uint32_t addr) {
    return umma_desc_sw128(addr) & ~(static_cast<uint64_t>(0x3FFF) << 16 | static_cast<uint64_t>(0x3FFF) << 32) | static_cast<uint64_t>(128 >> 4) << 16 | static_cast<uint64_t>(128 >> 4) << 32;
}
// in less room, without a swizzle: matrices of 8 x 8 elements 16 bytes apart (a product reads them at half the speed)
__device__ __forceinline__ uint64_t desc_ones_wide(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | static_cast<uint64_t>(1) << 16 | static_cast<uint64_t>(1) << 32 | static_cast<uint64_t>(1) << 46;
}
__host__ __device__ constexpr uint32_t idesc(int n, bool half, bool mn_major) {
    return umma_idesc_bf16(128, n) & ~(half ? (1u << 7) | (1u << 10) : 0u) | (mn_major ? (1u << 15) | (1u << 16) : 0u);
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void store_transposed(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ void sts32(uint32_t a, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }

__device__ __forceinline__ __nv_bfloat162 as_bf162(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
__device__ __forceinline__ uint32_t as_word(__nv_bfloat162 b) { return *reinterpret_cast<const uint32_t*>(&b); }
__device__ __forceinline__ __half2 as_half2(uint32_t w) { return *reinterpret_cast<const __half2*>(&w); }
__device__ __forceinline__ uint32_t as_word(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }
__device__ __forceinline__ uint32_t half_pair(float lo, float hi) { return as_word(__floats2half2_rn(lo, hi)); }
__device__ __forceinline__ float low_of(uint32_t w) { return __uint_as_float(w << 16); }        // of two bf16 numbers
__device__ __forceinline__ float high_of(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// m + s n in bf16 of the two codes in bits 0..3 and 16..19 of w
__device__ __forceinline__ uint32_t unpack_two(uint32_t w, uint32_t s, uint32_t m) {
    const uint32_t high = (w & 0x000F000Fu) | 0x43004300u;       // 128 + n
    return as_word(__hfma2(__hsub2(as_bf162(high), as_bf162(0x43004300u)), as_bf162(s), as_bf162(m)));
}
// m + s n in fp16 of the two codes in bits 0..3 and 16..19, or, with s / 16 for s, in bits 4..7 and 20..23
template <bool UPPER>
__device__ __forceinline__ uint32_t unpack_half(uint32_t w, uint32_t s, uint32_t m) {
    const uint32_t high = (w & (UPPER ? 0x00F000F0u : 0x000F000Fu)) | 0x64006400u;       // 1024 + n, or 16 n
    return as_word(__hfma2(__hsub2(as_half2(high), as_half2(0x64006400u)), as_half2(s), as_half2(m)));
}
__device__ __forceinline__ uint32_t sixteenth(uint32_t s) { return as_word(__hmul2(as_half2(s), as_half2(0x2C002C00u))); }
// The exponent bits of x, so that 2^-e x is 2^8 to 2^9 and neither power leaves the normal numbers.
__device__ __forceinline__ uint32_t exponent_of(float x) { return min(max(__float_as_uint(x) & 0x7F800000u, 9u << 23), 254u << 23); }
__device__ __forceinline__ float times_to_256(uint32_t e) { return __uint_as_float((262u << 23) - e); }
__device__ __forceinline__ float times_back(uint32_t e) { return __uint_as_float(e - (8u << 23)); }
__device__ __forceinline__ bool not_finite(uint32_t word) { return (word & 0x7F80u) == 0x7F80u || (word & 0x7F800000u) == 0x7F800000u; }

__device__ __forceinline__ void tmem_ld_32x4(uint32_t taddr, uint32_t (&r)[4]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr) : "memory");
}

// By one lane of a whole, converged warp.
__device__ __forceinline__ void umma_bf16_elect(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void umma_commit_elect(uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar)
        : "memory");
}

// Bit e: query row r0 + e of the tile's item sees the key key0 + lane of the tile.  Lane e gets the bits of row e for the 32 keys, and then
// all lanes get each row's.  Out of line: few tiles have keys that not every row sees.
__device__ __noinline__ uint32_t sees_of(const TreeArgs* a, const Tile* d, int r0, int key0) {
    const int lane = threadIdx.x & 31, key = key0 + lane;
    const RowBlock rows = row_block(*a, d->rb * d->rows_a_block + r0);
    const int tok = row_of(*a, rows, lane & 15).tok, node = d->blk * 16 + key0 - (d->len - d->n_rows);   // of lane 0; negative in the prefix
    uint32_t bits = 0;
    if (tok < d->n_rows) {
        const uint32_t* row = a->tree + static_cast<size_t>(d->row0 + tok) * a->tree_words;
        const int w = node >> 5;           // rounds down
        const uint32_t lo = w < 0 ? 0xffffffffu : w < a->tree_words ? row[w] : 0u, hi = w + 1 < 0 ? 0xffffffffu : w + 1 < a->tree_words ? row[w + 1] : 0u;
        bits = __funnelshift_r(lo, hi, node & 31);
    }
    const bool is = (key >> 4) < d->nb && ((d->present >> (key >> 4)) & 1u) && d->blk * 16 + key < d->len;
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) m |= ((__shfl_sync(0xffffffffu, bits, e) >> lane) & 1u) << e;
    return is ? m : 0u;
}

// The largest of each of the 16 values over the 32 lanes: lanes 2 e and 2 e + 1 get that of value e.  x is used up.
__device__ __forceinline__ float largest_across_lanes(float (&x)[16], int lane) {
#pragma unroll
    for (int half = 8; half > 0; half >>= 1)
#pragma unroll
        for (int e = 0; e < half; ++e) {
            const bool up = lane & (2 * half);
            const float give = up ? x[e] : x[e + half], keep = up ? x[e + half] : x[e];
            x[e] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, 2 * half));
        }
    return fmaxf(x[0], __shfl_xor_sync(0xffffffffu, x[0], 1));
}

// The largest magnitude among eight bf16 numbers, as bits; of an infinity or a NaN: 0x7F80 or more.
__device__ __forceinline__ uint32_t largest_bits(const uint4& v) {
    const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
    return max(m & 0xFFFFu, m >> 16);
}
__device__ __forceinline__ uint32_t to_half(uint32_t w) { return half_pair(low_of(w), high_of(w)); }

// Whether fp16 holds a sub-group's numbers well, from its word (step, minimum): s / 16 and what the values are rounded to.  `least`: the bits of the
// smallest step; the largest is 2^10 and the minimum up to 2^14, so that no value is above 2^15.
constexpr uint32_t kLeastKey = 0x3A80u, kLeastValue = 0x3900u;       // 2^-10: what is below fp16's normal numbers is 2^-18 of the key's largest; 2^-13: s / 16 is exact
__device__ __forceinline__ bool fits_half(uint32_t w, uint32_t least) { return w == 0 || ((w & 0xFFFFu) - least < 0x4480u - least && (w & 0x7FFF0000u) < 0x46800000u); }
// The same of a sub-group of one number (step 0): fp16 has its 8 digits as they are from 2^-14 up.
__device__ __forceinline__ bool constant_fits_half(uint32_t w) { return (w & 0xFFFFu) == 0 && (w & 0x7FFF0000u) - 0x38800000u < 0x46800000u - 0x38800000u; }

// The words of a warp's block of which some do not fit.  Out of line: few need it.  A key's are taken times a power of two so that its largest number is
// 2^8 to 2^9 (the power goes into its logits), unless keys are bf16.  Values' stay bf16 where one does not fit.
template <int NS>
__device__ __noinline__ bool odd_words(uint32_t words, float* key_by, bool wide_keys, float scale) {
    const int lane = threadIdx.x & 31;
    uint32_t w[(NS + 1) / 2];
    bool half = true;
#pragma unroll
    for (int i = 0; i < (NS + 1) / 2; ++i) {
        const int x = 32 * i + (NS > 1 ? lane : lane & 15);
        const uint32_t at = words + 4 * x, kw = lds32(at);
        float top = fmaxf(fabsf(high_of(kw)), fabsf(fmaf(15.f, low_of(kw), high_of(kw))));
#pragma unroll
        for (int o = 1; o < NS; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const uint32_t e = exponent_of(top);
        w[i] = lds32(at + 64 * NS);
        half = __all_sync(0xffffffffu, fits_half(w[i], kLeastValue) || constant_fits_half(w[i])) && half;
        if (!wide_keys) sts32(at, half_pair(low_of(kw) * times_to_256(e), high_of(kw) * times_to_256(e)));
        if (x % NS == 0) key_by[x / NS] = wide_keys ? scale : times_back(e) * scale;
    }
#pragma unroll
    for (int i = 0; i < (NS + 1) / 2; ++i)
        if (half) sts32(words + 64 * NS + 4 * (32 * i + (NS > 1 ? lane : lane & 15)), to_half(w[i]));
    return half;
}

// What two portions of an item's part weigh in their sum (x, y), and its reference.  -inf: the row has seen nothing.
__device__ __forceinline__ float3 weights_of(const float2& held, const float2& now) {
    const float top = fmaxf(held.x, now.x), use = top == -CUDART_INF_F ? 0.f : top;
    return make_float3(exp2_fast(held.x - use), exp2_fast(now.x - use), top);
}
// A portion's results `now` join those before it in `held`; of an item's last portion they go out.  By the four warps of a group: a thread has a channel of the rows first .. first + 15 and 32
// further on.  The weights in `held` change behind it (add_weights), when all have read them.  Out of line: one in 65536 keys needs it.
template <int ROWS, int D>
__device__ __noinline__ void add_portion(const TreeArgs* a, const Tile* d, float* held, const float* now, int first, int quarter) {
    const int channel = quarter * 32 + (threadIdx.x & 31);
    const bool out = d->begins && d->ends && !d->more;
    const RowBlock rows = row_block(*a, d->rb * ROWS);
    if (channel >= D) return;
#pragma unroll 1
    for (int e = 0; e < 32; ++e) {
        const int r = first + e + (e & 16);
        if (r >= d->item_rows) return;
        const float2 h = *reinterpret_cast<const float2*>(held + ROWS * D + 2 * r), n = *reinterpret_cast<const float2*>(now + ROWS * D + 2 * r);
        const float3 w = weights_of(h, n);
        const float x = fmaf(held[r * D + channel], w.x, now[r * D + channel] * w.y);
        if (out) {
            const float sum = fmaf(h.y, w.x, n.y * w.y);
            const RowOut ro = row_out(*a, d->row0, d->n_rows, d->kvh, row_of(*a, rows, r), D);
            if (ro.o) ro.o[channel] = __float2bfloat16_rn(ro.on && sum != 0.f ? __fdividef(x, sum) : 0.f);
        } else {
            held[r * D + channel] = x;
        }
    }
}
// by one warp, a row a lane
template <int ROWS, int D>
__device__ __noinline__ void add_weights(float* held, const float* now, int first) {
    const int r = first + (threadIdx.x & 31) + (threadIdx.x & 16);
    float2* h = reinterpret_cast<float2*>(held + ROWS * D + 2 * r);
    const float2 n = *reinterpret_cast<const float2*>(now + ROWS * D + 2 * r);
    const float3 w = weights_of(*h, n);
    *h = make_float2(w.z, fmaf(h->y, w.x, n.y * w.y));
}

// A warp's block of keys in bf16: the form of the kernel's loop for fp16.
template <int D, int G>
__device__ __noinline__ void wide_keys_of(uint32_t codes, uint32_t words, uint32_t row, int kr, int kc) {
    constexpr int kNS = D / G;
#pragma unroll 1
    for (int x = 0; x < D / 32; ++x) {          // channels 32 x + 8 kc ..
        const uint32_t at = codes + (x >> 1) * 512 + (kr * 4 + kc) * 16 + (x & 1) * 8, lo = lds32(at), hi = lds32(at + 4), i = 32 * x / G;
        const uint32_t w0 = lds32(words + (kr * kNS + i) * 4), w1 = lds32(words + ((kr + 8) * kNS + i) * 4), to = row + (x >> 1) * kHalf + (((4 * (x & 1) + kc) ^ kr) << 4);
        const uint32_t s0 = __byte_perm(w0, 0, 0x1010), m0 = __byte_perm(w0, 0, 0x3232), s1 = __byte_perm(w1, 0, 0x1010), m1 = __byte_perm(w1, 0, 0x3232);
        sts128(to, unpack_two(lo, s0, m0), unpack_two(lo >> 4, s0, m0), unpack_two(hi, s0, m0), unpack_two(hi >> 4, s0, m0));
        sts128(to + 8 * 128, unpack_two(lo >> 8, s1, m1), unpack_two(lo >> 12, s1, m1), unpack_two(hi >> 8, s1, m1), unpack_two(hi >> 12, s1, m1));
    }
}

// A warp's block of values in bf16: the form of the kernel's loop for fp16.
template <int D, int G>
__device__ __noinline__ void wide_values(uint32_t codes, uint32_t words, uint32_t row) {
    constexpr int kNS = D / G;
    const int lane = threadIdx.x & 31, t = lane & 3, token = (lane & 7) + 8 * (lane >> 4);
    row += token * 128;
#pragma unroll 1
    for (int x = 0; x < D / 16; ++x) {          // channels 64 (x / 4) + 32 (x / 2 % 2) + 4 g + 2 (x % 2) ..
        const int c = x >> 2, e = x & 3;
        const uint32_t at = words + (2 * t * kNS + (64 * c + 32 * (e >> 1)) / G) * 4, v = lds32(codes + c * 512 + lane * 16 + 4 * e);
        const uint32_t p0 = lds32(at), p1 = lds32(at + kNS * 4), p2 = lds32(at + 8 * kNS * 4), p3 = lds32(at + 9 * kNS * 4);
        const uint32_t s0 = __byte_perm(p0, p1, 0x5410), m0 = __byte_perm(p0, p1, 0x7632), s1 = __byte_perm(p2, p3, 0x5410), m1 = __byte_perm(p2, p3, 0x7632);
        const int piece = (e >> 1) * 4 + 2 * (e & 1) + ((lane >> 3) & 1);
        store_transposed(row + c * kHalf + ((piece ^ (token & 7)) << 4), unpack_two(v, s0, m0), unpack_two(v >> 4, s0, m0), unpack_two(v >> 8, s1, m1), unpack_two(v >> 12, s1, m1));
    }
}

// LONG: a CTA's part of an item may be longer than a portion.  (A form of its own: the call that joins portions, which few need, costs the softmax's warps 2 to 15 %.)
template <int D, int G, int NB, bool LONG>
__global__ void __launch_bounds__(32 * kWarps, 1) attn_tree_kernel(const __grid_constant__ TreeArgs a) {
    using L = Layout<D, G, NB>;
    constexpr int kRows = L::kRows, kNS = L::kNS, kSB = L::kSB, kRing = L::kRing;
    extern __shared__ uint8_t smem_raw[];
    __shared__ Shared sh;
    __shared__ long long part[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t sm = smem_u32(base);
    volatile int* abort_flag = &sh.abort;
    auto bar = [&](const uint64_t& b) { return smem_u32(&b); };
    if (tid == 0) {
        for (int i = 0; i < kRing; ++i) {
            mbar_init(bar(sh.ring_full[i]), 1);
            mbar_init(bar(sh.ring_empty[i]), kUnpackWarps);
        }
        mbar_init(bar(sh.k_full), kUnpackWarps);
        mbar_init(bar(sh.k_free), 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(sh.v_full[i]), kUnpackWarps);
            mbar_init(bar(sh.v_free[i]), 1);
            mbar_init(bar(sh.s_full[i]), 1);
            mbar_init(bar(sh.s_free[i]), NB == 1 ? kSoftWarps / 2 : kSoftWarps);
            mbar_init(bar(sh.p_full[i]), kSoftWarps / 2);
            mbar_init(bar(sh.read[i]), kSoftWarps / 2);
            mbar_init(bar(sh.pv_done[i]), 1);
        }
        for (int i = 0; i < kGroups; ++i) mbar_init(bar(sh.meet[i]), 4);
        mbar_init(bar(sh.q_meet), kUnpackWarps);
        sh.abort = 0;
        sh.n_tiles = 0x7fffffff;
        fence_barrier_init();
    }
    if (tid < 256) sh.spoilt[tid] = 0;
    for (int i = tid; i < (kOnes + kOnesWide) / 4; i += 32 * kWarps) reinterpret_cast<uint32_t*>(base + L::kOnesAt)[i] = i < kOnes / 4 ? 0x3C003C00u : 0x3F803F80u;
    fence_proxy_async_smem();

    grid_dep_wait();
    // (Tensor memory is taken after the kernel before has ended and before the next may come: no two wait for each other's.)
    if (warp == kScoreWarp) {
        tmem_alloc(smem_u32(&sh.tmem), L::kCols);
        tmem_relinquish();
    }
    prefetch_l2(a.mask_bits, static_cast<size_t>(a.q.rows) * a.words * 4);
    prefetch_l2(a.tree, static_cast<size_t>(a.q.rows) * a.tree_words * 4);
    prefetch_l2(a.q.page_table, static_cast<size_t>(a.q.n_seqs) * a.q.max_pages * 4);
    prefetch_l2(a.qm, (static_cast<size_t>(a.q.rows - 1) * a.qs + a.n_q * D) * 2);
    const Plan plan = plan_at(a.plan ? a.plan : base + L::kPlan, a.q.n_seqs, a.plan_words);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    grid_dep_launch();     // the joining kernel may take its place as soon as CTAs end; it waits for all of them
    if (!a.plan) make_plan<kRows>(a, plan, part, gridDim.x, blockIdx.x == 0);
    const uint32_t tmem = sh.tmem;

    const long long total = plan.offsets[a.q.n_seqs];
    const int same = *plan.same, cta = blockIdx.x;
    // a tile's worth of units a CTA at least
    const int ctas = same ? static_cast<int>(total) / same : static_cast<int>(min(static_cast<long long>(gridDim.x), (total + kTile - 1) / kTile));
    long long u0 = 0, u1 = 0;
    if (cta < ctas) {
        const long long share = total / ctas;
        const int more = static_cast<int>(total - share * ctas);
        u0 = share * cta + min(cta, more);
        u1 = u0 + share + (cta < more ? 1 : 0);
    }
    int* meta = a.meta + cta * 2 * kMeta;
    float* parts = a.parts + static_cast<size_t>(cta) * 2 * slot_floats(kRows, D);

    if (u0 < u1) {         // (uniform in the CTA)
        if (warp == kLoadWarp) {
            const Cursor k = locate(a, plan, u0, static_cast<int>(min(u1 - u0, 0x7fffffffLL)));
            if (lane == 0) sh.start = k;
        }
        __syncthreads();
    }
    int open = 0;          // which of the two partial results this CTA leaves; of the loading warp
    if (u0 < u1 && sh.start.blk < sh.start.end) {
        if (warp < kUnpackWarps) {
            // ------------------------------------------------------------------------ codes to bf16 tiles
            const int kr = ((lane >> 2) & 1) * 4 + (lane >> 3), kc = lane & 3;     // key (and key + 8), 8-channel piece: no bank twice in a store
            const int t = lane & 3;
            bool ok = true;
            int items = 0;
            bool wide_keys = false;
            for (int n = 0;; ++n) {
                const int st = n % kRing;
                if (!(ok = mbar_wait_asleep_warp(bar(sh.ring_full[st]), (n / kRing) & 1, a.wait_ns, abort_flag))) break;
                const Tile& d = sh.tiles[n % kDescs];
                const bool here = warp < d.nb && ((d.present >> warp) & 1u);
                const uint32_t codes = sm + L::kCodes + st * L::kStage + warp * kSB, words = codes + 16 * D;
                if (d.first) {
                    // ---- queries in fp16 where each eight neighbours are zeros or have their largest between 2^-9 (so that what falls below the type's normal
                    // numbers is 2^-16 of it) and 2^14; one that is not leaves the item's queries and keys in bf16
                    const RowBlock rows = row_block(a, d.rb * kRows);
                    constexpr int kRowLanes = D / 8, kStep = 32 * kUnpackWarps / kRowLanes;      // a thread has 16 bytes of every kStep-th row
                    const int c = tid % kRowLanes, r0 = tid / kRowLanes;
                    uint4 v[kRows / kStep];
                    bool odd = false;
#pragma unroll
                    for (int i = 0; i < kRows / kStep; ++i) {
                        const Row w = row_of(a, rows, r0 + i * kStep);
                        v[i] = make_uint4(0, 0, 0, 0);
                        if (w.tok < d.n_rows)
                            v[i] = *reinterpret_cast<const uint4*>(a.qm + static_cast<long long>(d.row0 + w.tok) * a.qs + (d.kvh * a.share + w.sub) * D + 8 * c);
                    }
#pragma unroll
                    for (int i = 0; i < kRows / kStep; ++i) {
                        const uint32_t top = largest_bits(v[i]);
                        odd |= top != 0 && top - 0x3B00u > 0x4680u - 0x3B00u;
                    }
                    odd = __any_sync(0xffffffffu, odd);
                    if (lane == 0) {
                        sh.q_wide[d.item & 3][warp] = odd;
                        mbar_arrive(bar(sh.q_meet));
                    }
                    if (!(ok = mbar_wait_asleep_warp(bar(sh.q_meet), items++ & 1, a.wait_ns, abort_flag))) break;
                    const uint2 odds = *reinterpret_cast<const uint2*>(sh.q_wide[d.item & 3]);
                    wide_keys = (odds.x | odds.y) != 0;
                    // the scores of the tile before have been made: Q may change
                    if (n > 0 && !(ok = mbar_wait_asleep_warp(bar(sh.k_free), (n - 1) & 1, a.wait_ns, abort_flag))) break;
#pragma unroll
                    for (int i = 0; i < kRows / kStep; ++i) {
                        const int r = r0 + i * kStep;
                        if (!wide_keys) v[i] = make_uint4(to_half(v[i].x), to_half(v[i].y), to_half(v[i].z), to_half(v[i].w));
                        sts128(sm + L::kQ + (c >> 3) * (kRows * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4), v[i].x, v[i].y, v[i].z, v[i].w);
                    }
                }
                // ---- the sub-groups' words become fp16, a word a lane
                bool half = true;
                {
                    uint32_t kw[(kNS + 1) / 2], vw[(kNS + 1) / 2];
                    bool fits = !wide_keys;
#pragma unroll
                    for (int i = 0; i < (kNS + 1) / 2; ++i) {
                        const uint32_t at = words + 4 * (32 * i + (kNS > 1 ? lane : lane & 15));
                        kw[i] = lds32(at);
                        vw[i] = lds32(at + 64 * kNS);
                        if (d.masked) {
                            // keys that are not there count as zeros, and so do sub-groups of new tokens' values that are not finite, which are noted
                            const int r = (32 * i + lane) / kNS & 15, key = (d.blk + warp) * 16 + r;
                            const bool is = here && key < d.len, bad = is && key >= d.len - d.n_rows && not_finite(vw[i]);
                            if (!is) kw[i] = 0;
                            if (!is || bad) vw[i] = 0;
                            const uint32_t bits = __ballot_sync(0xffffffffu, bad);
                            if (lane % kNS == 0) sh.odd[n & 3][warp * 16 + r] = (bits >> lane) & ((1u << kNS) - 1u);
                        }
                        fits = fits && fits_half(kw[i], kLeastKey) && fits_half(vw[i], kLeastValue);
                    }
                    if (__all_sync(0xffffffffu, fits)) {
#pragma unroll
                        for (int i = 0; i < (kNS + 1) / 2; ++i) {
                            const uint32_t at = words + 4 * (32 * i + (kNS > 1 ? lane : lane & 15));
                            sts32(at, to_half(kw[i]));
                            sts32(at + 64 * kNS, to_half(vw[i]));
                        }
                        if (lane < 16) sh.key_by[n & 3][warp * 16 + lane] = a.scale_log2e;
                    } else {
                        if (d.masked) {
#pragma unroll
                            for (int i = 0; i < (kNS + 1) / 2; ++i) {
                                const uint32_t at = words + 4 * (32 * i + (kNS > 1 ? lane : lane & 15));
                                sts32(at, kw[i]);
                                sts32(at + 64 * kNS, vw[i]);
                            }
                            __syncwarp();
                        }
                        half = odd_words<kNS>(words, sh.key_by[n & 3] + warp * 16, wide_keys, a.scale_log2e);
                    }
                    __syncwarp();
                }
                // (K may change)
                if (n > 0 && !d.first && !(ok = mbar_wait_asleep_warp(bar(sh.k_free), (n - 1) & 1, a.wait_ns, abort_flag))) break;
                if (here && wide_keys) wide_keys_of<D, G>(codes, words, sm + L::kK + (warp * 16 + kr) * 128, kr, kc);
                if (here && !wide_keys) {
                    const uint32_t row = sm + L::kK + (warp * 16 + kr) * 128;
#pragma unroll 1
                    for (int c = 0; c < D / 64; ++c) {
                        const uint4 v = lds128(codes + c * 512 + (kr * 4 + kc) * 16);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {                               // channels 64 c + 32 h + 8 kc ..
                            const int i = (64 * c + 32 * h) / G;
                            const uint32_t w0 = lds32(words + (kr * kNS + i) * 4), w1 = lds32(words + ((kr + 8) * kNS + i) * 4);
                            const uint32_t s0 = __byte_perm(w0, 0, 0x1010), m0 = __byte_perm(w0, 0, 0x3232), s1 = __byte_perm(w1, 0, 0x1010), m1 = __byte_perm(w1, 0, 0x3232);
                            const uint32_t t0 = sixteenth(s0), t1 = sixteenth(s1);
                            const uint32_t x = h ? v.z : v.x, y = h ? v.w : v.y;
                            const uint32_t at = row + c * kHalf + (((4 * h + kc) ^ kr) << 4);
                            sts128(at, unpack_half<false>(x, s0, m0), unpack_half<true>(x, t0, m0), unpack_half<false>(y, s0, m0), unpack_half<true>(y, t0, m0));
                            sts128(at + 8 * 128, unpack_half<false>(x >> 8, s1, m1), unpack_half<true>(x >> 8, t1, m1), unpack_half<false>(y >> 8, s1, m1),
                                   unpack_half<true>(y >> 8, t1, m1));
                        }
                    }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    sh.wide[n & 3][warp] = !half;
                    mbar_arrive(bar(sh.k_full));
                }
                __syncwarp();      // (whole-warp instructions behind code for some lanes: the lanes meet first, here and below)
                // ---- values
                if (n >= 2 && !(ok = mbar_wait_asleep_warp(bar(sh.v_free[n & 1]), ((n >> 1) & 1) ^ 1, a.wait_ns, abort_flag))) break;
                {
                    const int token = (lane & 7) + 8 * (lane >> 4);                 // whose row this lane's address is, and which nibble
                    const uint32_t row = sm + L::kV + (n & 1) * L::kTileBytes + (warp * 16 + token) * 128, params = words + 64 * kNS + 2 * t * kNS * 4;
                    if (half) {
#pragma unroll 1
                        for (int c = 0; c < D / 64; ++c) {
                            const uint4 v = lds128(codes + 8 * D + c * 512 + lane * 16);
                            uint32_t s0 = 0, m0 = 0, s1 = 0, m1 = 0, t0 = 0, t1 = 0;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {                               // channels 64 c + 32 (e / 2) + 4 g + 2 (e % 2) ..
                                if (e == 0 || (e == 2 && G == 32)) {                    // tokens 2t, 2t + 1, 2t + 8, 2t + 9
                                    const uint32_t at = params + (64 * c + 32 * (e >> 1)) / G * 4;
                                    const uint32_t p0 = lds32(at), p1 = lds32(at + kNS * 4), p2 = lds32(at + 8 * kNS * 4), p3 = lds32(at + 9 * kNS * 4);
                                    s0 = __byte_perm(p0, p1, 0x5410), m0 = __byte_perm(p0, p1, 0x7632);
                                    s1 = __byte_perm(p2, p3, 0x5410), m1 = __byte_perm(p2, p3, 0x7632);
                                    t0 = sixteenth(s0), t1 = sixteenth(s1);
                                }
                                const uint32_t x = e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w;
                                const int piece = (e >> 1) * 4 + 2 * (e & 1) + ((lane >> 3) & 1);
                                store_transposed(row + c * kHalf + ((piece ^ (token & 7)) << 4), unpack_half<false>(x, s0, m0), unpack_half<true>(x, t0, m0),
                                                 unpack_half<false>(x >> 8, s1, m1), unpack_half<true>(x >> 8, t1, m1));
                            }
                        }
                    } else {
                        wide_values<D, G>(codes + 8 * D, words + 64 * kNS, sm + L::kV + (n & 1) * L::kTileBytes + warp * 16 * 128);
                    }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(bar(sh.v_full[n & 1]));
                }
                if (d.final) break;
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(sh.ring_empty[st]));     // (the tile's description may go with it)
            }
            if (!ok && lane == 0) atomicExch(a.timeout, WIDE_ERR_TIMEOUT);
        } else if (warp < kUnpackWarps + kSoftWarps) {
            // ------------------------------------------------------------------------ softmax, outputs
            // Two streams of eight warps, each with a buffer of P, outputs and references of its own, that wait for each other only at the end of an
            // item: what one waits for (its product, its four warps' agreement) the other fills, and their steps of different kinds
            // overlap.  With 128 rows a stream has 64 of them; with 64 rows it has every other tile, and the two results are joined at the end.
            // Of its 64 rows a stream's group of four warps has the runs of 16 rows `gi` and gi + 2.
            const int stream = (warp - kUnpackWarps) >> 3, group = (warp - kUnpackWarps) >> 2, gi = group & 1, quarter = warp & 3;
            const int key = quarter * 32 + lane;                                    // of a tile
            const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
            const int row0 = NB == 1 ? 0 : 64 * stream;                             // of this stream in the item
            uint32_t ref_at = 0;             // which of the stream's two references is in use
            int meets = 0, uses = 0, items = 0;
            bool ok = true;
            auto meet = [&]() {              // the four warps of the group
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(sh.meet[group]));
                return mbar_wait_warp(bar(sh.meet[group]), meets++ & 1, a.wait_ns, abort_flag);
            };
            for (int n = NB == 1 ? stream : 0;; n += NB == 1 ? 2 : 1) {
                if (!(ok = mbar_wait_warp(bar(sh.s_full[n & 1]), (n >> 1) & 1, a.wait_ns, abort_flag))) break;
                if (NB == 1 && n >= *static_cast<volatile int*>(&sh.n_tiles)) break;
                tc_fence_after_sync();
                const Tile& d = sh.tiles[n % kDescs];
                const int n_rows = d.item_rows - row0, left = d.left;
                const bool final = d.final;
                if (n_rows > 0) {
                    const bool masked = d.masked, fresh = d.index < (NB == 1 ? 2 : 1);       // the stream's first tile of the item
                    const uint32_t scores = lanes + (n & 1) * kRows + row0;
                    uint32_t bad = 0;
                    if (masked) bad = sh.odd[n & 3][key];          // values that are not finite, of keys that some row may not see
                    const float by = sh.key_by[n & 3][key];
                    const uint2 wides = *reinterpret_cast<const uint2*>(sh.wide[n & 3]);
                    const bool plain = !masked && !(wides.x | wides.y);
                    // the product before has read P, and O holds the stream's tiles up to it
                    if (uses > 0 && !(ok = mbar_wait_warp(bar(sh.pv_done[stream]), (uses - 1) & 1, a.wait_ns, abort_flag))) break;
                    // its outputs of the item before have been read
                    if (NB == 1 && fresh && items > 0 && !(ok = mbar_wait_warp(bar(sh.read[stream]), (items - 1) & 1, a.wait_ns, abort_flag))) break;
                    uint32_t see0 = 0xffffu, see1 = 0xffffu;       // rows of the two runs that see this thread's key
                    if (masked) {
                        see0 = sees_of(&a, &d, row0 + 16 * gi, quarter * 32);
                        see1 = sees_of(&a, &d, row0 + 16 * gi + 32, quarter * 32);
                    }
                    bool again = fresh;
                    while (16 * gi < n_rows) {
                        if (again) {
                            // ---- new references: the largest logits so far; what is summed is scaled
                            tc_fence_after_sync();
#pragma unroll 1
                            for (int c = gi; c < 4; c += 2) {
                                const uint32_t see = c == gi ? see0 : see1;
                                uint32_t s[16];
                                float x[16];
                                tmem_ld_32x16(scores + 16 * c, s);
                                tmem_ld_wait();
#pragma unroll
                                for (int e = 0; e < 16; ++e) x[e] = (see >> e) & 1u ? __uint_as_float(s[e]) * by : -CUDART_INF_F;
                                const float top = largest_across_lanes(x, lane);
                                if (!(lane & 1)) sh.most[quarter][64 * stream + 16 * c + (lane >> 1)] = top;
                                __syncwarp();
                            }
                            if (!(ok = meet())) break;
#pragma unroll 1
                            for (int c = gi; c < 4; c += 2) {
                                const int r = 64 * stream + 16 * c + (lane & 15);
                                const float old = fresh ? -CUDART_INF_F : -sh.minus_ref[ref_at][r];
                                float now = fmaxf(fmaxf(fmaxf(sh.most[0][r], sh.most[1][r]), fmaxf(sh.most[2][r], sh.most[3][r])) - kHigh, old);
                                now = fmaxf(now, -kNothing);              // of a row that has seen nothing: below every logit
                                if (lane < 16) sh.minus_ref[ref_at ^ 1][r] = -now;         // (every warp of the group writes the same)
                                __syncwarp();
                                const float alpha = exp2_fast(old - now);
#pragma unroll 1
                                for (uint32_t at = L::kO; !fresh && at <= L::kSum; at += L::kSum - L::kO) {
                                    uint32_t o[16];
                                    tmem_ld_32x16(lanes + at + 64 * stream + 16 * c, o);
                                    tmem_ld_wait();
#pragma unroll
                                    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * __shfl_sync(0xffffffffu, alpha, e));
                                    tmem_st_32x16(lanes + at + 64 * stream + 16 * c, o);
                                }
                            }
                            tmem_st_wait();
                            __syncwarp();
                            ref_at ^= 1u;
                        }
                        // ---- P, and whether a logit passed its reference (the second run may have no row, and is worked out all the same)
                        const float* ref = sh.minus_ref[ref_at] + 64 * stream;
                        float most = -CUDART_INF_F;
                        auto probabilities = [&](auto is_plain) {
                            constexpr bool kPlain = decltype(is_plain)::value;
#pragma unroll 1
                            for (int c = gi; c < 4; c += 2) {
                                uint32_t s[16];
                                float x[16];
                                tmem_ld_32x16(scores + 16 * c, s);
                                tmem_ld_wait();
#pragma unroll
                                for (int e = 0; e < 16; e += 4) {
                                    const float4 r = *reinterpret_cast<const float4*>(ref + 16 * c + e);
                                    x[e] = fmaf(__uint_as_float(s[e]), by, r.x);
                                    x[e + 1] = fmaf(__uint_as_float(s[e + 1]), by, r.y);
                                    x[e + 2] = fmaf(__uint_as_float(s[e + 2]), by, r.z);
                                    x[e + 3] = fmaf(__uint_as_float(s[e + 3]), by, r.w);
                                }
                                if (!kPlain && masked) {
                                    const uint32_t see = c == gi ? see0 : see1;
#pragma unroll
                                    for (int e = 0; e < 16; ++e) x[e] = (see >> e) & 1u ? x[e] : -CUDART_INF_F;
                                    if (bad)
#pragma unroll 1
                                        for (int e = 0; e < 16; ++e)
                                            if ((see >> e) & 1u) atomicOr(&sh.spoilt[L::spoilt_at(d.item, row0 + 16 * c + e)], bad);
                                }
                                float top[4] = {most, x[0], x[1], x[2]};
#pragma unroll
                                for (int e = 3; e < 16; ++e) top[e & 3] = fmaxf(top[e & 3], x[e]);
                                most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                                uint32_t p[8];
#pragma unroll
                                for (int e = 0; e < 16; ++e) x[e] = exp2_fast(x[e]);
#pragma unroll
                                for (int e = 0; e < 8; ++e) p[e] = half_pair(x[2 * e], x[2 * e + 1]);
                                if (!kPlain && sh.wide[n & 3][key >> 4]) {
#pragma unroll
                                    for (int e = 0; e < 8; ++e) p[e] = as_word(__floats2bfloat162_rn(x[2 * e], x[2 * e + 1]));
                                }
                                const uint32_t row = sm + L::kP + stream * kHalf + key * 128;
                                sts128(row + (((2 * c) ^ (key & 7)) << 4), p[0], p[1], p[2], p[3]);
                                sts128(row + (((2 * c + 1) ^ (key & 7)) << 4), p[4], p[5], p[6], p[7]);
                                if (!kPlain) __syncwarp();
                            }
                        };
                        if (plain) probabilities(std::true_type{});
                        else probabilities(std::false_type{});
                        if (again) break;
                        const bool change = __any_sync(0xffffffffu, most > kSlack + kHigh);
                        int* flag = sh.flag[uses & 3][group];
                        if (lane == 0) flag[quarter] = change;
                        if (!(ok = meet())) break;
                        const int4 flags = *reinterpret_cast<const int4*>(flag);
                        if (!(flags.x | flags.y | flags.z | flags.w)) break;
                        again = true;
                    }
                    if (!ok) break;
                    const bool mine = left == 0, done = left <= (NB == 1 ? 1 : 0);       // whether this stream writes the item, has its last tile of it
                    if (done && lane == 0 && quarter == 0) sh.ref_at[group] = ref_at;
                    fence_proxy_async_smem();
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(bar(sh.p_full[stream]));
                        mbar_arrive(bar(sh.s_free[n & 1]));
                    }
                    ++uses;
                    if (done) ++items;
                    if (mine) {
                        // ---- end of the item or of the piece
                        const bool two = NB == 1 && d.index > 0;       // the other stream has a part of it
                        const int other = stream ^ 1;
                        if (!(ok = mbar_wait_warp(bar(sh.pv_done[stream]), (uses - 1) & 1, a.wait_ns, abort_flag))) break;
                        // (tile n - 1 was the other's ((n - 1) / 2 + 1)-th)
                        if (two && !(ok = mbar_wait_warp(bar(sh.pv_done[other]), ((n - 1) >> 1) & 1, a.wait_ns, abort_flag))) break;
                        tc_fence_after_sync();
                        // lane (c, a, j, g) of O has channel 64 c + 32 a + 4 g + j
                        const int at = quarter * 32 + lane, channel = (at & ~31) + 4 * (lane & 7) + (lane >> 3);
                        const bool goes_on = LONG && d.goes_on, whole = d.begins && d.ends && !(LONG && d.more) && !goes_on;
                        float *slot = parts + (d.begins ? slot_floats(kRows, D) : 0), *dst = goes_on ? a.heads + static_cast<size_t>(cta) * slot_floats(kRows, D) : slot;
                        const RowBlock rows = row_block(a, d.rb * kRows);
#pragma unroll 1
                        for (int c = gi; 16 * c < n_rows && c < 4; c += 2) {
                            // where the run's rows go, a row a lane: index of (row, head) in o, -1 for none; whether it is on; what its two parts weigh
                            const int r = row0 + 16 * c + (lane & 15);
                            const Row w = row_of(a, rows, r);
                            const int h = d.kvh * a.share + w.sub, row = d.row0 + w.tok;
                            const int place = w.tok < d.n_rows ? row * a.n_q + h : -1;
                            const bool on = place >= 0 && (!a.mask_bits || wide_mask_bit(a.mask_bits, a.words, row, h / a.hpg));
                            const uint32_t on_bits = __ballot_sync(0xffffffffu, on), spoilt = sh.spoilt[L::spoilt_at(d.item, r)];
                            float top = -sh.minus_ref[ref_at][64 * stream + 16 * c + (lane & 15)], by = 1.f, by_other = 0.f;
                            if (two) {
                                const float that = -sh.minus_ref[sh.ref_at[2 * other + gi]][64 * other + 16 * c + (lane & 15)], most = fmaxf(top, that);
                                by = exp2_fast(top - most);
                                by_other = exp2_fast(that - most);
                                top = most;
                            }
#pragma unroll 1
                            for (int e0 = 0; e0 < 16; e0 += 4) {
                                uint32_t o[4], l[4], o2[4], l2[4];     // outputs, sums of P (the same in all lanes)
                                tmem_ld_32x4(lanes + L::kO + 64 * stream + 16 * c + e0, o);
                                tmem_ld_32x4(lanes + L::kSum + 64 * stream + 16 * c + e0, l);
                                if (two) {
                                    tmem_ld_32x4(lanes + L::kO + 64 * other + 16 * c + e0, o2);
                                    tmem_ld_32x4(lanes + L::kSum + 64 * other + 16 * c + e0, l2);
                                }
                                tmem_ld_wait();
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const int to = __shfl_sync(0xffffffffu, place, e0 + e);
                                    const uint32_t bad_groups = __shfl_sync(0xffffffffu, spoilt, e0 + e);
                                    const float m = __shfl_sync(0xffffffffu, top, e0 + e);
                                    float x = __uint_as_float(o[e]), sum = __uint_as_float(l[e]);
                                    if (two) {
                                        const float f = __shfl_sync(0xffffffffu, by, e0 + e), f2 = __shfl_sync(0xffffffffu, by_other, e0 + e);
                                        x = fmaf(__uint_as_float(o2[e]), f2, x * f);
                                        sum = fmaf(__uint_as_float(l2[e]), f2, sum * f);
                                    }
                                    if ((bad_groups >> (channel / G)) & 1u) x = CUDART_NAN_F;
                                    if (at >= D || to < 0) continue;
                                    if (whole) {
                                        a.o[static_cast<size_t>(to) * D + channel] = __float2bfloat16_rn((on_bits >> (e0 + e)) & 1u && sum != 0.f ? __fdividef(x, sum) : 0.f);
                                    } else {
                                        const int rr = row0 + 16 * c + e0 + e;
                                        dst[rr * D + channel] = x;
                                        // (a row that has seen nothing has no weight among its other pieces)
                                        if (at == 0) *reinterpret_cast<float2*>(dst + kRows * D + 2 * rr) = make_float2(sum == 0.f ? -CUDART_INF_F : m, sum);
                                    }
                                }
                                __syncwarp();
                            }
                        }
                        if (!(ok = meet())) break;       // all have read what is cleared now
                        for (int c = gi; c < 4; c += 2)
                            if (quarter == 0 && lane < 16) sh.spoilt[L::spoilt_at(d.item, row0 + 16 * c + lane)] = 0;
                        if constexpr (LONG) {
                            if (goes_on) {
                                add_portion<kRows, D>(&a, &d, slot, dst, row0 + 16 * gi, quarter);
                                if (!(ok = meet())) break;
                                if (quarter == 0) add_weights<kRows, D>(slot, dst, row0 + 16 * gi);
                            }
                        }
                        tc_fence_before_sync();
                        __syncwarp();
                        if (NB == 1 && lane == 0) {
                            mbar_arrive(bar(sh.read[stream]));
                            if (two) mbar_arrive(bar(sh.read[other]));
                        }
                    }
                } else {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(sh.s_free[n & 1]));
                }
                if (final) break;
            }
            if (!ok && lane == 0) atomicExch(a.timeout, WIDE_ERR_TIMEOUT);
        } else if (warp == kLoadWarp) {
            // ------------------------------------------------------------------------ items, codes
            Cursor k = sh.start;
            const int sub_shift = a.c.page_shift - 4, sub_mask = (1 << sub_shift) - 1;
            bool ok = true, first = true;
            int index = 0, item = 0, portion = 0;
            int first_blk = k.blk, pt_first = -1000000, pt = -1, pt_next = -1;
            for (int n = 0;; ++n) {
                const int st = n % kRing, nb = min(kTile, k.end - k.blk), from = k.blk >> sub_shift, to = (k.blk + nb - 1) >> sub_shift;
                // page numbers: 32 at hand, the next 32 on their way
                auto pages_from = [&](int p) { return p + lane < a.q.max_pages ? a.q.page_table[static_cast<size_t>(k.seq) * a.q.max_pages + p + lane] : -1; };
                if (from < pt_first || to >= pt_first + 64) {
                    pt_first = from;
                    pt = pages_from(pt_first);
                    pt_next = pages_from(pt_first + 32);
                } else if (from >= pt_first + 32) {
                    pt_first += 32;
                    pt = pt_next;
                    pt_next = pages_from(pt_first + 32);
                }
                const int want = ((k.blk + min(lane, nb - 1)) >> sub_shift) - pt_first;
                int page = __shfl_sync(0xffffffffu, pt, want & 31);
                if (to >= pt_first + 32) {
                    const int far = __shfl_sync(0xffffffffu, pt_next, want & 31);
                    if (want >= 32) page = far;
                }
                const bool there = lane < nb && static_cast<unsigned>(page) < static_cast<unsigned>(a.c.n_pages);
                const uint32_t present = __ballot_sync(0xffffffffu, there);
                const int4 info = plan.seqs[k.seq];
                Cursor next = k;            // what comes behind this tile
                next.blk += nb;
                const bool last = next.blk >= next.end, begins = first_blk == 0, ends = k.end == k.n_blk;
                if (last && next.left > 0) next_item(a, plan, next);
                const bool final = last && next.blk >= next.end, closes = last || (LONG && index + 1 == kPortion);
                if (n >= kRing && !(ok = mbar_wait_asleep_warp(bar(sh.ring_empty[st]), ((n / kRing) & 1) ^ 1, a.wait_ns, abort_flag))) break;
                if (lane == 0) {
                    if (present != (1u << nb) - 1u) atomicExch(a.status, WIDE_ERR_BAD_INDEX);
                    Tile& d = sh.tiles[n % kDescs];
                    d.blk = k.blk, d.nb = nb, d.present = present, d.first = first;
                    d.masked = present != (1u << kTile) - 1u || (k.blk + nb) * 16 > info.z - info.y;
                    d.kvh = k.kvh, d.rb = k.rb, d.row0 = info.x, d.n_rows = info.y, d.len = info.z;
                    d.item_rows = min(kRows, info.y * a.share - k.rb * kRows), d.rows_a_block = kRows;
                    d.begins = begins, d.ends = ends, d.final = final;
                    if (LONG) d.goes_on = portion > 0, d.more = !last;
                    d.index = min(index, 2), d.item = item, d.left = closes ? 0 : k.end - (k.blk + nb) <= kTile || (LONG && index + 2 == kPortion) ? 1 : 2;
                    mbar_arrive_expect_tx(bar(sh.ring_full[st]), __popc(present) * kSB);
                }
                __syncwarp();
                if (there)
                    bulk_load(sm + L::kCodes + st * L::kStage + lane * kSB,
                              a.c.pages + static_cast<size_t>(page) * a.page_bytes + ((static_cast<size_t>(k.kvh) << sub_shift) + ((k.blk + lane) & sub_mask)) * kSB, kSB,
                              bar(sh.ring_full[st]));
                if (last && !(begins && ends)) {
                    int* m = meta + (begins ? kMeta : 0);
                    if (lane == 0) {
                        m[0] = ends ? 2 : 1;
                        m[1] = info.x;
                        m[2] = info.y;
                        m[3] = k.kvh;
                        m[4] = k.rb;
                    }
                    open |= begins ? 2 : 1;
                }
                if (final) break;
                first = closes;
                ++index;
                if (closes) {
                    index = 0;
                    ++item;
                    if (LONG) portion = last ? 0 : portion + 1;
                }
                if (last) {
                    if (next.seq != k.seq) pt_first = -1000000;
                    first_blk = next.blk;
                }
                k = next;
            }
            if (!ok && lane == 0) atomicExch(a.timeout, WIDE_ERR_TIMEOUT);
        } else if (warp == kScoreWarp) {
            // ------------------------------------------------------------------------ S^T = K Q^T
            // (The whole warp walks the loop and one lane is elected for each instruction: the operands, which the instruction takes from uniform
            // registers, are then computed there.  By lane 0 alone a product took 100 clocks to issue, twice its own time.)
            bool ok = true;
            for (int n = 0;; ++n) {
                if (!(ok = mbar_wait_asleep_warp(bar(sh.k_full), n & 1, a.wait_ns, abort_flag))) break;
                if (n >= 2 && !(ok = mbar_wait_asleep_warp(bar(sh.s_free[n & 1]), ((n >> 1) & 1) ^ 1, a.wait_ns, abort_flag))) break;
                tc_fence_after_sync();
                const uint64_t kd = umma_desc_sw128(sm + L::kK), qd = umma_desc_sw128(sm + L::kQ);
                const uint2 wides = *reinterpret_cast<const uint2*>(sh.q_wide[sh.tiles[n % kDescs].item & 3]);
                const bool half = !(wides.x | wides.y);
                const uint32_t shape = NB == 2 && sh.tiles[n % kDescs].item_rows <= 64 ? idesc(64, half, false) : idesc(kRows, half, false);
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
                    umma_bf16_elect(tmem + (n & 1) * kRows, kd + (i / 4) * (kHalf >> 4) + 2 * (i % 4), qd + (i / 4) * (kRows * 128 >> 4) + 2 * (i % 4), shape,
                                    i > 0 ? 1u : 0u);
                umma_commit_elect(bar(sh.k_free));
                umma_commit_elect(bar(sh.s_full[n & 1]));
                if (sh.tiles[n % kDescs].final) {
                    if (NB == 1) {      // the stream that waits for the next tile learns that there is none, once it is done with its last one
                        if (n > 0 && !(ok = mbar_wait_asleep_warp(bar(sh.s_free[(n + 1) & 1]), ((n - 1) >> 1) & 1, a.wait_ns, abort_flag))) break;
                        if (lane == 0) {
                            *static_cast<volatile int*>(&sh.n_tiles) = n + 1;
                            mbar_arrive(bar(sh.s_full[(n + 1) & 1]));
                        }
                    }
                    break;
                }
            }
            if (!ok && lane == 0) atomicExch(a.timeout, WIDE_ERR_TIMEOUT);
        } else if (warp == kValueWarp) {
            // ------------------------------------------------------------------------ O^T += V^T P^T
            bool ok = true;
            int uses[2] = {0, 0};
            for (int n = 0; ok; ++n) {
                if (!(ok = mbar_wait_asleep_warp(bar(sh.v_full[n & 1]), (n >> 1) & 1, a.wait_ns, abort_flag))) break;
                // (heads of 64: the upper 64 lanes take whatever lies behind the tile, and nobody reads them)
                const uint64_t vd = desc_mn(sm + L::kV + (n & 1) * L::kTileBytes, kHalf);
                const Tile& d = sh.tiles[n % kDescs];
                const bool fresh = d.index < (NB == 1 ? 2 : 1), final = d.final;
                const int blocks = (d.item_rows + 63) >> 6;
                const uint2 wides = *reinterpret_cast<const uint2*>(sh.wide[n & 3]);
                const uint64_t ones = desc_ones(sm + L::kOnesAt), ones_wide = desc_ones_wide(sm + L::kOnesAt + kOnes);
#pragma unroll 1
                for (int b = 0; b < blocks; ++b) {
                    const int stream = NB == 1 ? n & 1 : b;
                    if (!(ok = mbar_wait_asleep_warp(bar(sh.p_full[stream]), (stream ? uses[1]++ : uses[0]++) & 1, a.wait_ns, abort_flag))) break;
                    tc_fence_after_sync();
                    const uint64_t pd = desc_mn(sm + L::kP + stream * kHalf, kHalf);
                    // and, with ones in V's place, the sums of P over the keys
                    if (!(wides.x | wides.y)) {
#pragma unroll
                        for (int i = 0; i < kKeys / 16; ++i)
                            umma_bf16_elect(tmem + L::kO + 64 * stream, vd + i * (2048 >> 4), pd + i * (2048 >> 4), idesc(64, true, true), fresh && i == 0 ? 0u : 1u);
#pragma unroll
                        for (int i = 0; i < kKeys / 16; ++i)
                            umma_bf16_elect(tmem + L::kSum + 64 * stream, ones, pd + i * (2048 >> 4), idesc(64, true, true), fresh && i == 0 ? 0u : 1u);
                    } else {
#pragma unroll 1
                        for (int i = 0; i < kKeys / 16; ++i) {
                            const bool bf16 = ((i < 4 ? wides.x : wides.y) >> (8 * (i & 3))) & 1u;
                            const uint32_t type = bf16 ? idesc(64, false, true) : idesc(64, true, true), add = fresh && i == 0 ? 0u : 1u;
                            umma_bf16_elect(tmem + L::kO + 64 * stream, vd + i * (2048 >> 4), pd + i * (2048 >> 4), type, add);
                            umma_bf16_elect(tmem + L::kSum + 64 * stream, bf16 ? ones_wide : ones, pd + i * (2048 >> 4), type, add);
                        }
                    }
                    if (b + 1 == blocks) umma_commit_elect(bar(sh.v_free[n & 1]));
                    umma_commit_elect(bar(sh.pv_done[stream]));
                }
                if (final) break;
            }
            if (!ok && lane == 0) atomicExch(a.timeout, WIDE_ERR_TIMEOUT);
        }
        __syncwarp();
    }
    if (warp == kLoadWarp && lane == 0) {
        if (!(open & 1)) meta[0] = 0;
        if (!(open & 2)) meta[kMeta] = 0;
    }
    // rows that no item writes: KV heads that a sequence does not use, sequences that are left out
    for (int s = cta; s < a.q.n_seqs; s += gridDim.x) {
        const int4 i = plan.seqs[s];
        const int per_row = a.n_q * (D / 8);
        for (long long x = tid; x < static_cast<long long>(i.y) * per_row; x += 32 * kWarps) {
            const int r = static_cast<int>(x / per_row), v = static_cast<int>(x - static_cast<long long>(r) * per_row), h = v / (D / 8) / a.share;
            if (!((plan.masks[s * a.plan_words + (h >> 5)] >> (h & 31)) & 1u))
                reinterpret_cast<uint4*>(a.o + static_cast<size_t>(i.x + r) * a.n_q * D)[v] = make_uint4(0, 0, 0, 0);
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) let_copies_land();
    if (warp == kScoreWarp) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, L::kCols);
    }
}

// Items that more than one CTA had a piece of: block (c, .) joins the one that begins in CTA c and goes on in the next.  A warp takes a row: lane
// e reads the maximum and sum of piece e, and every lane its channels of all pieces, eight at a time.
constexpr int kJoinParts = 16;
template <int ROWS, int D>
__global__ void __launch_bounds__(256) attn_tree_join_kernel(const __grid_constant__ TreeArgs a, int ctas) {
    grid_dep_wait();
    const int c = blockIdx.x, lane = threadIdx.x & 31;
    const int* mine = a.meta + (2 * c + 1) * kMeta;
    const int4 meta = *reinterpret_cast<const int4*>(mine);
    const int rb = mine[4];
    int st = c + 1 + lane < ctas ? a.meta[2 * (c + 1 + lane) * kMeta] : 0;
    if (meta.x != 1 || static_cast<unsigned>(meta.w) >= static_cast<unsigned>(a.c.n_kv_heads)) return;
    int n = 1;         // pieces: CTAs c + 1, ... up to the one that ends the item
    for (int k = c + 1;;) {
        const uint32_t stop = __ballot_sync(0xffffffffu, st != 1);
        if (stop) {
            const int at = __ffs(stop) - 1;
            n += at + (__shfl_sync(0xffffffffu, st, at) == 2 ? 1 : 0);
            break;
        }
        n += 32;
        k += 32;
        st = k + lane < ctas ? a.meta[2 * (k + lane) * kMeta] : 0;
    }
    auto piece = [&](int i) -> const float* { return a.parts + static_cast<size_t>(i == 0 ? 2 * c + 1 : 2 * (c + i)) * slot_floats(ROWS, D); };
    constexpr int kEach = D / 32;        // channels of a lane
    const RowBlock rows = row_block(a, rb * ROWS);
    for (int r = (threadIdx.x >> 5) + 8 * blockIdx.y; r < ROWS; r += 8 * kJoinParts) {
        const RowOut ro = row_out(a, meta.y, meta.z, meta.w, row_of(a, rows, r), D);
        if (!ro.o) break;                // (rows behind it do not exist either)
        float m = -CUDART_INF_F, l = 0.f, x[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) x[e] = 0.f;
        for (int e0 = 0; e0 < n; e0 += 32) {
            const int last = min(32, n - e0);
            const float2 ml = lane < last ? *reinterpret_cast<const float2*>(piece(e0 + lane) + ROWS * D + 2 * r) : make_float2(-CUDART_INF_F, 0.f);
            float top = ml.x;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float m_new = fmaxf(m, top), m_use = m_new == -CUDART_INF_F ? 0.f : m_new;
            const float old = exp2_fast(m - m_use), w = exp2_fast(ml.x - m_use);
            float sum = ml.y * w;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            l = fmaf(l, old, sum);
            m = m_new;
#pragma unroll
            for (int e = 0; e < kEach; ++e) x[e] *= old;
            for (int p0 = 0; p0 < last; p0 += 8) {
                float v[8][kEach];
#pragma unroll
                for (int p = 0; p < 8; ++p) {
#pragma unroll
                    for (int e = 0; e < kEach; ++e) v[p][e] = 0.f;
                    if (p0 + p < last) {
                        const float* from = piece(e0 + p0 + p) + r * D + kEach * lane;
#pragma unroll
                        for (int e = 0; e < kEach; e += 2) *reinterpret_cast<float2*>(&v[p][e]) = *reinterpret_cast<const float2*>(from + e);
                    }
                }
#pragma unroll
                for (int p = 0; p < 8; ++p) {
                    const float we = __shfl_sync(0xffffffffu, w, (p0 + p) & 31);
#pragma unroll
                    for (int e = 0; e < kEach; ++e) x[e] = fmaf(v[p][e], we, x[e]);
                }
            }
        }
        const float inv = ro.on && l != 0.f ? 1.f / l : 0.f;
#pragma unroll
        for (int e = 0; e < kEach; e += 2) {
            const __nv_bfloat162 b = inv != 0.f ? __floats2bfloat162_rn(x[e] * inv, x[e + 1] * inv) : __floats2bfloat162_rn(0.f, 0.f);
            *reinterpret_cast<__nv_bfloat162*>(ro.o + kEach * lane + e) = b;
        }
    }
}

struct Work {
    size_t plan, parts, portions, meta, total;
};
Work work_layout() {
    Work w;
    size_t at = 0;
    w.plan = at;
    at += wide_align_up(plan_bytes(WIDE_MAX_SEQS, 8, 8), 256);
    w.parts = at;
    at += wide_align_up(static_cast<size_t>(kMaxCtas) * 2 * slot_floats(128, 128) * 4, 256);
    w.portions = at;
    at += wide_align_up(static_cast<size_t>(kMaxCtas) * slot_floats(128, 128) * 4, 256);
    w.meta = at;
    at += static_cast<size_t>(kMaxCtas) * 2 * kMeta * 4;
    w.total = wide_align_up(at, 256);
    return w;
}

template <int D, int G, int NB, bool LONG>
int launch(wide_ctx* ctx, cudaStream_t s, TreeArgs a, unsigned char* ws, int ctas, bool joins) {
    using L = Layout<D, G, NB>;
    auto kernel = attn_tree_kernel<D, G, NB, LONG>;
    const Work w = work_layout();
    a.heads = reinterpret_cast<float*>(ws + w.portions);
    a.parts = reinterpret_cast<float*>(ws + w.parts);
    a.meta = reinterpret_cast<int*>(ws + w.meta);
    a.plan = nullptr;
    if (plan_bytes(a.q.n_seqs, a.plan_words, a.words) > static_cast<size_t>(L::kPlanRoom)) {
        a.plan = ws + w.plan;
        WideLaunch l(ctx, s, "attn_tree_plan");
        WIDE_CUDA_CHECK(wide_launch_after(ctx, attn_cache_plan_kernel<L::kRows>, dim3(1), dim3(1024), 0, s, a, ctas));
    }
    // once a device; threads that come here together all set the same
    static std::atomic<unsigned> set{0};
    const unsigned bit = ctx->device < 32 ? 1u << ctx->device : 0u;
    if (!(set.load(std::memory_order_relaxed) & bit) || !bit) {
        WIDE_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kSmem));
        set.fetch_or(bit, std::memory_order_relaxed);
    }
    {
        WideLaunch l(ctx, s, "attn_tree");
        WIDE_CUDA_CHECK(wide_launch_after(ctx, kernel, dim3(ctas), dim3(32 * kWarps), L::kSmem, s, a));
    }
    if (joins) {
        WideLaunch l(ctx, s, "attn_tree_join");
        WIDE_CUDA_CHECK(wide_launch_after(ctx, attn_tree_join_kernel<L::kRows, D>, dim3(ctas, kJoinParts), dim3(256), 0, s, a, ctas));
    }
    return WIDE_OK;
}

template <int NB, bool LONG>
int launch_dims(wide_ctx* ctx, cudaStream_t s, const TreeArgs& a, int D, int G, unsigned char* ws, int ctas, bool joins) {
    if (D == 128) {
        if (G == 128) return launch<128, 128, NB, LONG>(ctx, s, a, ws, ctas, joins);
        if (G == 64) return launch<128, 64, NB, LONG>(ctx, s, a, ws, ctas, joins);
        return launch<128, 32, NB, LONG>(ctx, s, a, ws, ctas, joins);
    }
    if (G == 64) return launch<64, 64, NB, LONG>(ctx, s, a, ws, ctas, joins);
    return launch<64, 32, NB, LONG>(ctx, s, a, ws, ctas, joins);
}

template <int NB>
int launch_shape(wide_ctx* ctx, cudaStream_t s, const TreeArgs& a, int D, int G, unsigned char* ws) {
    const int ctas = ctx->sm_count < kMaxCtas ? ctx->sm_count : kMaxCtas;
    // What is known without the lengths: as many items at most, of as many blocks.
    const long long items = static_cast<long long>(a.c.n_kv_heads) * (static_cast<long long>(a.q.rows) * a.share / (64 * NB) + a.q.n_seqs);
    const long long blocks = static_cast<long long>(a.q.max_pages) << (a.c.page_shift - 4);
    // Nothing to join where the plan is certain to give every item a CTA of its own (make_plan).
    const bool joins = items > ctas || blocks > kItemShort;
    // The longest part of an item that a CTA can have: all of it, or the CTA's share of the line.
    const bool portions = blocks > kPortion * kTile && items * (blocks + kItemCost) / ctas >= kPortion * kTile;
    return portions ? launch_dims<NB, true>(ctx, s, a, D, G, ws, ctas, joins) : launch_dims<NB, false>(ctx, s, a, D, G, ws, ctas, joins);
}

}  // namespace

size_t wide_attn_tree_workspace() { return work_layout().total; }

int wide_launch_attn_tree(wide_ctx* ctx, cudaStream_t s, const wide_cache* cache, const wide_seqs* seqs, const void* q, int rows,
                          long long qs, int n_q, int hpg, const uint32_t* mask_bits, const uint32_t* tree_bits, int tree_words, float scale,
                          void* o, void* ws) {
    TreeArgs a{};
    a.c = wide_cache_view(cache);
    a.q = wide_seq_view(seqs, rows);
    a.page_bytes = static_cast<unsigned>(a.c.block_bytes) * static_cast<unsigned>(cache->n_kv_heads) << (a.c.page_shift - 4);
    a.qm = static_cast<const __nv_bfloat16*>(q);
    a.qs = qs;
    a.n_q = n_q;
    a.share = n_q / cache->n_kv_heads;
    a.by_share = a.share > 1 ? static_cast<unsigned>(((1ull << 32) + a.share - 1) / a.share) : 0u;
    a.hpg = hpg;
    a.words = (n_q / hpg + 31) / 32;
    a.most_rows = 32 * tree_words;
    a.mask_bits = mask_bits;
    a.tree = tree_bits;
    a.tree_words = tree_words;
    a.scale_log2e = scale * 1.4426950408889634f;
    a.o = static_cast<__nv_bfloat16*>(o);
    a.status = ctx->d_status + WIDE_STATUS_INDEX;
    a.timeout = ctx->d_status;
    a.wait_ns = ctx->wait_ns;
    a.plan_words = (cache->n_kv_heads + 31) / 32;
    // Query rows of a sequence and KV head, on average (the lengths are on the device): above 64, 128 share a pass over the cache.
    const long long rows_per_head = seqs->row_start ? static_cast<long long>(rows) * a.share / seqs->n_seqs : a.share;
    if (rows_per_head <= 64) return launch_shape<1>(ctx, s, a, cache->head_dim, cache->quant_group, static_cast<unsigned char*>(ws));
    return launch_shape<2>(ctx, s, a, cache->head_dim, cache->quant_group, static_cast<unsigned char*>(ws));
}
