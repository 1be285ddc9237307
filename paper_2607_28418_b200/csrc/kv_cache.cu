// Writing keys and values into the 4-bit paged cache and reading them back (layout and levels: wide.h).
//
// Both kernels move bytes: per value 2 (bf16) in and 0.56 out or the other way round, so HBM is the bound.
// A warp takes one block of the cache, 16 positions of one head, because that is the unit in
// which codes of several tokens share words: with all 16 tokens in hand it stores whole words, and where
// only some of them are new (a decode step: one) it stores the bytes that belong to them.  A lane holds
// 8 neighbouring channels, so a row is read in 16-byte pieces, coalesced, and the extremes of a
// sub-group are 8 values in registers and two to four shuffles.  The token of the block that a lane takes is
// chosen so that the tokens whose codes share a word meet in one lane.
#include <math_constants.h>

#include "cache.cuh"
#include "ptx.cuh"

namespace {

using wptx::add2;
using wptx::fma2;
using wptx::pair;
using wptx::unpair;

constexpr int kWarps = 4;           // of a CTA (8 start and end in larger steps: 8188 tokens written and read back 28.7 us, with four 27.5)

// 8 neighbouring channels as they lie in memory
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = __ldg(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void clear() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    // smallest and largest of LW lanes, NaN if any is: one register holds the minimum and the negated maximum
    template <int LW>
    __device__ __forceinline__ void range(float& lo, float& hi) const {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
        const __nv_bfloat162 a = __hmin2_nan(__hmin2_nan(h[0], h[1]), __hmin2_nan(h[2], h[3]));
        const __nv_bfloat162 b = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
        __nv_bfloat162 both = __halves2bfloat162(__hmin_nan(__low2bfloat16(a), __high2bfloat16(a)), __hneg(__hmax_nan(__low2bfloat16(b), __high2bfloat16(b))));
#pragma unroll
        for (int o = 1; o < LW; o <<= 1) {
            const uint32_t other = __shfl_xor_sync(0xffffffffu, *reinterpret_cast<const uint32_t*>(&both), o);
            both = __hmin2_nan(both, *reinterpret_cast<const __nv_bfloat162*>(&other));
        }
        lo = __low2float(both);
        hi = -__high2float(both);
    }
};
__device__ __forceinline__ float min_nan(float a, float b) {
    float c;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(c) : "f"(a), "f"(b));
    return c;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float c;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(c) : "f"(a), "f"(b));
    return c;
}
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = __ldg(reinterpret_cast<const float4*>(p));
        b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    }
    __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    template <int LW>
    __device__ __forceinline__ void range(float& lo, float& hi) const {
        lo = min_nan(min_nan(min_nan(a.x, a.y), min_nan(a.z, a.w)), min_nan(min_nan(b.x, b.y), min_nan(b.z, b.w)));
        hi = max_nan(max_nan(max_nan(a.x, a.y), max_nan(a.z, a.w)), max_nan(max_nan(b.x, b.y), max_nan(b.z, b.w)));
#pragma unroll
        for (int o = 1; o < LW; o <<= 1) {
            lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
            hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
    }
};

// sign-correct a - b - c for c near a - b: d = a - b rounded, e its exact remainder (two-sum)
__device__ __forceinline__ double exact_gap(double a, double b, double c) {
    const double d = a - b;
    const double bb = d - a;
    const double e = (a - (d - bb)) + ((-b) - bb);
    return (d - c) + e;
}

// Sub-groups that the fast way below leaves out: not finite, all channels alike, magnitudes at which fp32 overflows
// or has few bits left, a minimum whose low bits are out of reach of the borders.  x: parameter word, y: codes.
template <int LW, typename T>
__device__ __noinline__ uint2 quantise8_any(Raw8<T> raw) {
    float lo, hi, x[8];
    raw.template range<LW>(lo, hi);
    raw.get(x);
    lo += 0.f;   // zeros are +0
    hi += 0.f;
    const uint32_t mb = (lo < 0.f ? __float_as_uint(lo) + 0xFFFFu : __float_as_uint(lo)) & 0xFFFF0000u;
    const float m = __uint_as_float(mb);
    if (!(fabsf(m) <= 3.4e38f && hi <= 3.4028234e38f)) return make_uint2(0x7FC07FC0u, 0u);
    const double q = (static_cast<double>(hi) - static_cast<double>(m)) / 15.0;
    uint32_t sb = (__float_as_uint(__double2float_ru(q)) + 0xFFFFu) & 0xFFFF0000u;
    // the quotient is rounded: does the last level, rounded down, reach the maximum?
    if (__fma_rd(15.0, static_cast<double>(__uint_as_float(sb)), static_cast<double>(m)) < static_cast<double>(hi)) sb += 0x10000u;
    const float s = __uint_as_float(sb);
    uint32_t c = 0;
#pragma unroll 1
    for (int i = 0; i < 15 && s > 0.f; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            c += exact_gap(static_cast<double>(x[e]), static_cast<double>(m), (i + 0.5) * static_cast<double>(s)) >= 0.0 ? 1u << (4 * e) : 0u;
    return make_uint2((__float_as_uint(s) >> 16) | mb, c);
}

// two fp32 numbers at once, rounded up
__device__ __forceinline__ unsigned long long fma2_up(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rp.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

// Levels of 8 channels each of two tokens' sub-groups that span LW lanes: code e in bits 4e, the parameter word; false
// where quantise8_any has to do it.
//
// The definition is exact (how many borders m + (i + 1/2) s does x reach), so the same input always gives the
// same code.  What makes that cheap: for a number x and an exact y, x >= y holds iff x >= y rounded UP, and
// y >= x iff y rounded DOWN is, and one fma rounds the exact border once.  So the level is guessed in fp32, rounded to
// an integer by the addition of 2^23 and biased upwards by 2^-19 of itself, which leaves the right level or the one above
// (the error is below 2^-21), and one comparison with the guess's lower border, n s + (m - s / 2), settles it.  Likewise the
// scale, whose last level must reach the maximum.  The kernel is bound by the rate at which instructions issue, so the two
// tokens share them: six a value.
template <typename T>
struct Levels {
    float m, hi, s, mh, rs;
    uint32_t c, mb;
    bool fine;
    template <int LW>
    __device__ __forceinline__ void set(const Raw8<T>& raw) {
        float lo;
        raw.template range<LW>(lo, hi);
        lo += 0.f;   // zeros are +0
        mb = __float_as_uint(lo);
        if (sizeof(T) == 4) mb = (lo < 0.f ? mb + 0xFFFFu : mb) & 0xFFFF0000u;   // bf16 at or below lo
        m = __uint_as_float(mb);
        c = __float_as_uint((hi - m) * (0.999999f / 15.f)) & 0xFFFF0000u;
        c += __fmaf_rd(15.f, __uint_as_float(c), m) < hi ? 0x10000u : 0u;
        c += __fmaf_rd(15.f, __uint_as_float(c), m) < hi ? 0x10000u : 0u;
        s = __uint_as_float(c);
        mh = fmaf(s, -0.5f, m);
        const float kBig = 8.5070592e37f;   // 2^126
        fine = fabsf(m) < kBig && hi < kBig && s >= 1e-30f && m - mh == 0.5f * s && fmaf(s, 0.5f, mh) == m;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rs) : "f"(s));
        rs *= 1.0000019f;
    }
};

template <int LW, typename T>
__device__ __forceinline__ void quantise_two(const Raw8<T>& r0, const Raw8<T>& r1, uint32_t& code0, uint32_t& code1, uint32_t& word0,
                                             uint32_t& word1, bool& fine0, bool& fine1) {
    Levels<T> a, b;
    a.template set<LW>(r0);
    b.template set<LW>(r1);
    float x[8], y[8];
    r0.get(x);
    r1.get(y);
    constexpr float kMagic = 8388608.f;   // 2^23: its bits plus n are those of 2^23 + n
    const unsigned long long m2 = pair(-a.m, -b.m), rs2 = pair(a.rs, b.rs), s2 = pair(a.s, b.s), mh2 = pair(a.mh, b.mh),
                             magic2 = pair(kMagic, kMagic), back2 = pair(-kMagic, -kMagic);
    code0 = code1 = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const unsigned long long u = fma2(add2(pair(x[e], y[e]), m2), rs2, magic2);
        const unsigned long long border = fma2_up(add2(u, back2), s2, mh2);
        float u0, u1, b0, b1;
        unpair(u, u0, u1);
        unpair(border, b0, b1);
        uint32_t n0 = __float_as_uint(u0), n1 = __float_as_uint(u1);
        if (x[e] < b0) --n0;
        if (y[e] < b1) --n1;
        code0 = n0 * (1u << (4 * e)) + code0;
        code1 = n1 * (1u << (4 * e)) + code1;
    }
    code0 -= 0xFB000000u;     // the bits of 2^23 that the eight codes left in the word
    code1 -= 0xFB000000u;
    word0 = (a.c >> 16) | a.mb;
    word1 = (b.c >> 16) | b.mb;
    fine0 = a.fine;
    fine1 = b.fine;
}

// Which block a warp's unit is.  With row_start NULL it belongs to sequence unit / heads.  Else sequence s has the slots from
// slot_of(row_start[s], s) on: room for the most blocks that its n rows can touch, n of them or, where that is less for
// all sequences together, n / 16 + 2.  Slots that it does not need stay empty; so no sequence has to know the blocks of those
// before it, and a warp finds its own by a 32-way search.  (Summing the blocks of all sequences in every CTA, 4096 sequences of one
// row and 8 heads took 59 us to read instead of 32, 64 of five rows 3.6 instead of 3.1.)
struct Unit {
    int row0, first, len;   // rows from row0 on are positions [first, len)
    int seq, block, head;
    bool some, bad;
};

__device__ __forceinline__ int blocks_of(int n_rows, int len) {
    return n_rows > 0 && len > 0 ? ((len - 1) >> 4) - ((len - n_rows) >> 4) + 1 : 0;
}

__host__ __device__ __forceinline__ bool slot_a_row(const SeqView& q) { return q.rows <= q.rows / 16 + 2 * q.n_seqs; }
__host__ __device__ __forceinline__ int slots_of(const SeqView& q) {
    return !q.row_start ? q.n_seqs : slot_a_row(q) ? q.rows : q.rows / 16 + 2 * q.n_seqs;
}
__device__ __forceinline__ int slot_of(int row, int s, bool a_row) { return a_row ? row : (row >> 4) + 2 * s; }

// The whole warp.  Whatever row_start holds, the block found lies within its sequence.
__device__ __forceinline__ Unit find_unit(const SeqView& q, const CacheView& c, int unit) {
    Unit u;
    const int i = unit / c.n_kv_heads, lane = threadIdx.x & 31;
    u.head = unit - i * c.n_kv_heads;
    u.seq = i;
    long long nth = 0;
    if (q.row_start) {
        const bool a_row = slot_a_row(q);
        int lo = 0, at = 0;               // the last sequence whose slots begin at or before i, and where they do
        for (int n = q.n_seqs; n > 0;) {
            const int stride = (n + 31) >> 5, s = lo + lane * stride;
            const int first = lane * stride < n ? slot_of(q.row_start[s], s, a_row) : 0;
            const uint32_t before = __ballot_sync(0xffffffffu, lane * stride < n && first <= i);
            const int k = before ? 31 - __clz(before) : 0;
            at = __shfl_sync(0xffffffffu, first, k);
            lo += k * stride;
            n = stride > 1 ? min(stride, n - k * stride) : 0;
        }
        u.seq = lo;
        nth = static_cast<long long>(i) - at;
    }
    const SeqInfo f = wide_seq_info(q, u.seq, c.page_shift);
    u.row0 = f.row0;
    u.len = f.len;
    u.bad = f.bad;
    u.first = u.len - f.n_rows;
    u.some = nth >= 0 && nth < blocks_of(f.n_rows, u.len);
    u.block = u.some ? (u.first >> 4) + static_cast<int>(nth) : 0;
    return u;
}

// sequences that no unit leads to are checked too
__device__ __forceinline__ void report_bad(const SeqView& q, int page_shift, int* status) {
    if (q.row_start)
        for (int s = blockIdx.x * blockDim.x + threadIdx.x; s < q.n_seqs; s += gridDim.x * blockDim.x)
            if (wide_seq_info(q, s, page_shift).bad) atomicExch(status, WIDE_ERR_BAD_INDEX);
}

// A warp takes the keys or the values of a block (32 registers of loads in flight for bf16; with both, half as many
// warps fit: the write of 8188 tokens of 8 heads took 27 us instead).  32 warps an SM for the 16-bit types: those tokens
// written and read back take 28.5 us, with 24 30.0, with 40 (fewer loads in flight) 30.9, all in CTAs of eight warps.
template <typename T, int D, int G>
__global__ void __launch_bounds__(32 * kWarps, sizeof(T) == 2 ? 8 : 4)
cache_write_kernel(CacheView c, SeqView q, const T* __restrict__ k, const T* __restrict__ v, long long ks, long long vs,
                   int* __restrict__ status) {
    constexpr int kLT = D / 8;        // lanes of a token
    constexpr int kP = 32 / kLT;      // tokens a warp loads at once
    constexpr int kLW = G / 8;        // lanes of a sub-group
    constexpr int kNS = D / G;
    constexpr int kRounds = 16 / kP;
    const int lane = threadIdx.x & 31, p = lane / kLT, u8 = lane % kLT;
    const int cc = u8 >> 2, c0 = cc >> 1, c1 = cc & 1;   // 32-channel chunk of this lane's 8 channels
    const int total = slots_of(q);
    wptx::grid_dep_wait();
    const long long units = 2LL * total * c.n_kv_heads;
    for (long long unit = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5); unit < units;
         unit += static_cast<long long>(gridDim.x) * kWarps) {
        const Unit w = find_unit(q, c, static_cast<int>(unit >> 1));
        const bool values = unit & 1;
        if (w.bad && lane == 0) atomicExch(status, WIDE_ERR_BAD_INDEX);
        if (!w.some) continue;
        uint8_t* blk = wide_cache_block(c, q, w.seq, w.block << 4, w.head);
        if (!blk) {
            if (lane == 0) atomicExch(status, WIDE_ERR_BAD_INDEX);
            continue;
        }
        const int p0 = w.block << 4;
        const T* src = (values ? v : k) + w.head * D + 8 * u8;
        const long long stride = values ? vs : ks;
        // Tokens whose codes share words meet in a lane: g and g + 8 for keys; 2t, 2t + 8, 2t + 1, 2t + 9 for values, as
        // the rounds 4 t' .. 4 t' + 3.
        Raw8<T> raw[kRounds];
        uint32_t here = 0;            // bit i: the token of round i is new
        auto token = [&](int i) {
            return values ? 2 * ((i >> 2) * kP + p) + 8 * (i & 1) + ((i >> 1) & 1) : (i >> 1) * kP + p + 8 * (i & 1);
        };
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            const int pos = p0 + token(i);
            raw[i].clear();
            if (pos >= w.first && pos < w.len) {
                raw[i].load(src + static_cast<long long>(w.row0 + (pos - w.first)) * stride);
                here |= 1u << i;
            }
        }
        uint32_t* words = reinterpret_cast<uint32_t*>(blk + 16 * D + (values ? 64 * kNS : 0));
        uint32_t code[kRounds];
        // Rounds without a new token are left out: one row a sequence, 8 heads, 1024 sequences: 18 us instead of 29.5 (64: 3.7, 4.9);
        // 8188 tokens in full blocks pay 0.3 of 27 us.
        const uint32_t rounds = __reduce_or_sync(0xffffffffu, here);
        uint32_t odd = 0;             // rounds that need the slow way (the lanes of a sub-group agree)
#pragma unroll
        for (int i = 0; i < kRounds; i += 2) {
            code[i] = code[i + 1] = 0;
            if (!((rounds >> i) & 3u)) continue;
            uint32_t word[2];
            bool fine[2];
            quantise_two<kLW>(raw[i], raw[i + 1], code[i], code[i + 1], word[0], word[1], fine[0], fine[1]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!fine[h]) odd |= 1u << (i + h);
                if (((here >> (i + h)) & 1u) && u8 % kLW == 0) words[token(i + h) * kNS + u8 / kLW] = word[h];
            }
        }
        odd = __reduce_or_sync(0xffffffffu, odd & here);
        while (odd) {                 // rare: read the token again
            const int i = __ffs(odd) - 1;
            odd &= odd - 1;
            Raw8<T> again;
            again.clear();
            const bool on = (here >> i) & 1u;
            if (on) again.load(src + static_cast<long long>(w.row0 + (p0 + token(i) - w.first)) * stride);
            const uint2 r = quantise8_any<kLW>(again);
#pragma unroll
            for (int j = 0; j < kRounds; ++j)
                if (j == i) code[j] = r.y;
            if (on && u8 % kLW == 0) words[token(i) * kNS + u8 / kLW] = r.x;
        }
        if (!values) {
#pragma unroll
            for (int i = 0; i < kRounds; i += 2) {
                const bool on0 = (here >> i) & 1u, on1 = (here >> i) & 2u;
                uint32_t word[2];     // channels 0..3 and 4..7 of the lane
                uint8_t* at = blk + ((c0 * 8 + (i >> 1) * kP + p) * 4 + (u8 & 3)) * 16 + c1 * 8;
#pragma unroll
                for (int s1 = 0; s1 < 2; ++s1) {
                    uint32_t b[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t n = code[i + h] >> (16 * s1);
                        b[h] = (n & 0xFu) | ((n >> 4) & 0xF0u) | ((n << 12) & 0xF0000u) | ((n << 8) & 0xF00000u);
                    }
                    word[s1] = b[0] | (b[1] << 8);
                    if (!(on0 && on1)) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (h == 0 ? on0 : on1) {
                                at[4 * s1 + h] = static_cast<uint8_t>(b[h]);
                                at[4 * s1 + 2 + h] = static_cast<uint8_t>(b[h] >> 16);
                            }
                        }
                    }
                }
                if (on0 && on1) *reinterpret_cast<uint2*>(at) = make_uint2(word[0], word[1]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kRounds; i += 4) {
                const int t = (i >> 2) * kP + p;
#pragma unroll
                for (int a = 0; a < 2; ++a) {   // 4 channels each
                    uint8_t* at = blk + 8 * D + ((c0 * 8 + 2 * (u8 & 3) + a) * 4 + t) * 16 + c1 * 8;
                    if (((here >> i) & 15u) == 15u) {
                        // bytes a * 2 and a * 2 + 1 of the four codes
                        const uint32_t x = __byte_perm(code[i], code[i + 1], a == 0 ? 0x5140 : 0x7362);
                        const uint32_t y = __byte_perm(code[i + 2], code[i + 3], a == 0 ? 0x5140 : 0x7362);
                        *reinterpret_cast<uint2*>(at) = make_uint2(__byte_perm(x, y, 0x5410), __byte_perm(x, y, 0x7632));
                    } else {
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            if ((here >> (i + h)) & 1u) {
                                at[h] = static_cast<uint8_t>(code[i + h] >> (16 * a));
                                at[4 + h] = static_cast<uint8_t>(code[i + h] >> (16 * a + 8));
                            }
                        }
                    }
                }
            }
        }
    }
    report_bad(q, c.page_shift, status);
}

__device__ __forceinline__ void store_values(__nv_bfloat16* p, const float (&x)[8], bool) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_values(float* p, const float (&x)[8], bool wide) {
    const float4 a = make_float4(x[0], x[1], x[2], x[3]), b = make_float4(x[4], x[5], x[6], x[7]);
    if (wide) {
        wptx::st_global_256(p, a, b);
    } else {
        reinterpret_cast<float4*>(p)[0] = a;
        reinterpret_cast<float4*>(p)[1] = b;
    }
}
__device__ __forceinline__ void store_values(__nv_bfloat16* p, const float (&x)[4]) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ void store_values(float* p, const float (&x)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}

// The reverse: a lane takes the words that a lane of wide_attn_cache would (one 16-byte piece per 64
// channels), which hold 8 neighbouring channels of two keys and 4 of four values.  A warp's next block is on its way while
// it writes one out.  wide: rows of k allow 32-byte stores (fp32: two 16-byte stores leave half of every 32-byte sector to the
// second; 5356 tokens of 40 heads of 64 take 26 us with one, 27.6 with two).  Keys and values in warps of their own, more than
// 24 warps an SM, whole rows a store: no faster.
template <typename T, int D, int G>
__global__ void __launch_bounds__(32 * kWarps, 6)
cache_read_kernel(CacheView c, SeqView q, T* __restrict__ k, T* __restrict__ v, long long ks, long long vs, bool wide,
                  int* __restrict__ status) {
    constexpr int kNS = D / G;
    constexpr int kC = D / 64;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int total = slots_of(q);
    wptx::grid_dep_wait();
    const long long units = static_cast<long long>(total) * c.n_kv_heads, step = static_cast<long long>(gridDim.x) * kWarps;
    struct Block {
        Unit w;
        bool some;
        uint4 kw[kC], vw[kC];
        uint32_t kp[2][kNS], vp[4][kNS];
    };
    auto fetch = [&](long long unit, Block& b) {
        b.some = false;
        if (unit >= units) return;
        b.w = find_unit(q, c, static_cast<int>(unit));
        if (b.w.bad && lane == 0) atomicExch(status, WIDE_ERR_BAD_INDEX);
        b.some = b.w.some;
        if (!b.some) return;
        const uint8_t* blk = wide_cache_block(c, q, b.w.seq, b.w.block << 4, b.w.head);
        if (!blk && lane == 0) atomicExch(status, WIDE_ERR_BAD_INDEX);
        const uint32_t* kp = reinterpret_cast<const uint32_t*>(blk + 16 * D);
        const uint32_t* vp = reinterpret_cast<const uint32_t*>(blk + 16 * D + 64 * kNS);
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            b.kw[i] = b.vw[i] = make_uint4(0, 0, 0, 0);
            if (blk) {
                b.kw[i] = *reinterpret_cast<const uint4*>(blk + (i * 32 + lane) * 16);
                b.vw[i] = *reinterpret_cast<const uint4*>(blk + 8 * D + (i * 32 + lane) * 16);
            }
        }
#pragma unroll
        for (int i = 0; i < kNS; ++i) {
#pragma unroll
            for (int h = 0; h < 2; ++h) b.kp[h][i] = blk ? kp[(g + 8 * h) * kNS + i] : 0u;
#pragma unroll
            for (int h = 0; h < 4; ++h) b.vp[h][i] = blk ? vp[(2 * t + 8 * (h & 1) + (h >> 1)) * kNS + i] : 0u;
        }
    };
    long long unit = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    Block now, next;
    fetch(unit, now);
    for (; unit < units; unit += step, now = next) {
        fetch(unit + step, next);
        if (!now.some) continue;
        const Unit& w = now.w;
        const int p0 = w.block << 4;
        auto row_of = [&](int r) { return static_cast<long long>(w.row0 + (p0 + r - w.first)); };
        auto is_new = [&](int r) { return p0 + r >= w.first && p0 + r < w.len; };
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = g + 8 * h;
            if (!is_new(r)) continue;
            T* to = k + row_of(r) * ks + w.head * D + 8 * t;
#pragma unroll
            for (int cc = 0; cc < D / 32; ++cc) {
                const uint4 four = now.kw[cc >> 1];
                const uint32_t w0 = (cc & 1) ? four.z : four.x, w1 = (cc & 1) ? four.w : four.y;
                const float s = wide_cache_scale(now.kp[h][cc * 32 / G]), m = wide_cache_min(now.kp[h][cc * 32 / G]);
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t word = e < 4 ? w0 : w1;
                    const int shift = 8 * h + 16 * (e & 1) + 4 * ((e >> 1) & 1);
                    x[e] = fmaf(s, static_cast<float>((word >> shift) & 15u), m);
                }
                store_values(to + 32 * cc, x, wide);
            }
        }
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int r = 2 * t + 8 * (h & 1) + (h >> 1);
            if (!is_new(r)) continue;
            T* to = v + row_of(r) * vs + w.head * D + 4 * g;
#pragma unroll
            for (int cc = 0; cc < D / 32; ++cc) {
                const uint4 four = now.vw[cc >> 1];
                const uint32_t w0 = (cc & 1) ? four.z : four.x, w1 = (cc & 1) ? four.w : four.y;
                const float s = wide_cache_scale(now.vp[h][cc * 32 / G]), m = wide_cache_min(now.vp[h][cc * 32 / G]);
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[e] = fmaf(s, static_cast<float>(((e < 2 ? w0 : w1) >> (8 * h + 4 * (e & 1))) & 15u), m);
                store_values(to + 32 * cc, x);
            }
        }
    }
    report_bad(q, c.page_shift, status);
}

// CTAs for the slots.  Writing: twice what is resident of 16-bit types (four times of fp32), if there is so much.  Reading: what is resident,
// so that a warp asks for its next block ahead; but three times that where there is so much, since later CTAs then even out
// what the first ones finish unevenly (8 heads of 128 read into bf16, resident / three times: 8192 tokens 9.5 / 10.8 us, 16384
// 17.6 / 18.0, 24576 25.7 / 24.5, 65536 68.6 / 63.0).
int grid_for(const wide_ctx* ctx, const CacheView& c, const SeqView& q, bool write) {
    const long long units = static_cast<long long>(slots_of(q)) * c.n_kv_heads * (write ? 2 : 1);
    const long long ctas = (units + kWarps - 1) / kWarps, sms = ctx->sm_count;
    return static_cast<int>(max(1LL, min(ctas, write ? 16 * sms : ctas > 18 * sms ? 18 * sms : 6 * sms)));
}

template <typename T, int D, int G>
int launch(wide_ctx* ctx, cudaStream_t s, bool write, const CacheView& c, const SeqView& q, void* k, void* v, long long ks,
           long long vs) {
    const int grid = grid_for(ctx, c, q, write);
    int* status = ctx->d_status + WIDE_STATUS_INDEX;
    WideLaunch l(ctx, s, write ? "cache_write" : "cache_read");
    if (write)
        WIDE_CUDA_CHECK(wide_launch_after(ctx, cache_write_kernel<T, D, G>, dim3(grid), dim3(32 * kWarps), 0, s, c, q,
                                          static_cast<const T*>(k), static_cast<const T*>(v), ks, vs, status));
    else
        WIDE_CUDA_CHECK(wide_launch_after(ctx, cache_read_kernel<T, D, G>, dim3(grid), dim3(32 * kWarps), 0, s, c, q, static_cast<T*>(k),
                                          static_cast<T*>(v), ks, vs, wide_rows32(k, ks * static_cast<long long>(sizeof(T))), status));
    return WIDE_OK;
}

template <typename T>
int launch_dims(wide_ctx* ctx, cudaStream_t s, bool write, const CacheView& c, const SeqView& q, int D, int G, void* k, void* v,
                long long ks, long long vs) {
    if (D == 128) {
        if (G == 128) return launch<T, 128, 128>(ctx, s, write, c, q, k, v, ks, vs);
        if (G == 64) return launch<T, 128, 64>(ctx, s, write, c, q, k, v, ks, vs);
        return launch<T, 128, 32>(ctx, s, write, c, q, k, v, ks, vs);
    }
    if (G == 64) return launch<T, 64, 64>(ctx, s, write, c, q, k, v, ks, vs);
    return launch<T, 64, 32>(ctx, s, write, c, q, k, v, ks, vs);
}

}  // namespace

int wide_launch_cache_move(wide_ctx* ctx, cudaStream_t s, bool write, const wide_cache* cache, const wide_seqs* seqs, void* k,
                           void* v, int dtype, int rows, long long ks, long long vs) {
    const CacheView c = wide_cache_view(cache);
    const SeqView q = wide_seq_view(seqs, rows);
    if (dtype == WIDE_F32)
        return launch_dims<float>(ctx, s, write, c, q, cache->head_dim, cache->quant_group, k, v, ks, vs);
    return launch_dims<__nv_bfloat16>(ctx, s, write, c, q, cache->head_dim, cache->quant_group, k, v, ks, vs);
}
