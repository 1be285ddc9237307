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

constexpr int kWarps = 8;

__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8]) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// sign-correct a - b - c for c near a - b: d = a - b rounded, e its exact remainder (two-sum)
template <typename F>
__device__ __forceinline__ F exact_gap(F a, F b, F c) {
    const F d = a - b;
    const F bb = d - a;
    const F e = (a - (d - bb)) + ((-b) - bb);
    return (d - c) + e;
}

// Levels of 8 channels of a sub-group that spans LW lanes: code e in bits 4e.  Returns the parameter word.
// The definition is exact (how many borders does x reach), so the same input always gives the same code
// whatever the order of evaluation.  The border nearest to x is found in fp32 (2^-21 off at most, a
// border and a half apart from the next one), and x is compared with that one exactly: (i + 1/2) s has 13
// bits, x - m is a two-sum.  Scale: 15 c has 12 bits, so the smallest bf16 c with 15 c >= max - m is also
// found by exact comparison.  Magnitudes at which fp32 overflows or has few bits left go through fp64.
template <int LW>
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], uint32_t& codes) {
    float lo = x[0], hi = x[0];
    bool finite = fabsf(x[0]) <= 3.4028234e38f;
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        finite = finite && fabsf(x[i]) <= 3.4028234e38f;
    }
    int ok = finite ? 1 : 0;
#pragma unroll
    for (int o = 1; o < LW; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        ok &= __shfl_xor_sync(0xffffffffu, ok, o);
    }
    codes = 0;
    if (!ok) return 0x7FC07FC0u;
    // bf16 at or below lo: towards zero for positive numbers, away from it for negative ones
    lo += 0.f;   // zeros are +0
    hi += 0.f;
    const uint32_t lb = __float_as_uint(lo);
    const uint32_t mb = (lo < 0.f ? lb + 0xFFFFu : lb) & 0xFFFF0000u;
    const float m = __uint_as_float(mb);
    if (isinf(m)) return 0x7FC07FC0u;   // an fp32 minimum below the lowest bf16 number
    const float kBig = 8.5070592e37f;   // 2^126
    float s;
    bool plain = fabsf(lo) < kBig && fabsf(hi) < kBig;
    if (plain) {
        const float q = (hi - m) * (1.f / 15.f) * 0.999999f;
        uint32_t c = __float_as_uint(q) & 0xFFFF0000u;
        if (exact_gap(hi, m, 15.f * __uint_as_float(c)) > 0.f) c += 0x10000u;
        if (exact_gap(hi, m, 15.f * __uint_as_float(c)) > 0.f) c += 0x10000u;
        s = __uint_as_float(c);
        plain = s >= 1e-30f || s == 0.f;
    }
    if (!plain) {
        const double q = (static_cast<double>(hi) - static_cast<double>(m)) / 15.0;
        s = __uint_as_float((__float_as_uint(__double2float_ru(q)) + 0xFFFFu) & 0xFFFF0000u);
    }
    const uint32_t word = (__float_as_uint(s) >> 16) | mb;
    if (s == 0.f) return word;
    if (plain) {
        const float rs = 1.f / s;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = min(static_cast<int>((x[e] - m) * rs), 14);
            const float border = (static_cast<float>(i) + 0.5f) * s;
            const uint32_t n = i + (exact_gap(x[e], m, border) >= 0.f ? 1 : 0);
            codes |= n << (4 * e);
        }
    } else {
#pragma unroll 1
        for (int i = 0; i < 15; ++i) {
            const double border = (i + 0.5) * static_cast<double>(s);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                codes += exact_gap(static_cast<double>(x[e]), static_cast<double>(m), border) >= 0.0 ? 1u << (4 * e) : 0u;
        }
    }
    return word;
}

// Which block a warp's unit is.  With row_start NULL a unit is (sequence, head); else the CTA sums the
// sequences' block counts once and every warp finds its sequence by bisection.
struct Unit {
    SeqInfo info;
    int seq, block, head;
};

__device__ __forceinline__ int blocks_of(const SeqInfo& i) {
    return i.n_rows > 0 && i.len > 0 ? ((i.len - 1) >> 4) - ((i.len - i.n_rows) >> 4) + 1 : 0;
}

// offsets[s] = blocks of the sequences before s; returns the total.  All threads of the CTA.
__device__ int scan_blocks(const SeqView& q, int page_shift, int* offsets, int* part, int* status) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (q.n_seqs + 32 * kWarps - 1) / (32 * kWarps);
    const int a = min(q.n_seqs, tid * per), b = min(q.n_seqs, a + per);
    int sum = 0;
    for (int s = a; s < b; ++s) {
        const SeqInfo i = wide_seq_info(q, s, page_shift);
        if (i.bad && blockIdx.x == 0) atomicExch(status, WIDE_ERR_BAD_INDEX);
        offsets[s] = sum;
        sum += blocks_of(i);
    }
    int up = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, up, o);
        if (lane >= o) up += v;
    }
    if (lane == 31) part[warp] = up;
    __syncthreads();
    int base = up - sum, total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) base += part[w];
        total += part[w];
    }
    for (int s = a; s < b; ++s) offsets[s] += base;
    __syncthreads();
    return total;
}

__device__ __forceinline__ Unit find_unit(const SeqView& q, const CacheView& c, const int* offsets, int unit) {
    Unit u;
    const int i = unit / c.n_kv_heads;
    u.head = unit - i * c.n_kv_heads;
    u.seq = i;
    u.block = 0;
    if (q.row_start) {
        int lo = 0, hi = q.n_seqs - 1;   // the last sequence that starts at or before block i
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (offsets[mid] <= i) lo = mid;
            else hi = mid - 1;
        }
        u.seq = lo;
        u.block = i - offsets[lo];
    }
    u.info = wide_seq_info(q, u.seq, c.page_shift);
    if (blocks_of(u.info) > 0) u.block += (u.info.len - u.info.n_rows) >> 4;
    return u;
}

template <typename T, int D, int G>
__global__ void __launch_bounds__(32 * kWarps)
cache_write_kernel(CacheView c, SeqView q, const T* __restrict__ k, const T* __restrict__ v, long long ks, long long vs,
                   int* __restrict__ status) {
    constexpr int kLT = D / 8;        // lanes of a token
    constexpr int kP = 32 / kLT;      // tokens a warp loads at once
    constexpr int kLW = G / 8;        // lanes of a sub-group
    constexpr int kNS = D / G;
    extern __shared__ int offsets[];
    __shared__ int part[kWarps];
    const int lane = threadIdx.x & 31, p = lane / kLT, u8 = lane % kLT;
    const int cc = u8 >> 2, c0 = cc >> 1, c1 = cc & 1;   // 32-channel chunk of this lane's 8 channels
    int total = q.n_seqs;
    if (q.row_start) total = scan_blocks(q, c.page_shift, offsets, part, status);
    const long long units = static_cast<long long>(total) * c.n_kv_heads;
    for (long long unit = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5); unit < units;
         unit += static_cast<long long>(gridDim.x) * kWarps) {
        const Unit w = find_unit(q, c, offsets, static_cast<int>(unit));
        const int first = w.info.len - w.info.n_rows;
        if (!q.row_start && w.info.bad && lane == 0) atomicExch(status, WIDE_ERR_BAD_INDEX);
        if (blocks_of(w.info) == 0) continue;
        uint8_t* blk = wide_cache_block(c, q, w.seq, w.block << 4, w.head);
        if (!blk) {
            if (lane == 0) atomicExch(status, WIDE_ERR_BAD_INDEX);
            continue;
        }
        const int p0 = w.block << 4;
        auto row_of = [&](int r) { return static_cast<long long>(w.info.row0 + (p0 + r - first)); };
        auto is_new = [&](int r) { return p0 + r >= first && p0 + r < w.info.len; };
        const int col = w.head * D + 8 * u8;
        // keys: tokens g and g + 8 share words
#pragma unroll
        for (int it = 0; it < 8 / kP; ++it) {
            const int g = it * kP + p;
            uint32_t code[2];
            bool on[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = g + 8 * h;
                on[h] = is_new(r);
                float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (on[h]) load8(k + row_of(r) * ks + col, x);
                const uint32_t word = quantise8<kLW>(x, code[h]);
                if (on[h] && u8 % kLW == 0)
                    reinterpret_cast<uint32_t*>(blk + 16 * D)[r * kNS + u8 / kLW] = word;
            }
            uint32_t word[2];   // channels 0..3 and 4..7 of the lane
            uint8_t* at = blk + ((c0 * 8 + g) * 4 + (u8 & 3)) * 16 + c1 * 8;
#pragma unroll
            for (int s1 = 0; s1 < 2; ++s1) {
                uint32_t b[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t n = (code[h] >> (16 * s1)) & 0xFFFFu;
                    b[h] = (n & 0xFu) | ((n >> 4) & 0xF0u) | ((n << 12) & 0xF0000u) | ((n << 8) & 0xF00000u);
                }
                word[s1] = b[0] | (b[1] << 8);
                if (!(on[0] && on[1])) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (on[h]) {
                            at[4 * s1 + h] = static_cast<uint8_t>(b[h]);
                            at[4 * s1 + 2 + h] = static_cast<uint8_t>(b[h] >> 16);
                        }
                    }
                }
            }
            if (on[0] && on[1]) *reinterpret_cast<uint2*>(at) = make_uint2(word[0], word[1]);
        }
        // values: tokens 2t, 2t + 8, 2t + 1, 2t + 9 share words
#pragma unroll
        for (int it = 0; it < 4 / kP || it < 1; ++it) {
            const int t = it * kP + p;
            uint32_t code[4];
            bool on[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const int r = 2 * t + 8 * (h & 1) + (h >> 1);
                on[h] = is_new(r);
                float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (on[h]) load8(v + row_of(r) * vs + col, x);
                const uint32_t word = quantise8<kLW>(x, code[h]);
                if (on[h] && u8 % kLW == 0)
                    reinterpret_cast<uint32_t*>(blk + 16 * D + 64 * kNS)[r * kNS + u8 / kLW] = word;
            }
            const bool all = on[0] && on[1] && on[2] && on[3];
#pragma unroll
            for (int a = 0; a < 2; ++a) {   // 4 channels each
                const int g = 2 * (u8 & 3) + a;
                uint8_t* at = blk + 8 * D + ((c0 * 8 + g) * 4 + t) * 16 + c1 * 8;
                if (all) {
                    uint32_t word[2];
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        const int sh = 16 * a + 8 * m;
                        word[m] = ((code[0] >> sh) & 0xFFu) | (((code[1] >> sh) & 0xFFu) << 8) |
                                  (((code[2] >> sh) & 0xFFu) << 16) | (((code[3] >> sh) & 0xFFu) << 24);
                    }
                    *reinterpret_cast<uint2*>(at) = make_uint2(word[0], word[1]);
                } else {
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        if (on[h]) {
                            at[h] = static_cast<uint8_t>(code[h] >> (16 * a));
                            at[4 + h] = static_cast<uint8_t>(code[h] >> (16 * a + 8));
                        }
                    }
                }
            }
        }
    }
}

__device__ __forceinline__ void store_values(__nv_bfloat16* p, const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_values(float* p, const float (&x)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store_values(__nv_bfloat16* p, const float (&x)[4]) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ void store_values(float* p, const float (&x)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}

// The reverse: a lane takes the words that a lane of wide_attn_cache would (one 16-byte piece per 64
// channels), which hold 8 neighbouring channels of two keys and 4 of four values.
template <typename T, int D, int G>
__global__ void __launch_bounds__(32 * kWarps)
cache_read_kernel(CacheView c, SeqView q, T* __restrict__ k, T* __restrict__ v, long long ks, long long vs,
                  int* __restrict__ status) {
    constexpr int kNS = D / G;
    constexpr int kC = D / 64;
    extern __shared__ int offsets[];
    __shared__ int part[kWarps];
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    int total = q.n_seqs;
    if (q.row_start) total = scan_blocks(q, c.page_shift, offsets, part, status);
    const long long units = static_cast<long long>(total) * c.n_kv_heads;
    for (long long unit = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5); unit < units;
         unit += static_cast<long long>(gridDim.x) * kWarps) {
        const Unit w = find_unit(q, c, offsets, static_cast<int>(unit));
        const int first = w.info.len - w.info.n_rows;
        if (!q.row_start && w.info.bad && lane == 0) atomicExch(status, WIDE_ERR_BAD_INDEX);
        if (blocks_of(w.info) == 0) continue;
        const uint8_t* blk = wide_cache_block(c, q, w.seq, w.block << 4, w.head);
        if (!blk && lane == 0) atomicExch(status, WIDE_ERR_BAD_INDEX);
        const int p0 = w.block << 4;
        auto row_of = [&](int r) { return static_cast<long long>(w.info.row0 + (p0 + r - first)); };
        auto is_new = [&](int r) { return p0 + r >= first && p0 + r < w.info.len; };
        uint4 kw[kC], vw[kC];
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            kw[i] = vw[i] = make_uint4(0, 0, 0, 0);
            if (blk) {
                kw[i] = *reinterpret_cast<const uint4*>(blk + (i * 32 + lane) * 16);
                vw[i] = *reinterpret_cast<const uint4*>(blk + 8 * D + (i * 32 + lane) * 16);
            }
        }
        const uint32_t* kp = reinterpret_cast<const uint32_t*>(blk + 16 * D);
        const uint32_t* vp = reinterpret_cast<const uint32_t*>(blk + 16 * D + 64 * kNS);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = g + 8 * h;
            if (!is_new(r)) continue;
#pragma unroll
            for (int cc = 0; cc < D / 32; ++cc) {
                const uint32_t w0 = (cc & 1) ? kw[cc >> 1].z : kw[cc >> 1].x, w1 = (cc & 1) ? kw[cc >> 1].w : kw[cc >> 1].y;
                const uint32_t pw = blk ? kp[r * kNS + cc * 32 / G] : 0u;
                const float s = wide_cache_scale(pw), m = wide_cache_min(pw);
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t word = e < 4 ? w0 : w1;
                    const int shift = 8 * h + 16 * (e & 1) + 4 * ((e >> 1) & 1);
                    x[e] = fmaf(s, static_cast<float>((word >> shift) & 15u), m);
                }
                store_values(k + row_of(r) * ks + w.head * D + 32 * cc + 8 * t, x);
            }
        }
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int r = 2 * t + 8 * (h & 1) + (h >> 1);
            if (!is_new(r)) continue;
#pragma unroll
            for (int cc = 0; cc < D / 32; ++cc) {
                const uint32_t w0 = (cc & 1) ? vw[cc >> 1].z : vw[cc >> 1].x, w1 = (cc & 1) ? vw[cc >> 1].w : vw[cc >> 1].y;
                const uint32_t pw = blk ? vp[r * kNS + cc * 32 / G] : 0u;
                const float s = wide_cache_scale(pw), m = wide_cache_min(pw);
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[e] = fmaf(s, static_cast<float>(((e < 2 ? w0 : w1) >> (8 * h + 4 * (e & 1))) & 15u), m);
                store_values(v + row_of(r) * vs + w.head * D + 32 * cc + 4 * g, x);
            }
        }
    }
}

// CTAs for the most blocks that `rows` rows of these sequences can touch: a sequence's n rows lie in at
// most n / 16 + 2 blocks, and in at most n.
int grid_for(const wide_ctx* ctx, const CacheView& c, const SeqView& q) {
    const long long blocks = q.row_start ? min(static_cast<long long>(q.rows), q.rows / 16 + 2LL * q.n_seqs) : q.n_seqs;
    const long long ctas = (blocks * c.n_kv_heads + kWarps - 1) / kWarps;
    return static_cast<int>(max(1LL, min(ctas, 8LL * ctx->sm_count)));
}

template <typename T, int D, int G>
int launch(wide_ctx* ctx, cudaStream_t s, bool write, const CacheView& c, const SeqView& q, void* k, void* v, long long ks,
           long long vs) {
    const int grid = grid_for(ctx, c, q);
    const size_t smem = q.row_start ? static_cast<size_t>(q.n_seqs) * sizeof(int) : 0;
    int* status = ctx->d_status + WIDE_STATUS_INDEX;
    WideLaunch l(ctx, s, write ? "cache_write" : "cache_read");
    if (write)
        cache_write_kernel<T, D, G><<<grid, 32 * kWarps, smem, s>>>(c, q, static_cast<const T*>(k), static_cast<const T*>(v), ks, vs, status);
    else
        cache_read_kernel<T, D, G><<<grid, 32 * kWarps, smem, s>>>(c, q, static_cast<T*>(k), static_cast<T*>(v), ks, vs, status);
    return cudaGetLastError() == cudaSuccess ? WIDE_OK : WIDE_ERR_CUDA;
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
