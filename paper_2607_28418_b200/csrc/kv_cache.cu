// Writing keys and values into the 4-bit paged cache and reading them back (layout and levels: wide.h).
//
// Both kernels move bytes: per value 2 (bf16) in and 0.56 out or the other way round, so HBM is the bound.
// A warp takes one block of the cache, 16 positions of one head, because that is the unit in
// which codes of several tokens share words: with all 16 tokens in hand it stores whole words, and where
// only some of them are new (a decode step: one) it stores the bytes that belong to them.  A lane holds
// 8 neighbouring channels, so a row is read in 16-byte pieces, coalesced, and the extremes of a
// sub-group are 8 values in registers and two to four shuffles.  The token of the block that a lane takes is
// chosen so that the tokens whose codes share a word meet in one lane.
#include "cache_levels.cuh"

namespace {

constexpr int kWarps = 4;           // of a CTA (8 start and end in larger steps: 8188 tokens written and read back 28.7 us, with four 27.5)

// A warp takes the keys or the values of a block (32 registers of loads in flight for bf16; with both, half as many
// warps fit: the write of 8188 tokens of 8 heads took 27 us instead).  32 warps an SM for the 16-bit types: those tokens
// written and read back take 28.5 us, with 24 30.0, with 40 (fewer loads in flight) 30.9, all in CTAs of eight warps.
template <typename T, int D, int G>
__global__ void __launch_bounds__(32 * kWarps, sizeof(T) == 2 ? 8 : 4)
cache_write_kernel(CacheView c, SeqView q, const T* __restrict__ k, const T* __restrict__ v, long long ks, long long vs,
                   int* __restrict__ status) {
    constexpr int kLT = BlockLanes<D>::kLT, kRounds = BlockLanes<D>::kRounds;
    const int lane = threadIdx.x & 31, p = lane / kLT, u8 = lane % kLT;
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
        Raw8<T> raw[kRounds];
        uint32_t here = 0;            // bit i: the token of round i is new
        auto token = [&](int i) { return BlockLanes<D>::token(values, p, i); };
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            const int pos = p0 + token(i);
            raw[i].clear();
            if (pos >= w.first && pos < w.len) {
                raw[i].load(src + static_cast<long long>(w.row0 + (pos - w.first)) * stride);
                here |= 1u << i;
            }
        }
        put_block<T, D, G>(raw, here, blk, values, [&](int i, bool on) {
            Raw8<T> x;
            x.clear();
            if (on) x.load(src + static_cast<long long>(w.row0 + (p0 + token(i) - w.first)) * stride);
            return x;
        });
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
