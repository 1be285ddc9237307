// Head-group-masked causal attention of a batch of sequences over the 4-bit paged cache (wide_attn_cache).
//
// One CTA per (row, query head).  A warp takes blocks of 16 keys in turn; lane 4 g + t holds the key codes
// of tokens g and g + 8 and the value codes of tokens 2t, 2t + 1, 2t + 8, 2t + 9 (the order of the layout),
// dots its channels with the query, sums over the four lanes of a token, keeps a running maximum and sum, and
// adds the values of its four tokens; lanes and warps are joined at the end.
#include <math_constants.h>

#include "cache.cuh"
#include "ptx.cuh"

namespace {

constexpr int kWarps = 4;

template <int D, int G>
__global__ void __launch_bounds__(32 * kWarps)
attn_cache_kernel(CacheView c, SeqView q, const __nv_bfloat16* __restrict__ qm, long long qs, int n_q, int hpg,
                  const uint32_t* __restrict__ mask_bits, int words, int causal, float scale_log2e,
                  __nv_bfloat16* __restrict__ o, int* __restrict__ status) {
    constexpr int kNS = D / G;
    constexpr int kC = D / 32;
    __shared__ float sm_m[kWarps], sm_l[kWarps], sm_o[kWarps][D];
    const int row = blockIdx.x, head = blockIdx.y;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    int s = row;
    if (q.row_start) {
        int lo = 0, hi = q.n_seqs - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (q.row_start[mid] <= row) lo = mid;
            else hi = mid - 1;
        }
        s = lo;
    }
    if (s >= q.n_seqs) return;
    const SeqInfo info = wide_seq_info(q, s, c.page_shift);
    if (info.bad && threadIdx.x == 0) atomicExch(status, WIDE_ERR_BAD_INDEX);
    if (row < info.row0 || row >= info.row0 + info.n_rows) return;
    __nv_bfloat16* out = o + (static_cast<size_t>(row) * n_q + head) * D;
    const bool on = !mask_bits || wide_mask_bit(mask_bits, words, row, head / hpg);
    const int seen = !on ? 0 : causal ? info.len - info.n_rows + (row - info.row0) + 1 : info.len;
    if (seen <= 0) {
        for (int d = threadIdx.x; d < D; d += 32 * kWarps) out[d] = __float2bfloat16_rn(0.f);
        return;
    }
    const int kvh = head / (n_q / c.n_kv_heads);
    float qr[kC][8];
#pragma unroll
    for (int cc = 0; cc < kC; ++cc)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            qr[cc][e] = __bfloat162float(qm[row * qs + head * D + 32 * cc + 8 * t + e]) * scale_log2e;
    float m = -CUDART_INF_F, l = 0.f, acc[kC][4] = {};
    for (int b = warp; b * 16 < seen; b += kWarps) {
        const uint8_t* blk = wide_cache_block(c, q, s, b << 4, kvh);
        if (!blk) {
            if (lane == 0) atomicExch(status, WIDE_ERR_BAD_INDEX);
            continue;
        }
        const uint4* kw4 = reinterpret_cast<const uint4*>(blk);
        const uint4* vw4 = reinterpret_cast<const uint4*>(blk + 8 * D);
        const uint32_t* kp = reinterpret_cast<const uint32_t*>(blk + 16 * D);
        const uint32_t* vp = kp + 16 * kNS;
        float sc[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = g + 8 * h;
            float a = 0.f;
#pragma unroll
            for (int cc = 0; cc < kC; ++cc) {
                const uint4 w4 = kw4[(cc >> 1) * 32 + lane];
                const uint32_t w0 = (cc & 1) ? w4.z : w4.x, w1 = (cc & 1) ? w4.w : w4.y;
                const uint32_t pw = kp[r * kNS + cc * 32 / G];
                const float st = wide_cache_scale(pw), mi = wide_cache_min(pw);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int shift = 8 * h + 16 * (e & 1) + 4 * ((e >> 1) & 1);
                    a = fmaf(fmaf(st, static_cast<float>(((e < 4 ? w0 : w1) >> shift) & 15u), mi), qr[cc][e], a);
                }
            }
            a += __shfl_xor_sync(0xffffffffu, a, 1);
            a += __shfl_xor_sync(0xffffffffu, a, 2);
            sc[h] = b * 16 + r < seen ? a : -CUDART_INF_F;
        }
        float mx = fmaxf(sc[0], sc[1]);
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
        const float m_new = fmaxf(m, mx), m_use = m_new == -CUDART_INF_F ? 0.f : m_new;
        const float alpha = exp2f(m - m_use);
        float p[2] = {exp2f(sc[0] - m_use), exp2f(sc[1] - m_use)};
        float sum = p[0] + p[1];
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        l = l * alpha + sum;
        m = m_new;
#pragma unroll
        for (int cc = 0; cc < kC; ++cc)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[cc][e] *= alpha;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int r = 2 * t + 8 * (h & 1) + (h >> 1);
            const float pr = __shfl_sync(0xffffffffu, p[h & 1], 4 * (2 * t + (h >> 1)));
            if (b * 16 + r >= seen) continue;
#pragma unroll
            for (int cc = 0; cc < kC; ++cc) {
                const uint4 w4 = vw4[(cc >> 1) * 32 + lane];
                const uint32_t w0 = (cc & 1) ? w4.z : w4.x, w1 = (cc & 1) ? w4.w : w4.y;
                const uint32_t pw = vp[r * kNS + cc * 32 / G];
                const float st = wide_cache_scale(pw), mi = wide_cache_min(pw);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[cc][e] = fmaf(pr, fmaf(st, static_cast<float>(((e < 2 ? w0 : w1) >> (8 * h + 4 * (e & 1))) & 15u), mi), acc[cc][e]);
            }
        }
    }
#pragma unroll
    for (int cc = 0; cc < kC; ++cc)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            acc[cc][e] += __shfl_xor_sync(0xffffffffu, acc[cc][e], 1);
            acc[cc][e] += __shfl_xor_sync(0xffffffffu, acc[cc][e], 2);
            if (t == 0) sm_o[warp][32 * cc + 4 * g + e] = acc[cc][e];
        }
    if (lane == 0) {
        sm_m[warp] = m;
        sm_l[warp] = l;
    }
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += 32 * kWarps) {
        float mm = -CUDART_INF_F;
        for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, sm_m[w]);
        const float m_use = mm == -CUDART_INF_F ? 0.f : mm;
        float num = 0.f, den = 0.f;
        for (int w = 0; w < kWarps; ++w) {
            const float al = exp2f(sm_m[w] - m_use);
            num += sm_o[w][d] * al;
            den += sm_l[w] * al;
        }
        out[d] = __float2bfloat16_rn(den == 0.f ? 0.f : num / den);
    }
}

}  // namespace

size_t wide_attn_cache_workspace(int rows, int n_q, int n_kv, int head_dim) {
    (void)rows; (void)n_q; (void)n_kv; (void)head_dim;
    return 256;
}

int wide_launch_attn_cache(wide_ctx* ctx, cudaStream_t s, const wide_cache* cache, const wide_seqs* seqs, const void* q,
                           int rows, long long qs, int n_q, int hpg, const uint32_t* mask_bits, int causal, float scale,
                           void* o, void* ws) {
    (void)ws;
    const CacheView c = wide_cache_view(cache);
    const SeqView sv = wide_seq_view(seqs, rows);
    const int words = (n_q / hpg + 31) / 32;
    const dim3 grid(rows, n_q);
    WideLaunch l(ctx, s, "attn_cache");
#define GO(D, G)                                                                                                       \
    attn_cache_kernel<D, G><<<grid, 32 * kWarps, 0, s>>>(c, sv, static_cast<const __nv_bfloat16*>(q), qs, n_q, hpg, mask_bits, \
                                                         words, causal, scale * 1.4426950408889634f,                 \
                                                         static_cast<__nv_bfloat16*>(o), ctx->d_status + WIDE_STATUS_INDEX)
    if (cache->head_dim == 128) {
        if (cache->quant_group == 128) GO(128, 128);
        else if (cache->quant_group == 64) GO(128, 64);
        else GO(128, 32);
    } else {
        if (cache->quant_group == 64) GO(64, 64);
        else GO(64, 32);
    }
#undef GO
    return cudaGetLastError() == cudaSuccess ? WIDE_OK : WIDE_ERR_CUDA;
}
