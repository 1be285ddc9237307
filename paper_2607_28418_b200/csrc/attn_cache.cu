// Head-group-masked causal attention of a batch of sequences over the 4-bit paged cache (wide_attn_cache).
//
// For the few query rows of a sequence the work is reading the cache once, so HBM is the bound; a
// value costs half a byte, 46 of them arrive per clock and SM, and what can be spent on one is under three
// lane instructions.  Hence:
//   - The codes go into the tensor cores as they lie.  A 4-bit code in the low mantissa bits of an fp16
//     number IS a (subnormal) number, n * 2^-24, one nibble up n * 2^-20, so four operand registers of an
//     m16n8k16 instruction are five integer instructions away from a word of eight codes; scale and minimum
//     stay outside:  q . k = s (q . n) + m (sum q)  per sub-group, applied to the 16 x 8 scores, and
//     sum p v = sum (p s) n + sum p m.  Keys are the 16-row operand, up to eight query rows the 8-column one,
//     so nothing is padded but the queries.
//   - Queries enter as fp16 times a power of two of their own (exact for bf16 numbers within 2^-29 of the
//     row's largest), probabilities as fp16 (2^-11) times the step of the value relative to a running
//     power of two, so that neither can leave fp16's range.  Scores, sums and outputs are fp32.
//   - 16-key blocks are the unit of work.  All blocks of all (sequence, KV head in use, 8 * NB query
//     rows) items form one line that is cut into equal pieces for CTAs and warps, so uneven sequences load
//     the SMs evenly.  A warp streams its piece through a ring of its own (bulk copies, one per
//     block, issued ahead of the compute across item borders; no barrier between warps).
//   - A warp that covered an item writes its output; pieces of items are joined first within the
//     CTA, then (at most two per CTA) by a second small kernel.  The order of joining is fixed.
#include <math_constants.h>

#include "cache.cuh"
#include "ptx.cuh"

namespace {

using namespace wptx;

constexpr int kBlk = 2;            // blocks of a ring stage: 32 keys
constexpr int kMaxCtas = 160;
constexpr int kPlanSmem = 4096;    // bytes of shared memory for the plan of a small batch

struct AttnArgs {
    CacheView c;
    SeqView q;
    const __nv_bfloat16* qm;
    long long qs;
    int n_q, share, hpg, words, causal;
    const uint32_t* mask_bits;
    float scale_log2e;
    __nv_bfloat16* o;
    int* status;                   // device status word (timeouts); index errors go to WIDE_STATUS_INDEX
    unsigned long long wait_ns;
    int stages, plan_words;        // plan_words: words of a sequence's head mask
    unsigned char* plan;           // the plan in the workspace, or NULL: every CTA makes its own in shared memory
    float* heads;                  // partial results of warps whose first item began before their piece
    float* parts;                  // [CTA][2] partial results of CTAs
    int* meta;                     // [CTA][2][4] {0 / 1 / 2: none, more follows, last piece; sequence, KV head, row block}
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }   // -126 <= e <= 127

// d (16x8, fp32) += a (16x16, fp16) * b (16x8, fp16)
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
template <int N>
__device__ __forceinline__ void lds_words(uint32_t a, uint32_t (&w)[N]) {
    if (N == 1) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(a));
    if (N == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[N > 1]) : "r"(a));
    if (N == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[N > 1]), "=r"(w[N > 2 ? 2 : 0]), "=r"(w[N > 3 ? 3 : 0]) : "r"(a));
}

// ------------------------------------------------------------------------------------------------ the plan
// offsets[s] = units (16-key blocks of items) of the sequences before s, masks[s] = KV heads in use.
struct Plan {
    long long* offsets;
    uint32_t* masks;
};
__device__ __forceinline__ Plan plan_at(unsigned char* p, int n_seqs) {
    return Plan{reinterpret_cast<long long*>(p), reinterpret_cast<uint32_t*>(p + 8 * (n_seqs + 1))};
}
size_t plan_bytes(int n_seqs, int words) { return 8 * static_cast<size_t>(n_seqs + 1) + 4 * static_cast<size_t>(n_seqs) * words; }

__device__ __forceinline__ int row_blocks(int n_rows, int share, int rows_per) { return (n_rows * share + rows_per - 1) / rows_per; }

// Does any new row of the sequence use KV head h?  Looked at for up to 16 new rows.
__device__ __forceinline__ bool head_used(const AttnArgs& a, const SeqInfo& i, int h) {
    if (!a.mask_bits || i.n_rows > 16) return true;
    const int g0 = h * a.share / a.hpg, g1 = (h * a.share + a.share - 1) / a.hpg;
    bool any = false;
    for (int r = 0; r < i.n_rows; ++r)
        for (int g = g0; g <= g1; ++g) any |= wide_mask_bit(a.mask_bits, a.words, i.row0 + r, g);
    return any;
}

template <int ROWS>
__device__ void make_plan(const AttnArgs& a, const Plan& p, long long* part, bool report) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
    // a warp per sequence: lanes are heads
    for (int s = warp; s < a.q.n_seqs; s += n_warps) {
        const SeqInfo i = wide_seq_info(a.q, s, a.c.page_shift);
        if (i.bad && report && lane == 0) atomicExch(a.status + WIDE_STATUS_INDEX, WIDE_ERR_BAD_INDEX);
        int used = 0;
        const bool some = i.n_rows > 0 && i.len > 0;
        for (int w = 0; w < a.plan_words; ++w) {
            const int h = 32 * w + lane;
            const uint32_t m = __ballot_sync(0xffffffffu, some && h < a.c.n_kv_heads && head_used(a, i, h));
            used += __popc(m);
            if (lane == 0) p.masks[s * a.plan_words + w] = m;
        }
        if (lane == 0)
            p.offsets[s] = static_cast<long long>(used) * ((i.len + 15) >> 4) * (some ? row_blocks(i.n_rows, a.share, ROWS) : 0);
    }
    __syncthreads();
    // exclusive sums
    const int per = (a.q.n_seqs + blockDim.x - 1) / blockDim.x;
    const int s0 = min(a.q.n_seqs, tid * per), s1 = min(a.q.n_seqs, s0 + per);
    long long sum = 0;
    for (int s = s0; s < s1; ++s) {
        const long long n = p.offsets[s];
        p.offsets[s] = sum;
        sum += n;
    }
    long long up = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, up, o);
        if (lane >= o) up += v;
    }
    if (lane == 31) part[warp] = up;
    __syncthreads();
    long long base = up - sum, total = 0;
    for (int w = 0; w < n_warps; ++w) {
        if (w < warp) base += part[w];
        total += part[w];
    }
    for (int s = s0; s < s1; ++s) p.offsets[s] += base;
    if (tid == 0) p.offsets[a.q.n_seqs] = total;
    __syncthreads();
}

template <int ROWS>
__global__ void __launch_bounds__(1024) attn_cache_plan_kernel(AttnArgs a) {
    __shared__ long long part[32];
    make_plan<ROWS>(a, plan_at(a.plan, a.q.n_seqs), part, true);
}

// A place on the line of units: block `blk` of an item.
struct Cursor {
    int seq, kvh, rb;      // the item
    int blk, n_blk, n_rb;
};

__device__ __forceinline__ int next_head(const AttnArgs& a, const Plan& p, int seq, int from) {
    for (int w = from >> 5; w < a.plan_words; ++w) {
        uint32_t m = p.masks[seq * a.plan_words + w];
        if (w == from >> 5) m &= 0xffffffffu << (from & 31);
        if (m) return 32 * w + __ffs(m) - 1;
    }
    return -1;
}

template <int ROWS>
__device__ __forceinline__ void enter_seq(const AttnArgs& a, Cursor& k) {
    const SeqInfo i = wide_seq_info(a.q, k.seq, a.c.page_shift);
    k.n_blk = (i.len + 15) >> 4;
    k.n_rb = row_blocks(i.n_rows, a.share, ROWS);
}

template <int ROWS>
__device__ Cursor locate(const AttnArgs& a, const Plan& p, long long u) {
    Cursor k;
    int lo = 0, hi = a.q.n_seqs - 1;   // the last sequence that starts at or before u: it holds u
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.offsets[mid] <= u) lo = mid;
        else hi = mid - 1;
    }
    k.seq = lo;
    enter_seq<ROWS>(a, k);
    long long r = u - p.offsets[lo];
    const long long item = r / k.n_blk;
    k.blk = static_cast<int>(r - item * k.n_blk);
    int nth = static_cast<int>(item / k.n_rb);
    k.rb = static_cast<int>(item - static_cast<long long>(nth) * k.n_rb);
    k.kvh = next_head(a, p, lo, 0);
    for (; nth > 0; --nth) k.kvh = next_head(a, p, lo, k.kvh + 1);
    return k;
}

// to the first block of the next item; the caller knows that there is one
template <int ROWS>
__device__ __forceinline__ void next_item(const AttnArgs& a, const Plan& p, Cursor& k) {
    k.blk = 0;
    if (++k.rb < k.n_rb) return;
    k.rb = 0;
    const int h = next_head(a, p, k.seq, k.kvh + 1);
    if (h >= 0) {
        k.kvh = h;
        return;
    }
    do ++k.seq;
    while (k.seq + 1 < a.q.n_seqs && p.offsets[k.seq + 1] == p.offsets[k.seq]);
    enter_seq<ROWS>(a, k);
    k.kvh = next_head(a, p, k.seq, 0);
}

// What the epilogues need of a row of an item.
struct RowOut {
    __nv_bfloat16* o;   // nullptr: the row does not exist
    bool on;
};
__device__ __forceinline__ RowOut row_out(const AttnArgs& a, const SeqInfo& i, int kvh, int rr, int head_dim) {
    RowOut r;
    const int tok = rr / a.share, h = kvh * a.share + rr - tok * a.share;
    r.o = tok < i.n_rows ? a.o + (static_cast<size_t>(i.row0 + tok) * a.n_q + h) * head_dim : nullptr;
    r.on = r.o && (!a.mask_bits || wide_mask_bit(a.mask_bits, a.words, i.row0 + tok, h / a.hpg));
    return r;
}

__host__ __device__ constexpr int slot_floats(int rows, int D) { return rows * (D + 4); }   // rows of D values, then m and l of each

// Joins `n` partial results of one item, the e-th at at(e): out rows, or a partial again (dst).
template <int ROWS, int D, typename At>
__device__ __forceinline__ void join(const AttnArgs& a, int seq, int kvh, int rb, int n, const At& at, float* dst, int tid, int n_threads) {
    const SeqInfo info = wide_seq_info(a.q, seq, a.c.page_shift);
    for (int i = tid; i < ROWS * (D / 4); i += n_threads) {
        const int r = i / (D / 4), d = i % (D / 4) * 4;
        float m = -CUDART_INF_F;
        for (int e = 0; e < n; ++e) m = fmaxf(m, at(e)[ROWS * D + 2 * r]);
        const float m_use = m == -CUDART_INF_F ? 0.f : m;
        float l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
        for (int e = 0; e < n; ++e) {
            const float* p = at(e);
            const float w = exp2_fast(p[ROWS * D + 2 * r] - m_use);
            const float4 v = *reinterpret_cast<const float4*>(p + r * D + d);
            l = fmaf(p[ROWS * D + 2 * r + 1], w, l);
            x[0] = fmaf(v.x, w, x[0]);
            x[1] = fmaf(v.y, w, x[1]);
            x[2] = fmaf(v.z, w, x[2]);
            x[3] = fmaf(v.w, w, x[3]);
        }
        if (dst) {
            *reinterpret_cast<float4*>(dst + r * D + d) = make_float4(x[0], x[1], x[2], x[3]);
            if (d == 0) {
                dst[ROWS * D + 2 * r] = m;
                dst[ROWS * D + 2 * r + 1] = l;
            }
        } else {
            const RowOut ro = row_out(a, info, kvh, rb * ROWS + r, D);
            if (!ro.o) continue;
            const float inv = ro.on && l != 0.f ? 1.f / l : 0.f;
            uint2 w = make_uint2(0, 0);
            if (inv != 0.f) {
                const __nv_bfloat162 b0 = __floats2bfloat162_rn(x[0] * inv, x[1] * inv), b1 = __floats2bfloat162_rn(x[2] * inv, x[3] * inv);
                w = make_uint2(*reinterpret_cast<const uint32_t*>(&b0), *reinterpret_cast<const uint32_t*>(&b1));
            }
            *reinterpret_cast<uint2*>(ro.o + d) = w;
        }
    }
}

// ------------------------------------------------------------------------------------------------ the kernel
template <int D, int G, int NB, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, 1) attn_cache_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int kRows = 8 * NB;
    constexpr int kNS = D / G;
    constexpr int kSteps = D / 16;              // k16 steps of a key, m16 tiles of a value
    constexpr int kSB = 16 * D + 128 * kNS;     // bytes of a block
    constexpr int kStage = kBlk * kSB;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint64_t bars[WARPS * 8];
    __shared__ long long part[WARPS];
    __shared__ int s_abort;
    // per warp two partial results: [0] of an item that began before the piece (in global memory), [1] of the
    // piece's last item (over the ring).  state: 0 none, else 1 | begins here << 1 | ends here << 2
    __shared__ int e_state[WARPS][2], e_seq[WARPS][2], e_kvh[WARPS][2], e_rb[WARPS][2];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    unsigned char* ring = smem + kPlanSmem + static_cast<size_t>(warp) * a.stages * kStage;
    const uint32_t ring_a = smem_u32(ring), bar_a = smem_u32(&bars[warp * 8]);
    if (lane < a.stages) mbar_init(bar_a + 8 * lane, 1);
    if (tid < 2 * WARPS) e_state[tid >> 1][tid & 1] = 0;
    if (tid == 0) s_abort = 0;
    fence_barrier_init();
    const Plan plan = plan_at(a.plan ? a.plan : smem, a.q.n_seqs);
    __syncthreads();
    if (!a.plan) make_plan<kRows>(a, plan, part, blockIdx.x == 0);

    // rows that no item writes: KV heads that a sequence does not use, sequences that are left out
    for (int s = blockIdx.x; s < a.q.n_seqs; s += gridDim.x) {
        const SeqInfo i = wide_seq_info(a.q, s, a.c.page_shift);
        const int per_row = a.n_q * (D / 8);
        for (long long x = tid; x < static_cast<long long>(i.n_rows) * per_row; x += 32 * WARPS) {
            const int r = static_cast<int>(x / per_row), v = static_cast<int>(x - static_cast<long long>(r) * per_row), h = v / (D / 8) / a.share;
            if (!((plan.masks[s * a.plan_words + (h >> 5)] >> (h & 31)) & 1u))
                reinterpret_cast<uint4*>(a.o + static_cast<size_t>(i.row0 + r) * a.n_q * D)[v] = make_uint4(0, 0, 0, 0);
        }
    }

    // the line of units, cut for the CTAs that are worth using (16 units each at least) and their warps
    const long long total = plan.offsets[a.q.n_seqs];
    const long long ctas = min(static_cast<long long>(gridDim.x), (total + 15) / 16);
    const bool idle = blockIdx.x >= ctas;
    const long long c0 = idle ? 0 : total * blockIdx.x / ctas, c1 = idle ? 0 : total * (blockIdx.x + 1) / ctas;
    const long long u0 = c0 + (c1 - c0) * warp / WARPS, u1 = c0 + (c1 - c0) * (warp + 1) / WARPS;

    bool ok = true;
    if (u0 < u1) {
        Cursor ic = locate<kRows>(a, plan, u0), cc = ic;
        long long to_issue = u1 - u0, to_use = u1 - u0;
        int issued = 0, used = 0;      // stages
        uint32_t live = 0;             // kBlk bits a stage, newest lowest: which of its blocks have a page
        int pt_seq = -1, pt_first = 0, pt = 0;   // page numbers [pt_first, pt_first + 32) of sequence pt_seq, one a lane

        auto issue = [&]() {
            const int nb = static_cast<int>(min(static_cast<long long>(min(kBlk, ic.n_blk - ic.blk)), to_issue));
            if (nb <= 0) {      // only if a length changes under the running kernel
                to_issue = 0;
                return;
            }
            const int first = (ic.blk << 4) >> a.c.page_shift, last = ((ic.blk + nb - 1) << 4) >> a.c.page_shift;
            if (pt_seq != ic.seq || first < pt_first || last >= pt_first + 32) {
                pt_seq = ic.seq;
                pt_first = first;
                pt = first + lane < a.q.max_pages ? a.q.page_table[static_cast<size_t>(ic.seq) * a.q.max_pages + first + lane] : -1;
            }
            const int blk = ic.blk + min(lane, nb - 1);
            const int page = __shfl_sync(0xffffffffu, pt, ((blk << 4) >> a.c.page_shift) - pt_first);
            const bool good = static_cast<unsigned>(page) < static_cast<unsigned>(a.c.n_pages) && lane < nb;
            const uint32_t m = __ballot_sync(0xffffffffu, good);
            if (m != (1u << nb) - 1u && lane == 0) atomicExch(a.status + WIDE_STATUS_INDEX, WIDE_ERR_BAD_INDEX);
            live = (live << kBlk) | m;
            const int slot = issued % a.stages;
            const uint32_t bar = bar_a + 8 * slot;
            if (lane == 0) mbar_arrive_expect_tx(bar, __popc(m) * kSB);
            __syncwarp();
            if (good) {
                const int sub = blk & ((1 << (a.c.page_shift - 4)) - 1);
                const size_t at = (((static_cast<size_t>(page) * a.c.n_kv_heads + ic.kvh) << (a.c.page_shift - 4)) + sub) * kSB;
                bulk_load(ring_a + slot * kStage + lane * kSB, a.c.pages + at, kSB, bar);
            }
            ++issued;
            ic.blk += nb;
            to_issue -= nb;
            if (ic.blk == ic.n_blk && to_issue > 0) next_item<kRows>(a, plan, ic);
        };
        for (int s = 0; s < a.stages && to_issue > 0; ++s) issue();

        while (to_use > 0 && ok) {
            // ---- an item, or the part of it that lies in this piece
            const SeqInfo info = wide_seq_info(a.q, cc.seq, a.c.page_shift);
            const int first_blk = cc.blk;
            const int end_blk = static_cast<int>(min(static_cast<long long>(cc.n_blk), cc.blk + to_use));
            if (end_blk <= first_blk) break;
            uint32_t qf[NB][kSteps][2];
            float qsum[NB][kNS][2], qscale[NB][2];   // of this lane's score columns 2t, 2t + 1
            int last_key[NB][2];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const int rr = cc.rb * kRows + 8 * n + g, tok = rr / a.share, h = cc.kvh * a.share + rr - tok * a.share;
                uint4 w[kSteps / 2];
                float top = 0.f, sum[kNS];
                bool finite = true;
#pragma unroll
                for (int i = 0; i < kSteps / 2; ++i) {
                    w[i] = make_uint4(0, 0, 0, 0);
                    if (tok < info.n_rows)
                        w[i] = *reinterpret_cast<const uint4*>(a.qm + (info.row0 + tok) * a.qs + h * D + 32 * i + 8 * t);
                }
#pragma unroll
                for (int i = 0; i < kNS; ++i) sum[i] = 0.f;
#pragma unroll
                for (int i = 0; i < kSteps / 2; ++i) {
                    const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float lo = __uint_as_float(x[e] << 16), hi = __uint_as_float(x[e] & 0xFFFF0000u);
                        top = fmaxf(top, fmaxf(fabsf(lo), fabsf(hi)));
                        finite = finite && fabsf(lo) <= 3.4e38f && fabsf(hi) <= 3.4e38f;
                        sum[32 * i / G] += lo + hi;
                    }
                }
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    finite = __shfl_xor_sync(0xffffffffu, finite ? 1 : 0, o) && finite;
#pragma unroll
                    for (int i = 0; i < kNS; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
                }
                // the row times 2^-e has its largest number in [2^14, 2^15)
                const int e = min(100, max(-100, static_cast<int>((__float_as_uint(top) >> 23) & 255) - 127 - 14));
                const float down = pow2(-e);
#pragma unroll
                for (int i = 0; i < kSteps / 2; ++i) {
                    const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        // words 0, 1 of step 2i: channels 0, 1 and 2, 3 (whose codes come 16 times too large); 2, 3: step 2i + 1
                        const float f = (j & 1) ? down * 0.0625f : down;
                        qf[n][2 * i + (j >> 1)][j & 1] = pack_f16(__uint_as_float(x[j] << 16) * f, __uint_as_float(x[j] & 0xFFFF0000u) * f);
                    }
                }
                const float scale = finite ? pow2(e) * a.scale_log2e * 16777216.f : CUDART_NAN_F;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int src = 4 * (2 * t + c);
                    qscale[n][c] = __shfl_sync(0xffffffffu, scale, src);
#pragma unroll
                    for (int i = 0; i < kNS; ++i)
                        qsum[n][i][c] = __shfl_sync(0xffffffffu, finite ? sum[i] * a.scale_log2e : CUDART_NAN_F, src);
                    const int rc = cc.rb * kRows + 8 * n + 2 * t + c;
                    last_key[n][c] = a.causal ? min(info.len - 1, info.len - info.n_rows + rc / a.share) : info.len - 1;
                }
            }
            // keys before this are seen by every row of the item
            const int all_see = a.causal ? min(info.len, info.len - info.n_rows + cc.rb * kRows / a.share + 1) : info.len;

            float acc[NB][kSteps][4], m[NB][2], l[NB][2], pm[NB][kNS][2];
            int ev = -110;      // the exponent that the values' steps are relative to
#pragma unroll
            for (int n = 0; n < NB; ++n) {
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[n][i][e] = 0.f;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    m[n][c] = -CUDART_INF_F;
                    l[n][c] = 0.f;
#pragma unroll
                    for (int i = 0; i < kNS; ++i) pm[n][i][c] = 0.f;
                }
            }
            while (cc.blk < end_blk) {
                const int nb = min(kBlk, end_blk - cc.blk);
                const int slot = used % a.stages;
                ok = mbar_wait_warp(bar_a + 8 * slot, (used / a.stages) & 1, a.wait_ns, &s_abort);
                if (!ok) break;
                const uint32_t here = (live >> (kBlk * (issued - 1 - used))) & ((1u << kBlk) - 1u);
                const uint32_t base = ring_a + slot * kStage;
                const int key0 = cc.blk << 4;
                const bool masked = here != (1u << kBlk) - 1u || key0 + 16 * kBlk > all_see;
                // ---- scores
                float s[kBlk][NB][4];
#pragma unroll
                for (int b = 0; b < kBlk; ++b) {
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[b][n][e] = -CUDART_INF_F;
                    if (!((here >> b) & 1u)) continue;
                    const uint32_t at = base + b * kSB;
                    uint32_t w0[kNS], w1[kNS];
                    lds_words<kNS>(at + 16 * D + 4 * kNS * g, w0);
                    lds_words<kNS>(at + 16 * D + 4 * kNS * (g + 8), w1);
                    uint4 w[kSteps / 4];
#pragma unroll
                    for (int i = 0; i < kSteps / 4; ++i) w[i] = lds128(at + (i * 32 + lane) * 16);
                    float raw[NB][4], mins[NB][4];
#pragma unroll
                    for (int i = 0; i < kNS; ++i) {
                        float d[NB][4];
#pragma unroll
                        for (int n = 0; n < NB; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e) d[n][e] = 0.f;
#pragma unroll
                        for (int k = i * (G / 16); k < (i + 1) * (G / 16); ++k) {
                            const uint4 v = w[k >> 2];
                            const uint32_t x = (k & 3) == 0 ? v.x : (k & 3) == 1 ? v.y : (k & 3) == 2 ? v.z : v.w;
                            const uint32_t y = x >> 8;
#pragma unroll
                            for (int n = 0; n < NB; ++n)
                                mma_f16(d[n], x & 0x000F000Fu, y & 0x000F000Fu, x & 0x00F000F0u, y & 0x00F000F0u, qf[n][k][0], qf[n][k][1]);
                        }
                        const float s0 = wide_cache_scale(w0[i]), s1 = wide_cache_scale(w1[i]);
                        const float m0 = wide_cache_min(w0[i]), m1 = wide_cache_min(w1[i]);
#pragma unroll
                        for (int n = 0; n < NB; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float st = e < 2 ? s0 : s1, mi = e < 2 ? m0 : m1;
                                raw[n][e] = i == 0 ? d[n][e] * st : fmaf(d[n][e], st, raw[n][e]);
                                mins[n][e] = i == 0 ? mi * qsum[n][i][e & 1] : fmaf(mi, qsum[n][i][e & 1], mins[n][e]);
                            }
                    }
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[b][n][e] = fmaf(raw[n][e], qscale[n][e & 1], mins[n][e]);
                            if (masked && key0 + 16 * b + g + 8 * (e >> 1) > last_key[n][e & 1]) s[b][n][e] = -CUDART_INF_F;
                        }
                }
                // ---- steps of the values: parameters of this lane's keys, the largest exponent of the stage
                uint32_t v0[kBlk][kNS], v1[kBlk][kNS], big = 0;
#pragma unroll
                for (int b = 0; b < kBlk; ++b) {
                    const uint32_t at = base + b * kSB + 16 * D + 64 * kNS;
                    lds_words<kNS>(at + 4 * kNS * g, v0[b]);
                    lds_words<kNS>(at + 4 * kNS * (g + 8), v1[b]);
                    if (masked) {   // nothing of a position behind the end may reach a sum
                        const bool k0 = ((here >> b) & 1u) && key0 + 16 * b + g < info.len;
                        const bool k1 = ((here >> b) & 1u) && key0 + 16 * b + g + 8 < info.len;
#pragma unroll
                        for (int i = 0; i < kNS; ++i) {
                            v0[b][i] = k0 ? v0[b][i] : 0u;
                            v1[b][i] = k1 ? v1[b][i] : 0u;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kNS; ++i) {
                        const uint32_t x = v0[b][i] & 0xFFFFu, y = v1[b][i] & 0xFFFFu;
                        big = max(big, x < 0x7F80u ? x : 0u);
                        big = max(big, y < 0x7F80u ? y : 0u);
                    }
                }
                big = __reduce_max_sync(0xffffffffu, big);
                const int ev_new = max(ev, static_cast<int>(big >> 7) - 127);
                const bool ev_up = ev_new != ev;
                // ---- running maximum; what is summed so far is scaled down when it (or the exponent) rises
                float alpha[NB][2];
                bool change = ev_up;
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float mx = m[n][c];
#pragma unroll
                        for (int b = 0; b < kBlk; ++b) mx = fmaxf(mx, fmaxf(s[b][n][c], s[b][n][c + 2]));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                        change = change || mx != m[n][c];
                        alpha[n][c] = mx == m[n][c] ? 1.f : exp2_fast(m[n][c] - mx);
                        m[n][c] = mx;
                    }
                if (__any_sync(0xffffffffu, change)) {
                    const float ev_f = ev_up ? pow2(max(-126, ev - ev_new)) : 1.f;
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            l[n][c] *= alpha[n][c];
#pragma unroll
                            for (int i = 0; i < kNS; ++i) pm[n][i][c] *= alpha[n][c];
                        }
#pragma unroll
                        for (int i = 0; i < kSteps; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[n][i][e] *= alpha[n][e & 1] * ev_f;
                    }
                    ev = ev_new;
                }
                const float inv = pow2(13 - ev);
                // ---- probabilities, and the values they weigh
#pragma unroll
                for (int b = 0; b < kBlk; ++b) {
                    if (!((here >> b) & 1u)) continue;
                    float p[NB][4];
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float mx = m[n][e & 1];
                            p[n][e] = exp2_fast(s[b][n][e] - (mx == -CUDART_INF_F ? 0.f : mx));
                            l[n][e & 1] += p[n][e];
                        }
                    const uint32_t at = base + b * kSB + 8 * D;
                    uint4 w[kSteps / 4];
#pragma unroll
                    for (int i = 0; i < kSteps / 4; ++i) w[i] = lds128(at + (i * 32 + lane) * 16);
#pragma unroll
                    for (int i = 0; i < kNS; ++i) {
                        const float s0 = wide_cache_scale(v0[b][i]) * inv, s1 = wide_cache_scale(v1[b][i]) * inv;
                        const float m0 = wide_cache_min(v0[b][i]), m1 = wide_cache_min(v1[b][i]);
                        uint32_t pb[NB][2];
#pragma unroll
                        for (int n = 0; n < NB; ++n) {
                            float x[4], y[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                x[e] = p[n][e] * (e < 2 ? s0 : s1);
                                y[e] = p[n][e] * (e < 2 ? m0 : m1);
                                if (masked && s[b][n][e] == -CUDART_INF_F) x[e] = y[e] = 0.f;   // NaN steps behind the mask
                            }
                            pb[n][0] = transpose8x8(pack_f16(x[0], x[1]));
                            pb[n][1] = transpose8x8(pack_f16(x[2], x[3]));
                            pm[n][i][0] += y[0] + y[2];
                            pm[n][i][1] += y[1] + y[3];
                        }
#pragma unroll
                        for (int k = i * (G / 16); k < (i + 1) * (G / 16); ++k) {
                            const uint4 v = w[k >> 2];
                            const uint32_t x = (k & 3) == 0 ? v.x : (k & 3) == 1 ? v.y : (k & 3) == 2 ? v.z : v.w;
                            const uint32_t y = x >> 8;
#pragma unroll
                            for (int n = 0; n < NB; ++n)
                                mma_f16(acc[n][k], x & 0x000F000Fu, x & 0x00F000F0u, y & 0x000F000Fu, y & 0x00F000F0u, pb[n][0], pb[n][1]);
                        }
                    }
                }
                __syncwarp();     // every lane has read the stage
                ++used;
                cc.blk += nb;
                to_use -= nb;
                if (to_issue > 0) issue();
            }
            if (!ok) break;
            // ---- end of the item or of the piece: sums over the lanes, results in the values' own scale
            const float f0 = pow2(11) * pow2(ev), f1 = f0 * 0.0625f;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) {
                        l[n][c] += __shfl_xor_sync(0xffffffffu, l[n][c], o);
#pragma unroll
                        for (int i = 0; i < kNS; ++i) pm[n][i][c] += __shfl_xor_sync(0xffffffffu, pm[n][i][c], o);
                    }
            const bool begins = first_blk == 0, ends = end_blk == cc.n_blk;
            if (begins && ends) {
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const RowOut ro = row_out(a, info, cc.kvh, cc.rb * kRows + 8 * n + 2 * t + c, D);
                        if (!ro.o) continue;
                        const float r = ro.on && l[n][c] != 0.f ? 1.f / l[n][c] : 0.f;
#pragma unroll
                        for (int i = 0; i < kSteps / 2; ++i) {
                            const float add = pm[n][32 * i / G][c];
                            uint2 w = make_uint2(0, 0);
                            if (r != 0.f) {
                                const __nv_bfloat162 b0 = __floats2bfloat162_rn(fmaf(acc[n][2 * i][c], f0, add) * r, fmaf(acc[n][2 * i][c + 2], f1, add) * r);
                                const __nv_bfloat162 b1 = __floats2bfloat162_rn(fmaf(acc[n][2 * i + 1][c], f0, add) * r, fmaf(acc[n][2 * i + 1][c + 2], f1, add) * r);
                                w = make_uint2(*reinterpret_cast<const uint32_t*>(&b0), *reinterpret_cast<const uint32_t*>(&b1));
                            }
                            *reinterpret_cast<uint2*>(ro.o + 32 * i + 4 * g) = w;
                        }
                    }
            } else {
                const bool tail = to_use == 0;    // the ring is free now
                float* dst = tail ? reinterpret_cast<float*>(ring) : a.heads + static_cast<size_t>(blockIdx.x * WARPS + warp) * slot_floats(kRows, D);
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int r = 8 * n + 2 * t + c;
#pragma unroll
                        for (int i = 0; i < kSteps / 2; ++i) {
                            const float add = pm[n][32 * i / G][c];
                            *reinterpret_cast<float4*>(dst + r * D + 32 * i + 4 * g) =
                                make_float4(fmaf(acc[n][2 * i][c], f0, add), fmaf(acc[n][2 * i][c + 2], f1, add),
                                            fmaf(acc[n][2 * i + 1][c], f0, add), fmaf(acc[n][2 * i + 1][c + 2], f1, add));
                        }
                        if (g == 0) {
                            dst[kRows * D + 2 * r] = m[n][c];
                            dst[kRows * D + 2 * r + 1] = l[n][c];
                        }
                    }
                const int e = tail ? 1 : 0;
                if (lane == 0) {
                    e_state[warp][e] = 1 | (begins ? 2 : 0) | (ends ? 4 : 0);
                    e_seq[warp][e] = cc.seq;
                    e_kvh[warp][e] = cc.kvh;
                    e_rb[warp][e] = cc.rb;
                }
            }
            if (to_use > 0) next_item<kRows>(a, plan, cc);
        }
        if (!ok) {
            if (lane == 0) {
                atomicExch(a.status, WIDE_ERR_TIMEOUT);
                // copies may still be on their way into this CTA's shared memory
                volatile int never = 0;
                for (int i = used; i < issued; ++i) mbar_wait(bar_a + 8 * (i % a.stages), (i / a.stages) & 1, a.wait_ns, &never);
            }
            __syncwarp();
        }
    }
    __syncthreads();
    if (s_abort) return;

    // ---- join the warps' pieces of each item; what is still a piece goes to the second kernel
    int* meta = a.meta + blockIdx.x * 8;
    bool out[2] = {false, false};
    int at = 0;
    while (at < 2 * WARPS) {
        const int w = at >> 1, e = at & 1, st = e_state[w][e];
        if (!st) {
            ++at;
            continue;
        }
        // the pieces that follow, up to the one that ends the item or the CTA
        int end = st, n = 1;
        int to = at + 1;
        uint32_t which = 1u << at;
        if (!(st & 4)) {
            for (; to < 2 * WARPS; ++to) {
                const int s2 = e_state[to >> 1][to & 1];
                if (!s2) continue;
                which |= 1u << to;
                ++n;
                end = s2;
                if (s2 & 4) {
                    ++to;
                    break;
                }
            }
        }
        const bool begins = (st & 2) != 0, ends = (end & 4) != 0;
        float* dst = nullptr;
        if (!(begins && ends)) {
            const int slot = begins ? 1 : 0;
            out[slot] = true;
            dst = a.parts + static_cast<size_t>(blockIdx.x * 2 + slot) * slot_floats(kRows, D);
            if (tid == 0) {
                meta[4 * slot] = ends ? 2 : 1;
                meta[4 * slot + 1] = e_seq[w][e];
                meta[4 * slot + 2] = e_kvh[w][e];
                meta[4 * slot + 3] = e_rb[w][e];
            }
        }
        auto piece = [&](int i) -> const float* {
            uint32_t m = which;
            for (; i > 0; --i) m &= m - 1;
            const int x = __ffs(m) - 1;
            return (x & 1) ? reinterpret_cast<const float*>(smem + kPlanSmem + static_cast<size_t>(x >> 1) * a.stages * kStage)
                           : a.heads + static_cast<size_t>(blockIdx.x * WARPS + (x >> 1)) * slot_floats(kRows, D);
        };
        join<kRows, D>(a, e_seq[w][e], e_kvh[w][e], e_rb[w][e], n, piece, dst, tid, 32 * WARPS);
        at = to;
    }
    if (tid == 0) {
        if (!out[0]) meta[0] = 0;
        if (!out[1]) meta[4] = 0;
    }
}

// Items that more than one CTA had a piece of: block c joins the one that begins in CTA c and goes on in the next.
template <int ROWS, int D>
__global__ void __launch_bounds__(256) attn_cache_join_kernel(const __grid_constant__ AttnArgs a, int ctas) {
    grid_dep_wait();
    const int c = blockIdx.x;
    if (*reinterpret_cast<volatile int*>(a.status) != WIDE_OK) return;   // some CTA gave up: its pieces are not there
    const int* meta = a.meta + c * 8 + 4;
    if (meta[0] != 1) return;
    int n = 1;
    while (c + n < ctas && a.meta[(c + n) * 8] == 1) ++n;
    if (c + n < ctas) ++n;     // the piece that ends it
    auto piece = [&](int i) -> const float* {
        return a.parts + static_cast<size_t>(i == 0 ? 2 * c + 1 : 2 * (c + i)) * slot_floats(ROWS, D);
    };
    join<ROWS, D>(a, meta[1], meta[2], meta[3], n, piece, nullptr, threadIdx.x + 256 * blockIdx.y, 256 * gridDim.y);
}

constexpr int warps_of(int nb) { return nb == 1 ? 16 : 8; }

struct Work {
    size_t plan, heads, parts, meta, total;
};
Work work_layout() {
    Work w;
    size_t at = 0;
    w.plan = at;
    at += wide_align_up(plan_bytes(WIDE_MAX_SEQS, 8), 256);
    w.heads = at;
    at += wide_align_up(static_cast<size_t>(kMaxCtas) * 16 * slot_floats(8, 128) * 4, 256);
    w.parts = at;
    at += wide_align_up(static_cast<size_t>(kMaxCtas) * 2 * slot_floats(16, 128) * 4, 256);
    w.meta = at;
    at += static_cast<size_t>(kMaxCtas) * 8 * 4;
    w.total = wide_align_up(at, 256);
    return w;
}

template <int D, int G, int NB>
int launch(wide_ctx* ctx, cudaStream_t s, AttnArgs a, unsigned char* ws) {
    constexpr int W = warps_of(NB), kRows = 8 * NB;
    constexpr int stage = kBlk * (16 * D + 128 * (D / G));
    constexpr int room = 227 * 1024 - 4096 - kPlanSmem;   // 4 KB for the static arrays
    constexpr int stages = room / (W * stage) > 6 ? 6 : room / (W * stage);
    static_assert(stages >= 2 && stages * stage >= slot_floats(kRows, D) * 4, "ring");
    a.stages = stages;
    const int smem = kPlanSmem + W * stages * stage;
    const int ctas = ctx->sm_count < kMaxCtas ? ctx->sm_count : kMaxCtas;
    const Work w = work_layout();
    a.heads = reinterpret_cast<float*>(ws + w.heads);
    a.parts = reinterpret_cast<float*>(ws + w.parts);
    a.meta = reinterpret_cast<int*>(ws + w.meta);
    a.plan = nullptr;
    if (plan_bytes(a.q.n_seqs, a.plan_words) > kPlanSmem) {
        a.plan = ws + w.plan;
        WideLaunch l(ctx, s, "attn_cache_plan");
        attn_cache_plan_kernel<kRows><<<1, 1024, 0, s>>>(a);
        WIDE_CUDA_CHECK(cudaGetLastError());
    }
    WIDE_CUDA_CHECK(cudaFuncSetAttribute(attn_cache_kernel<D, G, NB, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    {
        WideLaunch l(ctx, s, "attn_cache");
        attn_cache_kernel<D, G, NB, W><<<ctas, 32 * W, smem, s>>>(a);
        WIDE_CUDA_CHECK(cudaGetLastError());
    }
    {
        WideLaunch l(ctx, s, "attn_cache_join");
        const dim3 grid(ctas, 2);
        if (ctx->prof) attn_cache_join_kernel<kRows, D><<<grid, 256, 0, s>>>(a, ctas);
        else WIDE_CUDA_CHECK(wide_launch_dependent(attn_cache_join_kernel<kRows, D>, grid, dim3(256), 0, s, a, ctas));
        WIDE_CUDA_CHECK(cudaGetLastError());
    }
    return WIDE_OK;
}

template <int NB>
int launch_shape(wide_ctx* ctx, cudaStream_t s, const AttnArgs& a, int D, int G, unsigned char* ws) {
    if (D == 128) {
        if (G == 128) return launch<128, 128, NB>(ctx, s, a, ws);
        if (G == 64) return launch<128, 64, NB>(ctx, s, a, ws);
        return launch<128, 32, NB>(ctx, s, a, ws);
    }
    if (G == 64) return launch<64, 64, NB>(ctx, s, a, ws);
    return launch<64, 32, NB>(ctx, s, a, ws);
}

}  // namespace

size_t wide_attn_cache_workspace(int rows, int n_q, int n_kv, int head_dim) {
    // the same for every call, so that a workspace taken once serves a growing batch
    (void)rows; (void)n_q; (void)n_kv; (void)head_dim;
    return work_layout().total;
}

int wide_launch_attn_cache(wide_ctx* ctx, cudaStream_t s, const wide_cache* cache, const wide_seqs* seqs, const void* q,
                           int rows, long long qs, int n_q, int hpg, const uint32_t* mask_bits, int causal, float scale,
                           void* o, void* ws) {
    AttnArgs a{};
    a.c = wide_cache_view(cache);
    a.q = wide_seq_view(seqs, rows);
    a.qm = static_cast<const __nv_bfloat16*>(q);
    a.qs = qs;
    a.n_q = n_q;
    a.share = n_q / cache->n_kv_heads;
    a.hpg = hpg;
    a.words = (n_q / hpg + 31) / 32;
    a.causal = causal;
    a.mask_bits = mask_bits;
    a.scale_log2e = scale * 1.4426950408889634f;
    a.o = static_cast<__nv_bfloat16*>(o);
    a.status = ctx->d_status;
    a.wait_ns = ctx->wait_ns;
    a.plan_words = (cache->n_kv_heads + 31) / 32;
    // Rows of a sequence and KV head: `share` where a sequence has one new row, else an average (the lengths
    // are on the device).  Above eight, 16 rows share a pass over the cache.
    const long long rows_per_head = seqs->row_start ? static_cast<long long>(rows) * a.share / seqs->n_seqs : a.share;
    if (rows_per_head <= 8) return launch_shape<1>(ctx, s, a, cache->head_dim, cache->quant_group, static_cast<unsigned char*>(ws));
    return launch_shape<2>(ctx, s, a, cache->head_dim, cache->quant_group, static_cast<unsigned char*>(ws));
}
