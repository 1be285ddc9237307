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

#include <type_traits>

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
    int* status;                   // takes WIDE_ERR_BAD_INDEX
    int plan_words;                // words of a sequence's head mask
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
// d = a * b
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
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

// Up to one 128-byte line a thread of the grid.
__device__ __forceinline__ void prefetch_l2(const void* p, size_t bytes) {
    const size_t at = (static_cast<size_t>(blockIdx.x) * blockDim.x + threadIdx.x) * 128;
    if (p && at < bytes) asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const char*>(p) + at));
}

// ------------------------------------------------------------------------------------------------ the plan
// offsets[s] = units (16-key blocks of items) of the sequences before s, masks[s] = KV heads in use.
struct Plan {
    long long* offsets;
    uint32_t *masks, *groups;
};
__device__ __forceinline__ Plan plan_at(unsigned char* p, int n_seqs, int plan_words) {
    uint32_t* m = reinterpret_cast<uint32_t*>(p + 8 * (n_seqs + 1));
    return Plan{reinterpret_cast<long long*>(p), m, m + n_seqs * plan_words};
}
size_t plan_bytes(int n_seqs, int plan_words, int words) {
    return 8 * static_cast<size_t>(n_seqs + 1) + 4 * static_cast<size_t>(n_seqs) * (plan_words + words);
}

__device__ __forceinline__ int row_blocks(int n_rows, int share, int rows_per) { return (n_rows * share + rows_per - 1) / rows_per; }

// Two rounds of loads (lengths, masks; one thread a sequence), then arithmetic.  Up to 16 new rows are looked at
// for the KV heads in use; of more rows all heads are taken.
template <int ROWS>
__device__ void make_plan(const AttnArgs& a, const Plan& p, long long* part, bool report) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
    const int per = (a.q.n_seqs + blockDim.x - 1) / blockDim.x;
    const int s0 = min(a.q.n_seqs, tid * per), s1 = min(a.q.n_seqs, s0 + per);
    for (int s = s0; s < s1; ++s) {
        const SeqInfo i = wide_seq_info(a.q, s, a.c.page_shift);
        if (i.bad && report) atomicExch(a.status, WIDE_ERR_BAD_INDEX);
        const bool some = i.n_rows > 0 && i.len > 0;
        const int looked = a.mask_bits && i.n_rows <= 16 ? i.n_rows : 0;
        for (int w = 0; w < a.words; ++w) {      // groups that any new row uses
            uint32_t m = some && looked == 0 ? 0xffffffffu : 0u;
            if (some)
                for (int r = 0; r < looked; ++r) m |= a.mask_bits[static_cast<size_t>(i.row0 + r) * a.words + w];
            p.groups[s * a.words + w] = m;
        }
        p.offsets[s] = some ? static_cast<long long>((i.len + 15) >> 4) * row_blocks(i.n_rows, a.share, ROWS) : 0;   // of one head
    }
    __syncthreads();
    for (int x = warp; x < a.q.n_seqs * a.plan_words; x += n_warps) {     // lanes are KV heads
        const int s = x / a.plan_words, w = x - s * a.plan_words, h = 32 * w + lane;
        bool any = false;
        if (h < a.c.n_kv_heads) {
            const int g1 = (h * a.share + a.share - 1) / a.hpg;
            for (int g = h * a.share / a.hpg; g <= g1; ++g) any |= (p.groups[s * a.words + (g >> 5)] >> (g & 31)) & 1u;
        }
        const uint32_t m = __ballot_sync(0xffffffffu, any);
        if (lane == 0) p.masks[x] = m;
    }
    __syncthreads();
    long long sum = 0;
    for (int s = s0; s < s1; ++s) {
        int used = 0;
        for (int w = 0; w < a.plan_words; ++w) used += __popc(p.masks[s * a.plan_words + w]);
        const long long n = p.offsets[s] * used;
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
    make_plan<ROWS>(a, plan_at(a.plan, a.q.n_seqs, a.plan_words), part, true);
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
__device__ __noinline__ Cursor locate(const AttnArgs& a, const Plan& p, long long u) {
    Cursor k;
    int lo = 0, hi = a.q.n_seqs - 1;   // the last sequence that starts at or before u: it holds u
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.offsets[mid] <= u) lo = mid;
        else hi = mid - 1;
    }
    k.seq = lo;
    enter_seq<ROWS>(a, k);
    const long long r = u - p.offsets[lo];
    int nth;
    if (r <= 0x7fffffffLL) {
        const int r32 = static_cast<int>(r), item = r32 / k.n_blk;
        k.blk = r32 - item * k.n_blk;
        nth = k.n_rb == 1 ? item : item / k.n_rb;
        k.rb = item - nth * k.n_rb;
    } else {
        const long long item = r / k.n_blk;
        k.blk = static_cast<int>(r - item * k.n_blk);
        nth = static_cast<int>(item / k.n_rb);
        k.rb = static_cast<int>(item - static_cast<long long>(nth) * k.n_rb);
    }
    k.kvh = next_head(a, p, lo, 0);
    for (; nth > 0; --nth) k.kvh = next_head(a, p, lo, k.kvh + 1);
    return k;
}

// to the first block of the next item; the caller knows that there is one
template <int ROWS>
__device__ __noinline__ void next_item(const AttnArgs& a, const Plan& p, Cursor& k) {
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

// Joins `n` partial results of one item, the e-th at at(e): out rows, or a partial again (dst).  A thread takes four
// channels of a row.  Executed once a launch, so kept short: its time is that of fetching its instructions.
template <int ROWS, int D, typename At>
__device__ __forceinline__ void join(const AttnArgs& a, int seq, int kvh, int rb, int n, const At& at, float* dst, int first, int step) {
#pragma unroll 1
    for (int i = first; i < ROWS * (D / 4); i += step) {
        const int r = i / (D / 4), d = i % (D / 4) * 4;
        float m = -CUDART_INF_F, l = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int e = 0; e < n; ++e) m = fmaxf(m, at(e)[ROWS * D + 2 * r]);
        const float m_use = m == -CUDART_INF_F ? 0.f : m;
#pragma unroll 4
        for (int e = 0; e < n; ++e) {
            const float* p = at(e);
            const float w = exp2_fast(p[ROWS * D + 2 * r] - m_use);
            const float4 v = *reinterpret_cast<const float4*>(p + r * D + d);
            l = fmaf(p[ROWS * D + 2 * r + 1], w, l);
            x = make_float4(fmaf(v.x, w, x.x), fmaf(v.y, w, x.y), fmaf(v.z, w, x.z), fmaf(v.w, w, x.w));
        }
        if (dst) {
            *reinterpret_cast<float4*>(dst + r * D + d) = x;
            if (d == 0) *reinterpret_cast<float2*>(dst + ROWS * D + 2 * r) = make_float2(m, l);
        } else {
            const SeqInfo info = wide_seq_info(a.q, seq, a.c.page_shift);
            const RowOut ro = row_out(a, info, kvh, rb * ROWS + r, D);
            if (!ro.o) continue;
            const float inv = ro.on && l != 0.f ? 1.f / l : 0.f;
            uint2 w = make_uint2(0, 0);
            if (inv != 0.f) {
                const __nv_bfloat162 b0 = __floats2bfloat162_rn(x.x * inv, x.y * inv), b1 = __floats2bfloat162_rn(x.z * inv, x.w * inv);
                w = make_uint2(*reinterpret_cast<const uint32_t*>(&b0), *reinterpret_cast<const uint32_t*>(&b1));
            }
            *reinterpret_cast<uint2*>(ro.o + d) = w;
        }
    }
}

// ------------------------------------------------------------------------------------------------ the kernel
template <int D, int G, int NB, int WARPS, int STAGES>
__global__ void __launch_bounds__(32 * WARPS, 1) attn_cache_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int kRows = 8 * NB;
    constexpr int kNS = D / G;
    constexpr int kSteps = D / 16;              // k16 steps of a key, m16 tiles of a value
    constexpr int kSB = 16 * D + 128 * kNS;     // bytes of a block
    constexpr int kStage = kBlk * kSB;
    constexpr int kPieces = (kSB + 511) / 512;  // 16-byte copies of a lane for a block
    constexpr uint32_t kFull = (1u << kBlk) - 1u;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ long long part[WARPS];
    // per warp two partial results: [0] of an item that began before the piece (in global memory), [1] of the
    // piece's last item (over the ring).  state: 0 none, else 1 | begins here << 1 | ends here << 2
    __shared__ const float* e_at[WARPS];        // the pieces of one item, at most one of a warp
    __shared__ int e_state[WARPS][2], e_seq[WARPS][2], e_kvh[WARPS][2], e_rb[WARPS][2];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    if (tid < 2 * WARPS) e_state[tid >> 1][tid & 1] = 0;
    // All CTAs together bring what the plan will lead to (masks, page table, queries) into L2 while it is made.
    prefetch_l2(a.mask_bits, static_cast<size_t>(a.q.rows) * a.words * 4);
    prefetch_l2(a.q.page_table, static_cast<size_t>(a.q.n_seqs) * a.q.max_pages * 4);
    prefetch_l2(a.qm, (static_cast<size_t>(a.q.rows - 1) * a.qs + a.n_q * D) * 2);
    const Plan plan = plan_at(a.plan ? a.plan : smem, a.q.n_seqs, a.plan_words);
    __syncthreads();
    if (!a.plan) make_plan<kRows>(a, plan, part, blockIdx.x == 0);

    // the line of units, cut for the CTAs that are worth using (16 units each at least) and their warps
    const long long total = plan.offsets[a.q.n_seqs];
    const int ctas = static_cast<int>(min(static_cast<long long>(gridDim.x), (total + 15) / 16)), cta = blockIdx.x;
    long long u0 = 0, u1 = 0;
    if (cta < ctas) {
        const long long share = total <= 0x7fffffffLL ? static_cast<int>(total) / ctas : total / ctas;
        const int more = static_cast<int>(total - share * ctas);
        const long long c0 = share * cta + min(cta, more);
        const int n = static_cast<int>(share + (cta < more ? 1 : 0));
        const int each = n / WARPS, extra = n - each * WARPS;
        u0 = c0 + each * warp + min(warp, extra);
        u1 = u0 + each + (warp < extra ? 1 : 0);
    }
    if (u0 < u1) {
        Cursor cc = locate<kRows>(a, plan, u0), ic = cc;     // used, requested
        int to_use = static_cast<int>(u1 - u0), to_issue = to_use, slot = 0;
        uint32_t live = 0;             // kBlk bits a stage, newest lowest: which of its blocks have a page
        int pt_seq = -1, pt_first = 0, pt = 0;   // page numbers [pt_first, pt_first + 32) of sequence pt_seq, one a lane
        const int sub_shift = a.c.page_shift - 4, sub_mask = (1 << sub_shift) - 1;
        const uint32_t ring_a = smem_u32(smem + kPlanSmem) + warp * (STAGES * kStage);
        const uint32_t lane16 = lane * 16, params = 16 * D + 4 * kNS * g;
        // request the next stage, up to kBlk blocks of one item, into place `to` (a group of copies even where nothing is left)
        auto issue = [&](int to) {
            uint32_t m = 0;
            if (to_issue > 0) {
                const int nb = min(min(kBlk, ic.n_blk - ic.blk), to_issue);
                const int last = (ic.blk + nb - 1) >> sub_shift;
                if (pt_seq != ic.seq || last - pt_first >= 32 || (ic.blk >> sub_shift) < pt_first) {
                    pt_seq = ic.seq;
                    pt_first = ic.blk >> sub_shift;
                    pt = pt_first + lane < a.q.max_pages ? a.q.page_table[static_cast<size_t>(ic.seq) * a.q.max_pages + pt_first + lane] : -1;
                }
#pragma unroll
                for (int b = 0; b < kBlk; ++b) {
                    if (b < nb) {
                        const int blk = ic.blk + b;
                        const int page = __shfl_sync(0xffffffffu, pt, (blk >> sub_shift) - pt_first);
                        if (static_cast<unsigned>(page) < static_cast<unsigned>(a.c.n_pages)) {
                            m |= 1u << b;
                            const unsigned char* from = a.c.pages + lane16 +
                                (((static_cast<size_t>(page) * a.c.n_kv_heads + ic.kvh) << sub_shift) + (blk & sub_mask)) * kSB;
                            const uint32_t dst = ring_a + to * kStage + b * kSB + lane16;
#pragma unroll
                            for (int i = 0; i < kPieces; ++i)
                                if (512 * (i + 1) <= kSB || lane16 + 512 * i < kSB) cp_async_16(dst + 512 * i, from + 512 * i);
                        }
                    }
                }
                if (m != (1u << max(nb, 0)) - 1u && lane == 0) atomicExch(a.status, WIDE_ERR_BAD_INDEX);
                ic.blk += nb;
                to_issue = nb > 0 ? to_issue - nb : 0;       // nb <= 0: a length changed under the running kernel
                if (ic.blk >= ic.n_blk && to_issue > 0) next_item<kRows>(a, plan, ic);
            }
            cp_async_commit();
            live = (live << kBlk) | m;
        };
#pragma unroll 1
        for (int i = 0; i < STAGES; ++i) issue(i);

        while (true) {
            // ---- an item, or the part of it that lies in this piece
            const SeqInfo info = wide_seq_info(a.q, cc.seq, a.c.page_shift);
            const int first_blk = cc.blk;
            const int end_blk = min(cc.n_blk, cc.blk + to_use);
            if (end_blk <= first_blk) break;
            uint32_t qf[NB][kSteps][2];
            float qsum[NB][kNS][2], qscale[NB][2];   // of this lane's score columns 2t, 2t + 1
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const int rr = cc.rb * kRows + 8 * n + g, tok = rr / a.share, h = cc.kvh * a.share + rr - tok * a.share;
                uint4 qw[kSteps / 2];      // 8 channels of every 32
#pragma unroll
                for (int i = 0; i < kSteps / 2; ++i) {
                    qw[i] = make_uint4(0, 0, 0, 0);
                    if (tok < info.n_rows)
                        qw[i] = *reinterpret_cast<const uint4*>(a.qm + (info.row0 + tok) * a.qs + h * D + 32 * i + 8 * t);
                }
                uint32_t top = 0;
                float sum[kNS];
#pragma unroll
                for (int i = 0; i < kNS; ++i) sum[i] = 0.f;
#pragma unroll
                for (int i = 0; i < kSteps / 2; ++i) {
                    const uint32_t x[4] = {qw[i].x, qw[i].y, qw[i].z, qw[i].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        top = max(top, max((x[e] << 16) & 0x7FFFFFFFu, x[e] & 0x7FFF0000u));   // orders NaN above all numbers
                        sum[32 * i / G] += __uint_as_float(x[e] << 16) + __uint_as_float(x[e] & 0xFFFF0000u);
                    }
                }
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
#pragma unroll
                    for (int i = 0; i < kNS; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
                }
                const bool finite = top < 0x7F800000u;
                // the row times 2^-e has its largest number in [2^14, 2^15)
                const int e = min(100, max(-100, static_cast<int>(top >> 23) - 127 - 14));
                const float down = pow2(-e);
#pragma unroll
                for (int i = 0; i < kSteps / 2; ++i) {
                    const uint32_t x[4] = {qw[i].x, qw[i].y, qw[i].z, qw[i].w};
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
                }
            }
            // keys before this are seen by every row of the item
            const int all_see = a.causal ? min(info.len, info.len - info.n_rows + cc.rb * kRows / a.share + 1) : info.len;

            float acc[NB][kSteps][4], m[NB][2], l[NB][2], pm[NB][kNS][2];
            int ev = -110;              // the exponent that the values' steps are relative to
            float inv = pow2(13 + 110);
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
            // One stage, kBlk blocks.  Masked: with blocks that are not there, or keys that some row does not see.
            auto turn = [&](auto masked_c, uint32_t here) {
                constexpr bool masked = decltype(masked_c)::value;
                const uint32_t base = ring_a + slot * kStage;
                const int key0 = cc.blk << 4;
                // ---- scores
                // (A block that is not there is computed like the others, from whatever the ring holds, and left out by
                // selection.  The blocks take turns: eight dependent instructions on one accumulator would wait for each other.)
                float s[kBlk][NB][4], mins[kBlk][NB][4];
                uint4 w[kBlk][kSteps / 4];
                uint32_t w0[kBlk][kNS], w1[kBlk][kNS];
#pragma unroll
                for (int b = 0; b < kBlk; ++b) {
#pragma unroll
                    for (int i = 0; i < kSteps / 4; ++i) w[b][i] = lds128(base + lane16 + b * kSB + i * 512);
                    lds_words<kNS>(base + params + b * kSB, w0[b]);
                    lds_words<kNS>(base + params + b * kSB + 32 * kNS, w1[b]);
                }
#pragma unroll
                for (int i = 0; i < kNS; ++i) {
                    float d[kBlk][NB][4];
#pragma unroll
                    for (int k = i * (G / 16); k < (i + 1) * (G / 16); ++k)
#pragma unroll
                        for (int b = 0; b < kBlk; ++b) {
                            const uint4 v = w[b][k >> 2];
                            const uint32_t x = (k & 3) == 0 ? v.x : (k & 3) == 1 ? v.y : (k & 3) == 2 ? v.z : v.w;
                            const uint32_t y = x >> 8;
#pragma unroll
                            for (int n = 0; n < NB; ++n) {
                                if (k == i * (G / 16))
                                    mma_f16_first(d[b][n], x & 0x000F000Fu, y & 0x000F000Fu, x & 0x00F000F0u, y & 0x00F000F0u, qf[n][k][0], qf[n][k][1]);
                                else
                                    mma_f16(d[b][n], x & 0x000F000Fu, y & 0x000F000Fu, x & 0x00F000F0u, y & 0x00F000F0u, qf[n][k][0], qf[n][k][1]);
                            }
                        }
#pragma unroll
                    for (int b = 0; b < kBlk; ++b) {
                        const float s0 = wide_cache_scale(w0[b][i]), s1 = wide_cache_scale(w1[b][i]);
                        const float m0 = wide_cache_min(w0[b][i]), m1 = wide_cache_min(w1[b][i]);
#pragma unroll
                        for (int n = 0; n < NB; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float st = e < 2 ? s0 : s1, mi = e < 2 ? m0 : m1;
                                s[b][n][e] = i == 0 ? d[b][n][e] * st : fmaf(d[b][n][e], st, s[b][n][e]);
                                mins[b][n][e] = i == 0 ? mi * qsum[n][i][e & 1] : fmaf(mi, qsum[n][i][e & 1], mins[b][n][e]);
                            }
                    }
                }
#pragma unroll
                for (int b = 0; b < kBlk; ++b)
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[b][n][e] = fmaf(s[b][n][e], qscale[n][e & 1], mins[b][n][e]);
                            if (masked) {
                                const int row = cc.rb * kRows + 8 * n + 2 * t + (e & 1);
                                const int last = a.causal ? min(info.len - 1, info.len - info.n_rows + row / a.share) : info.len - 1;
                                if (key0 + 16 * b + g + 8 * (e >> 1) > last || !((here >> b) & 1u)) s[b][n][e] = -CUDART_INF_F;
                            }
                        }
                // ---- the values' parameters, and their largest step (scales are not negative: their words compare like numbers)
                uint32_t v0[kBlk][kNS], v1[kBlk][kNS], big = 0;
#pragma unroll
                for (int b = 0; b < kBlk; ++b) {
                    lds_words<kNS>(base + params + 64 * kNS + b * kSB, v0[b]);
                    lds_words<kNS>(base + params + 96 * kNS + b * kSB, v1[b]);
#pragma unroll
                    for (int i = 0; i < kNS; ++i) {
                        if (masked) {   // nothing of a position behind the end may reach a sum
                            const bool is = (here >> b) & 1u;
                            v0[b][i] = is && key0 + 16 * b + g < info.len ? v0[b][i] : 0u;
                            v1[b][i] = is && key0 + 16 * b + g + 8 < info.len ? v1[b][i] : 0u;
                        }
                        big = max(big, max(v0[b][i] << 16, v1[b][i] << 16));
                    }
                }
                big = __reduce_max_sync(0xffffffffu, big);
                // ---- running maximum; what is summed so far is scaled down when it rises, or when the steps do
                float alpha[NB][2], mu[NB][2], top[NB][2];
                bool change = static_cast<int>(big >> 23) - 127 > ev;
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
                        top[n][c] = mx;
                        mu[n][c] = mx == -CUDART_INF_F ? 0.f : mx;
                    }
                if (__any_sync(0xffffffffu, change)) {
                    if (big >= 0x7F800000u) {   // a value that is not finite: leave it out of the scaling
                        big = 0;
#pragma unroll
                        for (int b = 0; b < kBlk; ++b)
#pragma unroll
                            for (int i = 0; i < kNS; ++i) {
                                const uint32_t x = v0[b][i] << 16, y = v1[b][i] << 16;
                                big = max(big, max(x < 0x7F800000u ? x : 0u, y < 0x7F800000u ? y : 0u));
                            }
                        big = __reduce_max_sync(0xffffffffu, big);
                    }
                    const int up = max(ev, static_cast<int>(big >> 23) - 127);
                    const float ev_f = pow2(max(-126, ev - up));
                    ev = up;
                    inv = pow2(13 - ev);
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            alpha[n][c] = exp2_fast(m[n][c] - mu[n][c]);
                            m[n][c] = top[n][c];
                            l[n][c] *= alpha[n][c];
#pragma unroll
                            for (int i = 0; i < kNS; ++i) pm[n][i][c] *= alpha[n][c];
                        }
#pragma unroll
                        for (int i = 0; i < kSteps; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[n][i][e] *= alpha[n][e & 1] * ev_f;
                    }
                }
                // ---- probabilities, and the values they weigh
#pragma unroll
                for (int b = 0; b < kBlk; ++b) {
#pragma unroll
                    for (int i = 0; i < kSteps / 4; ++i) w[b][i] = lds128(base + lane16 + 8 * D + b * kSB + i * 512);
                    float p[NB][4];
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            p[n][e] = exp2_fast(s[b][n][e] - mu[n][e & 1]);
                            l[n][e & 1] += p[n][e];
                        }
#pragma unroll
                    for (int i = 0; i < kNS; ++i) {
                        const float s0 = wide_cache_scale(v0[b][i]) * inv, s1 = wide_cache_scale(v1[b][i]) * inv;
                        const float m0 = wide_cache_min(v0[b][i]), m1 = wide_cache_min(v1[b][i]);
                        uint32_t pb[NB][2];
#pragma unroll
                        for (int n = 0; n < NB; ++n) {
                            float x[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                x[e] = p[n][e] * (e < 2 ? s0 : s1);
                                const float next = fmaf(p[n][e], e < 2 ? m0 : m1, pm[n][i][e & 1]);
                                if (masked) {   // a step or minimum that is not finite, of a key this row does not see
                                    const bool unseen = s[b][n][e] == -CUDART_INF_F;
                                    x[e] = unseen ? 0.f : x[e];
                                    pm[n][i][e & 1] = unseen ? pm[n][i][e & 1] : next;
                                } else {
                                    pm[n][i][e & 1] = next;
                                }
                            }
                            pb[n][0] = transpose8x8(pack_f16(x[0], x[1]));
                            pb[n][1] = transpose8x8(pack_f16(x[2], x[3]));
                        }
#pragma unroll
                        for (int k = i * (G / 16); k < (i + 1) * (G / 16); ++k) {
                            // Rows g take a whole byte, low code + 16 * high code: the rows g + 8, 16 * high code, come off
                            // again at the end.  That saves an instruction a word.
                            const uint4 v = w[b][k >> 2];
                            const uint32_t x = (k & 3) == 0 ? v.x : (k & 3) == 1 ? v.y : (k & 3) == 2 ? v.z : v.w;
                            const uint32_t y = __byte_perm(x, 0, 0x4341);
#pragma unroll
                            for (int n = 0; n < NB; ++n)
                                mma_f16(acc[n][k], x & 0x00FF00FFu, x & 0x00F000F0u, y, y & 0x00F000F0u, pb[n][0], pb[n][1]);
                        }
                    }
                }
                // every lane has read the stage: its place takes the next one
                __syncwarp();
                issue(slot);
                slot = slot + 1 == STAGES ? 0 : slot + 1;
            };
            auto arrived = [&]() -> uint32_t {       // the oldest stage in flight
                cp_async_wait<STAGES - 1>();
                __syncwarp();
                return (live >> (kBlk * (STAGES - 1))) & kFull;
            };
            int run = (min(end_blk, all_see >> 4) - cc.blk) & -kBlk;     // blocks that every row sees whole
            while (cc.blk < end_blk) {
                uint32_t here = arrived();
                while (run > 0 && here == kFull) {
                    turn(std::false_type{}, kFull);
                    cc.blk += kBlk;
                    run -= kBlk;
                    if (cc.blk >= end_blk) break;
                    here = arrived();
                }
                if (cc.blk >= end_blk) break;
                turn(std::true_type{}, here);
                cc.blk = min(cc.blk + kBlk, end_blk);
                run = max(0, run - kBlk);
            }
            to_use -= end_blk - first_blk;
            // ---- end of the item or of the piece: sums over the lanes, results in the values' own scale
            const float f0 = pow2(11) * pow2(ev), f1 = f0 * 0.0625f;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    acc[n][i][0] -= acc[n][i][2];
                    acc[n][i][1] -= acc[n][i][3];
                }
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
                float* dst = tail ? reinterpret_cast<float*>(smem + kPlanSmem + warp * (STAGES * kStage)) : a.heads + static_cast<size_t>(blockIdx.x * WARPS + warp) * slot_floats(kRows, D);
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
            if (to_use <= 0) break;
            next_item<kRows>(a, plan, cc);
        }
        cp_async_wait_all();
    }
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

    __syncthreads();

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
        if (tid < 2 * WARPS && ((which >> tid) & 1u)) {
            const int i = __popc(which & ((1u << tid) - 1u));
            e_at[i] = (tid & 1) ? reinterpret_cast<const float*>(smem + kPlanSmem + static_cast<size_t>(tid >> 1) * STAGES * kStage)
                                : a.heads + static_cast<size_t>(blockIdx.x * WARPS + (tid >> 1)) * slot_floats(kRows, D);
        }
        __syncthreads();
        join<kRows, D>(a, e_seq[w][e], e_kvh[w][e], e_rb[w][e], n, [&](int i) { return e_at[i]; }, dst, tid, 32 * WARPS);
        __syncthreads();
        at = to;
    }
    if (tid == 0) {
        if (!out[0]) meta[0] = 0;
        if (!out[1]) meta[4] = 0;
    }
}

// Items that more than one CTA had a piece of: block c joins the one that begins in CTA c and goes on in the next.
// A warp takes half a row's channels (a whole row of 64): lane e reads the maximum and sum of piece e.
template <int ROWS, int D>
__global__ void __launch_bounds__(256) attn_cache_join_kernel(const __grid_constant__ AttnArgs a, int ctas) {
    grid_dep_wait();
    const int c = blockIdx.x, lane = threadIdx.x & 31, unit = threadIdx.x >> 5;
    // one round of loads: what does CTA c leave open, how far does it go (CTAs c + 1, ...:
    // the first piece of each belongs to the item, up to the one that ends it)
    const int4 meta = *reinterpret_cast<const int4*>(a.meta + c * 8 + 4);
    int st = c + 1 + lane < ctas ? a.meta[(c + 1 + lane) * 8] : 0;
    if (meta.x != 1) return;
    int n = 1;
    for (int k = c + 1;;) {
        const uint32_t stop = __ballot_sync(0xffffffffu, st != 1);
        if (stop) {
            const int at = __ffs(stop) - 1;
            n += at + (__shfl_sync(0xffffffffu, st, at) == 2 ? 1 : 0);
            break;
        }
        n += 32;
        k += 32;
        st = k + lane < ctas ? a.meta[(k + lane) * 8] : 0;
    }
    const SeqInfo info = wide_seq_info(a.q, meta.y, a.c.page_shift);
    auto piece = [&](int i) -> const float* {
        return a.parts + static_cast<size_t>(i == 0 ? 2 * c + 1 : 2 * (c + i)) * slot_floats(ROWS, D);
    };
    constexpr int kHalves = D / 64;
    for (int u = unit + 8 * blockIdx.y; u < ROWS * kHalves; u += 8 * gridDim.y) {
        const int r = u / kHalves, d = u % kHalves * 64 + 2 * lane;
        const RowOut ro = row_out(a, info, meta.z, meta.w * ROWS + r, D);
        if (!ro.o) continue;
        float m = -CUDART_INF_F, l = 0.f;
        float2 x = make_float2(0.f, 0.f);
        for (int e0 = 0; e0 < n; e0 += 32) {
            const float2 ml = e0 + lane < n ? *reinterpret_cast<const float2*>(piece(e0 + lane) + ROWS * D + 2 * r) : make_float2(-CUDART_INF_F, 0.f);
            float top = ml.x;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float m_new = fmaxf(m, top), m_use = m_new == -CUDART_INF_F ? 0.f : m_new;
            const float old = exp2_fast(m - m_use), w = exp2_fast(ml.x - m_use);
            float sum = ml.y * w;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            l = fmaf(l, old, sum);
            x = make_float2(x.x * old, x.y * old);
            m = m_new;
            const int last = min(32, n - e0);
#pragma unroll 8
            for (int e = 0; e < last; ++e) {
                const float2 v = *reinterpret_cast<const float2*>(piece(e0 + e) + r * D + d);
                const float we = __shfl_sync(0xffffffffu, w, e);
                x = make_float2(fmaf(v.x, we, x.x), fmaf(v.y, we, x.y));
            }
        }
        const float inv = ro.on && l != 0.f ? 1.f / l : 0.f;
        __nv_bfloat162 b = __floats2bfloat162_rn(0.f, 0.f);
        if (inv != 0.f) b = __floats2bfloat162_rn(x.x * inv, x.y * inv);
        *reinterpret_cast<__nv_bfloat162*>(ro.o + d) = b;
    }
}

struct Work {
    size_t plan, heads, parts, meta, total;
};
Work work_layout() {
    Work w;
    size_t at = 0;
    w.plan = at;
    at += wide_align_up(plan_bytes(WIDE_MAX_SEQS, 8, 8), 256);
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
    constexpr int kRows = 8 * NB;
    constexpr int stage = kBlk * (16 * D + 128 * (D / G));
    constexpr int room = 227 * 1024 - 5120 - kPlanSmem;   // 5 KB for the static arrays
    // 16 warps have 128 registers each, which two blocks of eight query rows do not fit
    constexpr int W = NB == 2 ? 8 : 16 * 3 * stage <= room ? 16 : 12;
    constexpr int S = room / (W * stage) > 6 ? 6 : room / (W * stage);
    static_assert(S >= 3 && S * stage >= slot_floats(kRows, D) * 4, "ring");
    auto kernel = attn_cache_kernel<D, G, NB, W, S>;
    const int smem = kPlanSmem + W * S * stage;
    const int ctas = ctx->sm_count < kMaxCtas ? ctx->sm_count : kMaxCtas;
    const Work w = work_layout();
    a.heads = reinterpret_cast<float*>(ws + w.heads);
    a.parts = reinterpret_cast<float*>(ws + w.parts);
    a.meta = reinterpret_cast<int*>(ws + w.meta);
    a.plan = nullptr;
    if (plan_bytes(a.q.n_seqs, a.plan_words, a.words) > kPlanSmem) {
        a.plan = ws + w.plan;
        WideLaunch l(ctx, s, "attn_cache_plan");
        attn_cache_plan_kernel<kRows><<<1, 1024, 0, s>>>(a);
        WIDE_CUDA_CHECK(cudaGetLastError());
    }
    WIDE_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    {
        WideLaunch l(ctx, s, "attn_cache");
        kernel<<<ctas, 32 * W, smem, s>>>(a);
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
    a.status = ctx->d_status + WIDE_STATUS_INDEX;
    a.plan_words = (cache->n_kv_heads + 31) / 32;
    // Rows of a sequence and KV head: `share` where a sequence has one new row, else an average (the lengths
    // are on the device).  Above eight, 16 rows share a pass over the cache.
    const long long rows_per_head = seqs->row_start ? static_cast<long long>(rows) * a.share / seqs->n_seqs : a.share;
    if (rows_per_head <= 8) return launch_shape<1>(ctx, s, a, cache->head_dim, cache->quant_group, static_cast<unsigned char*>(ws));
    return launch_shape<2>(ctx, s, a, cache->head_dim, cache->quant_group, static_cast<unsigned char*>(ws));
}
