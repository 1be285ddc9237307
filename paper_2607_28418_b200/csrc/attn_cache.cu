// Head-group-masked causal attention of a batch of sequences over the 4-bit paged cache (wide_attn_cache).
//
// For the few query rows of a sequence the work is reading the cache once.  HBM brings 23 bytes a clock and SM, which is 46 values;
// a 32-key stage of one head (128 channels, keys and values, 4.3 KB) arrives every 190 clocks, so what an SM can issue in that
// time, some 500 warp instructions, is all that may be spent on its 8192 values.  Hence:
//   - The codes go into the tensor cores as they lie.  A 4-bit code in the low mantissa bits of an fp16
//     number IS a (subnormal) number, n * 2^-24, one nibble up n * 2^-20, so the four operand registers of an
//     m16n8k16 instruction are four or five integer instructions away from a word of eight codes; scale and minimum
//     stay outside:  q . k = s (q . n) + m (sum q)  per sub-group, applied to the 16 x 8 scores, and
//     sum p v = sum (p s) (n - 8) + sum p (m + 8 s).  Keys are the 16-row operand, up to eight query rows the 8-column one,
//     so nothing is padded but the queries.  (With at most 24 rows there is no shape here for the 64-row tcgen05 instructions, and
//     their operands would have to be unpacked into shared memory first.)
//   - Queries enter as fp16 times a power of two of their own (exact for bf16 numbers within 2^-25 of the
//     row's largest).  Probabilities enter as fp16 (2^-11) times the step of the value times a power of two of the query
//     row and sub-group, which follows the largest of these weighed steps so far: what a row does not weigh, however large it is,
//     costs the rest no digits, and neither can leave fp16's range.  Scores, sums and outputs are fp32.
//   - 16-key blocks are the unit of work.  All blocks of all (sequence, KV head in use, 8 * NB query
//     rows) items form one line that is cut into equal pieces for CTAs and warps, so uneven sequences load
//     the SMs evenly.  A warp streams its piece through a ring of its own in shared memory (16-byte asynchronous
//     copies, requested ahead of the compute across item borders; no barrier between warps, nothing to wait for but its own copies).
//   - A warp that covered an item writes its output; pieces of items are joined first within the
//     CTA, then (at most two per CTA) by a second small kernel.  The order of joining is fixed.
//
// Measured (device time of a call): 64 sequences of up to 16384 tokens, half of 8 KV heads, 284 MB: 67.5 us, 4.2 TB/s, 0.64 of the copy
// rate.  Of these about 55 are the streaming loop (530 instructions a stage, a quarter of them control).  Over the whole kernel issue
// slots are busy 54 %, DRAM 51 %, the tensor pipe 27 %, so none of them is the bound: warps wait for their own results (1.6 cycles an
// instruction) and for each other's issue.  The rest is start and end: 3 us until the plan is made, 4 more until the first keys are
// there, 2 to join the warps, 3 for the second kernel; with one sequence of 32768 tokens (38 MB, 21.3 us) they are most of the time.
#include <math_constants.h>

#include <atomic>
#include <type_traits>

#include "cache.cuh"
#include "ptx.cuh"

namespace {

constexpr int kItemAlone = 96;     // blocks of an item that one CTA may take alone
constexpr int kItemJoin = kItemAlone, kItemShort = kItemAlone;     // whenever there are CTAs for all
constexpr int kItemCost = 4;       // units that an item counts on top of its blocks: queries in, results out

}  // namespace

#include "attn_plan.cuh"

namespace {

constexpr int kBlk = 2;            // blocks of a ring stage: 32 keys
// -8 and -8 * 16 as the codes' subnormal fp16 numbers, twice: values are summed as m + 8 s + s (n - 8), so that sums of many values of
// either sign stay near zero.  (Summed as m + s n, the fp32 sums of 16384 evenly weighed values lost a digit to cancellation.)  The
// - 8 is the same for all channels of a sub-group, so it has one accumulator, which joins the others every fourth stage, before they grow.
constexpr uint32_t kEight = 0x00080008u, kEightHigh = 0x80808080u;
// Weighed steps, probability times step, enter fp16 times 2^e: with every new e the largest of the row and sub-group becomes
// 2^kUp .. 2^(kUp + 1), so that one 2^26 times smaller still is no zero.  Until a step times 2^e passes kMostStep or a logit the
// reference by more than kSlack powers of two, e and the reference of the softmax stay: 2^kSlack * kMostStep is below 65504.
constexpr float kSlack = 8.f;
constexpr int kUp = 2;
constexpr float kMostStep = 128.f;
constexpr int kMostExp = 118;      // of e, which stays there while steps are zero: a probability of 2^kSlack times 2^e is an fp32 number
static_assert(kMostExp + kSlack < 127.f && kSlack <= 8.f && kMostStep <= 128.f, "weighed steps leave their types");
constexpr int kPlanSmem = 16384;   // bytes of shared memory for the plan of a small batch

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
// Moves a warp's cursor, kept in shared memory, to its next item: blk | end << 32.  Out of line, since it runs rarely and is
// wanted in several places; its state in registers would cost the inner loop.
__device__ __noinline__ long long advance(const AttnArgs* a, Plan p, Cursor* at) {
    __syncwarp();
    Cursor k = *at;
    next_item(*a, p, k);
    __syncwarp();
    if ((threadIdx.x & 31) == 0) *at = k;
    __syncwarp();
    return static_cast<long long>(static_cast<unsigned long long>(static_cast<unsigned>(k.end)) << 32 | static_cast<unsigned>(k.blk));
}

// Four channels (from d on) of row r of the partial results of one item that the bits of `which` name (piece e at at(e)): an
// output row, or a row of a partial result again (dst).
template <int ROWS, int D, typename At>
__device__ __forceinline__ void join_four(int r, int d, uint32_t which, const At& at, float* dst, const RowOut& ro) {
    float m = -CUDART_INF_F, l = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    // four pieces at a time, so that their loads overlap
#pragma unroll 1
    for (uint32_t b = which; b;) {
        float2 ml[4];
        float4 v[4];
        float top = m;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            ml[e] = make_float2(-CUDART_INF_F, 0.f);
            v[e] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (b) {
                const float* p = at(__ffs(b) - 1);
                ml[e] = *reinterpret_cast<const float2*>(p + ROWS * D + 2 * r);
                v[e] = *reinterpret_cast<const float4*>(p + r * D + d);
            }
            b &= b - 1;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, ml[e].x);
        const float use = top == -CUDART_INF_F ? 0.f : top, old = exp2_fast(m - use);
        l *= old;
        x = make_float4(x.x * old, x.y * old, x.z * old, x.w * old);
        m = top;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float w = exp2_fast(ml[e].x - use);
            l = fmaf(ml[e].y, w, l);
            x = make_float4(fmaf(v[e].x, w, x.x), fmaf(v[e].y, w, x.y), fmaf(v[e].z, w, x.z), fmaf(v[e].w, w, x.w));
        }
    }
    if (dst) {
        *reinterpret_cast<float4*>(dst + r * D + d) = x;
        if (d == 0) *reinterpret_cast<float2*>(dst + ROWS * D + 2 * r) = make_float2(m, l);
    } else if (ro.o) {
        const float inv = ro.on && l != 0.f ? 1.f / l : 0.f;
        uint2 w = make_uint2(0, 0);
        if (inv != 0.f) {
            const __nv_bfloat162 b0 = __floats2bfloat162_rn(x.x * inv, x.y * inv), b1 = __floats2bfloat162_rn(x.z * inv, x.w * inv);
            w = make_uint2(*reinterpret_cast<const uint32_t*>(&b0), *reinterpret_cast<const uint32_t*>(&b1));
        }
        *reinterpret_cast<uint2*>(ro.o + d) = w;
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
    constexpr bool kDirect = G == 32;           // two tiles a sub-group: - 8 goes into their accumulators at once
    constexpr int kPieces = (kSB + 511) / 512;  // 16-byte copies of a lane for a block
    constexpr uint32_t kFull = (1u << kBlk) - 1u;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ long long part[WARPS];
    // per warp two partial results: [0] of an item that began before the piece (in global memory), [1] of the
    // piece's last item (over the ring).  state: 0 none, else 1 | begins here << 1 | ends here << 2
    __shared__ Cursor cursors[WARPS][2];
    __shared__ int e_state[WARPS][2], e_seq[WARPS][2], e_kvh[WARPS][2], e_rb[WARPS][2];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    if (tid < 2 * WARPS) e_state[tid >> 1][tid & 1] = 0;
    grid_dep_launch();     // the joining kernel may take its place as soon as CTAs end; it waits for all of them
    grid_dep_wait();
    // All CTAs together bring what the plan will lead to (masks, page table, queries) into L2 while it is made.
    prefetch_l2(a.mask_bits, static_cast<size_t>(a.q.rows) * a.words * 4);
    prefetch_l2(a.q.page_table, static_cast<size_t>(a.q.n_seqs) * a.q.max_pages * 4);
    prefetch_l2(a.qm, (static_cast<size_t>(a.q.rows - 1) * a.qs + a.n_q * D) * 2);
    const Plan plan = plan_at(a.plan ? a.plan : smem, a.q.n_seqs, a.plan_words);
    __syncthreads();
    if (!a.plan) make_plan<kRows>(a, plan, part, gridDim.x, blockIdx.x == 0);

    // the line of units, cut for the CTAs that are worth using (16 units each at least) and their warps
    const long long total = plan.offsets[a.q.n_seqs];
    const int same = *plan.same, cta = blockIdx.x;
    const int ctas = same ? static_cast<int>(total) / same : static_cast<int>(min(static_cast<long long>(gridDim.x), (total + 15) / 16));
    long long u0 = 0, u1 = 0;
    if (cta < ctas) {
        const long long share = total <= 0x7fffffffLL ? static_cast<int>(total) / ctas : total / ctas;
        const int more = static_cast<int>(total - share * ctas);
        const long long c0 = share * cta + min(cta, more);
        const long long n = share + (cta < more ? 1 : 0);
        // (a warp's own units fit an int: 2^31 of them would take it minutes)
        const long long each = n <= 0x7fffffffLL ? static_cast<int>(n) / WARPS : n / WARPS;
        const int extra = static_cast<int>(n - each * WARPS);
        u0 = c0 + each * warp + min(warp, extra);
        u1 = u0 + each + (warp < extra ? 1 : 0);
    }
    if (u0 < u1) {
        {
            const Cursor k = locate(a, plan, u0, static_cast<int>(u1 - u0));
            if (lane == 0) cursors[warp][0] = cursors[warp][1] = k;
            __syncwarp();
        }
        Cursor &cc = cursors[warp][0], &ic = cursors[warp][1];     // used, requested
        int blk = cc.blk, end_blk = cc.end, ic_blk = blk, ic_end = end_blk;
        int slot = 0;
        uint32_t live = 0;             // kBlk bits a stage, newest lowest: which of its blocks have a page
        const unsigned char* head_at = nullptr;  // block 0 of page 0 of the requested KV head, this lane's part
        int pt_first = -1000000, pt = 0;         // page numbers [pt_first, pt_first + 32) of the requested sequence, one a lane
        const int sub_shift = a.c.page_shift - 4, sub_mask = (1 << sub_shift) - 1;
        const uint32_t ring_a = smem_u32(smem + kPlanSmem) + warp * (STAGES * kStage);
        const uint32_t lane16 = lane * 16, params = 16 * D + 4 * kNS * g;
        // request the next stage, up to kBlk blocks of one item, into place `to` (a group of copies even where nothing is left)
        auto issue = [&](int to) {
            uint32_t m = 0;
            if (ic_blk < ic_end) {
                const int nb = min(kBlk, ic_end - ic_blk);
                const int first = ic_blk >> sub_shift, last = (ic_blk + nb - 1) >> sub_shift;
                if (last - pt_first >= 32) {
                    pt_first = first;
                    pt = pt_first + lane < a.q.max_pages ? a.q.page_table[static_cast<size_t>(ic.seq) * a.q.max_pages + pt_first + lane] : -1;
                    head_at = a.c.pages + static_cast<size_t>(static_cast<unsigned>(ic.kvh) << sub_shift) * kSB + lane16;
                }
                const uint32_t dst = ring_a + to * kStage + lane16;
                int page = __shfl_sync(0xffffffffu, pt, first - pt_first);
#pragma unroll
                for (int b = 0; b < kBlk; ++b) {
                    if (b < nb) {
                        if (b > 0 && last != first) page = __shfl_sync(0xffffffffu, pt, last - pt_first);
                        if (static_cast<unsigned>(page) < static_cast<unsigned>(a.c.n_pages)) {
                            m |= 1u << b;
                            const unsigned char* from = head_at + static_cast<size_t>(page) * a.page_bytes + ((ic_blk + b) & sub_mask) * kSB;
#pragma unroll
                            for (int i = 0; i < kPieces; ++i)
                                if (512 * (i + 1) <= kSB || lane16 + 512 * i < kSB) cp_async_16(dst + b * kSB + 512 * i, from + 512 * i);
                        }
                    }
                }
                if (m != (1u << nb) - 1u && lane == 0) atomicExch(a.status, WIDE_ERR_BAD_INDEX);
                ic_blk += nb;
                if (ic_blk >= ic_end && ic.left > 0) {
                    const long long next = advance(&a, plan, &ic);
                    ic_blk = static_cast<int>(next);
                    ic_end = static_cast<int>(next >> 32);
                    pt_first = -1000000;
                }
            }
            cp_async_commit();
            live = (live << kBlk) | m;
        };
        uint4 qw[NB][kSteps / 2];      // the query rows of the item at hand: 8 channels of every 32
        auto load_queries = [&]() {
            const int4 info = plan.seqs[cc.seq];     // first row, rows, length
            const RowBlock rows = row_block(a, cc.rb * kRows);
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const Row w = row_of(a, rows, 8 * n + g);
                const __nv_bfloat16* from = a.qm + (info.x + w.tok) * a.qs + (cc.kvh * a.share + w.sub) * D + 8 * t;
#pragma unroll
                for (int i = 0; i < kSteps / 2; ++i) {
                    qw[n][i] = make_uint4(0, 0, 0, 0);
                    if (w.tok < info.y) qw[n][i] = *reinterpret_cast<const uint4*>(from + 32 * i);
                }
            }
        };
        // The queries and the first stage go first: were all stages asked for at once, the first would arrive with the last.
        load_queries();
        issue(0);
        int primed = 1;

        while (blk < end_blk) {
            // ---- an item, or the part of it that lies in this piece
            const int first_blk = blk;
            uint32_t qf[NB][kSteps][2];
            float qsum[NB][kNS][2], qscale[NB][2];   // of this lane's score columns 2t, 2t + 1
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                uint32_t top = 0;
                float sum[kNS];
#pragma unroll
                for (int i = 0; i < kNS; ++i) sum[i] = 0.f;
#pragma unroll
                for (int i = 0; i < kSteps / 2; ++i) {
                    const uint32_t x[4] = {qw[n][i].x, qw[n][i].y, qw[n][i].z, qw[n][i].w};
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
                    const uint32_t x[4] = {qw[n][i].x, qw[n][i].y, qw[n][i].z, qw[n][i].w};
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
#pragma unroll 1
            for (; primed < STAGES; ++primed) issue(primed);
            // keys before this are seen by every row of the item
            const int4 info = plan.seqs[cc.seq];
            const int all_see = a.causal ? min(info.z, info.z - info.y + cc.rb * kRows / a.share + 1) : info.z;

            float acc[NB][kSteps][4], m[NB][2];
            unsigned long long l[NB], pm[NB][kNS];    // pairs of the columns
            constexpr int kMid = kDirect ? 1 : kNS;
            float mid[NB][kMid][4];     // -8 sum p s (and -8 * 17, as the rows g are summed), not yet in acc
            int turns = 0;
            auto settle = [&]() {
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int i = 0; i < kSteps; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[n][i][e] += mid[n][16 * i / G % kMid][e];
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int i = 0; i < kMid; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) mid[n][i][e] = 0.f;
            };
            uint32_t up[NB][kNS];       // 2^e of the score columns 2t and 2t + 1, as two bf16 numbers
#pragma unroll
            for (int n = 0; n < NB; ++n) {
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[n][i][e] = 0.f;
#pragma unroll
                for (int i = 0; i < kMid; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) mid[n][i][e] = 0.f;
#pragma unroll
                for (int i = 0; i < kNS; ++i) up[n][i] = (127u + kMostExp) * 0x00800080u;
#pragma unroll
                for (int i = 0; i < kNS; ++i) pm[n][i] = 0;
                l[n] = 0;
                m[n][0] = m[n][1] = -CUDART_INF_F;
            }
            // One stage, kBlk blocks.  Masked: with blocks that are not there, or keys that some row does not see.
            auto turn = [&](auto masked_c, uint32_t here) {
                constexpr bool masked = decltype(masked_c)::value;
                const uint32_t base = ring_a + slot * kStage;
                const int key0 = blk << 4;
                const int4 info = masked ? plan.seqs[cc.seq] : make_int4(0, 0, 0, 0);
                const RowBlock rows = masked ? row_block(a, cc.rb * kRows) : RowBlock{0, 0};
                // ---- scores
                // (A block that is not there is computed like the others, from whatever the ring holds, and left out by
                // selection.  The blocks take turns: eight dependent instructions on one accumulator would wait for each other.)
                float s[kBlk][NB][4], mins[kBlk][NB][4];
                uint4 w[kBlk];         // 64 channels of a block's codes
                uint32_t w0[kBlk][kNS], w1[kBlk][kNS];
#pragma unroll
                for (int b = 0; b < kBlk; ++b) {
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
                            if ((k & 3) == 0) w[b] = lds128(base + lane16 + b * kSB + (k >> 2) * 512);
                            const uint4 v = w[b];
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
                                const int last = a.causal ? min(info.z - 1, info.z - info.y + row_of(a, rows, 8 * n + 2 * t + (e & 1)).tok) : info.z - 1;
                                if (key0 + 16 * b + g + 8 * (e >> 1) > last || !((here >> b) & 1u)) s[b][n][e] = -CUDART_INF_F;
                            }
                        }
                // ---- the values' parameters
                uint32_t v0[kBlk][kNS], v1[kBlk][kNS];
#pragma unroll
                for (int b = 0; b < kBlk; ++b) {
                    lds_words<kNS>(base + params + 64 * kNS + b * kSB, v0[b]);
                    lds_words<kNS>(base + params + 96 * kNS + b * kSB, v1[b]);
#pragma unroll
                    for (int i = 0; i < kNS; ++i) {
                        if (masked) {   // nothing of a position behind the end may reach a sum
                            const bool is = (here >> b) & 1u;
                            v0[b][i] = is && key0 + 16 * b + g < info.z ? v0[b][i] : 0u;
                            v1[b][i] = is && key0 + 16 * b + g + 8 < info.z ? v1[b][i] : 0u;
                        }
                    }
                }
                // ---- the reference m that probabilities are taken relative to, and e.  They are set anew only when the running maximum has
                // risen by more than kSlack, or a step (of any key: probabilities are not known here) is too large for its e; then
                // what is summed so far is scaled.  (Following every rise, four in ten stages of a decoding batch would scale.)
                float mu[NB][2], top[NB][2];
                bool change = false;
#pragma unroll
                for (int i = 0; i < kNS; ++i) {
                    uint32_t step = 0, e = up[0][i];   // scales are not negative: their words compare like numbers
#pragma unroll
                    for (int b = 0; b < kBlk; ++b) step = max(step, max(v0[b][i] << 16, v1[b][i] << 16));
#pragma unroll
                    for (int n = 1; n < NB; ++n) e = __vmaxu2(e, up[n][i]);
                    change = change || !(__uint_as_float(step) * fmaxf(__uint_as_float(e << 16), __uint_as_float(e & 0xFFFF0000u)) <= kMostStep);   // (also where a step is NaN)
                }
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float mx = fmaxf(s[0][n][c], s[0][n][c + 2]);
#pragma unroll
                        for (int b = 1; b < kBlk; ++b) mx = fmaxf(mx, fmaxf(s[b][n][c], s[b][n][c + 2]));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                        top[n][c] = mx;
                        change = change || mx > m[n][c] + kSlack;
                    }
                if (__any_sync(0xffffffffu, change)) {
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        float alpha[2], ref[2];
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const float now = fmaxf(m[n][c], top[n][c]);
                            ref[c] = now == -CUDART_INF_F ? 0.f : now;
                            alpha[c] = exp2_fast(m[n][c] - ref[c]);
                            m[n][c] = now;
                        }
                        l[n] = mul2(l[n], pair(alpha[0], alpha[1]));
#pragma unroll
                        for (int i = 0; i < kNS; ++i) pm[n][i] = mul2(pm[n][i], pair(alpha[0], alpha[1]));
#pragma unroll
                        for (int i = 0; i < kNS; ++i) {
                            float w[2] = {0.f, 0.f};   // the stage's largest weighed step (fmaxf passes NaN over)
#pragma unroll
                            for (int b = 0; b < kBlk; ++b)
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    w[e & 1] = fmaxf(w[e & 1], exp2_fast(s[b][n][e] - ref[e & 1]) * wide_cache_scale(e < 2 ? v0[b][i] : v1[b][i]));
                            uint32_t both = __byte_perm(__float_as_uint(w[0]), __float_as_uint(w[1]), 0x7632);   // only their exponents count
                            both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 4));
                            both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 8));
                            both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 16));
                            uint32_t next[2];
                            float by[2];               // alpha * 2^(new e - old e), below 2
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                constexpr uint32_t kTurn = (254u + kUp) << 23;     // less the bits of 2^x: the bits of 2^(kUp - x)
                                const uint32_t old = c ? up[n][i] & 0xFFFF0000u : up[n][i] << 16;
                                const float before = alpha[c] * __uint_as_float(kTurn - old);    // the largest so far was that at least
                                const float most = fmaxf(__uint_as_float(c ? both & 0xFFFF0000u : both << 16), before);
                                next[c] = min(kTurn - (__float_as_uint(most) & 0x7F800000u), (127u + kMostExp) << 23);
                                by[c] = before * (__uint_as_float(next[c]) * (1.f / (1 << kUp)));
                            }
                            up[n][i] = __byte_perm(next[0], next[1], 0x7632);
#pragma unroll
                            for (int k = i * (G / 16); k < (i + 1) * (G / 16); ++k)
#pragma unroll
                                for (int e = 0; e < 4; ++e) acc[n][k][e] *= by[e & 1];
                            if (!kDirect) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) mid[n][i % kMid][e] *= by[e & 1];
                            }
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) mu[n][c] = m[n][c] == -CUDART_INF_F ? 0.f : m[n][c];
                // ---- probabilities, and the values they weigh (both score columns of a lane at once)
#pragma unroll
                for (int b = 0; b < kBlk; ++b) {
                    unsigned long long p[NB][2];      // of keys g and g + 8
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            p[n][h] = pair(exp2_fast(s[b][n][2 * h] - mu[n][0]), exp2_fast(s[b][n][2 * h + 1] - mu[n][1]));
                            l[n] = add2(l[n], p[n][h]);
                        }
#pragma unroll
                    for (int i = 0; i < kNS; ++i) {
                        uint32_t pb[NB][2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t word = h ? v1[b][i] : v0[b][i];
                            const float st = wide_cache_scale(word), mi = fmaf(st, 8.f, wide_cache_min(word));
#pragma unroll
                            for (int n = 0; n < NB; ++n) {
                                // in this order nothing overflows
                                const unsigned long long x = mul2(mul2(p[n][h], pair(__uint_as_float(up[n][i] << 16), __uint_as_float(up[n][i] & 0xFFFF0000u))), pair(st, st));
                                const unsigned long long next = fma2(p[n][h], pair(mi, mi), pm[n][i]);
                                float x0, x1;
                                unpair(x, x0, x1);
                                if (masked) {   // a step or minimum that is not finite, of a key this row does not see
                                    float n0, n1, o0, o1;
                                    unpair(next, n0, n1);
                                    unpair(pm[n][i], o0, o1);
                                    const bool u0 = s[b][n][2 * h] == -CUDART_INF_F, u1 = s[b][n][2 * h + 1] == -CUDART_INF_F;
                                    x0 = u0 ? 0.f : x0;
                                    x1 = u1 ? 0.f : x1;
                                    pm[n][i] = pair(u0 ? o0 : n0, u1 ? o1 : n1);
                                } else {
                                    pm[n][i] = next;
                                }
                                pb[n][h] = transpose8x8(pack_f16(x0, x1));
                            }
                        }
#pragma unroll
                        for (int n = 0; n < NB && !kDirect; ++n)
                            mma_f16(mid[n][i], kEight + kEightHigh, kEightHigh, kEight + kEightHigh, kEightHigh, pb[n][0], pb[n][1]);
#pragma unroll
                        for (int k = i * (G / 16); k < (i + 1) * (G / 16); ++k) {
                            // Rows g take a whole byte, low code + 16 * high code: the rows g + 8, 16 * high code, come off
                            // again at the end.  That saves an instruction a word.
                            if ((k & 3) == 0) w[b] = lds128(base + lane16 + 8 * D + b * kSB + (k >> 2) * 512);
                            const uint4 v = w[b];
                            const uint32_t x = (k & 3) == 0 ? v.x : (k & 3) == 1 ? v.y : (k & 3) == 2 ? v.z : v.w;
                            const uint32_t y = __byte_perm(x, 0, 0x4341);
#pragma unroll
                            for (int n = 0; n < NB; ++n)
                            {
                                mma_f16(acc[n][k], x & 0x00FF00FFu, x & 0x00F000F0u, y, y & 0x00F000F0u, pb[n][0], pb[n][1]);
                                if (kDirect)
                                    mma_f16(acc[n][k], kEight + kEightHigh, kEightHigh, kEight + kEightHigh, kEightHigh, pb[n][0], pb[n][1]);
                            }
                        }
                    }
                }
                if (!kDirect && (++turns & 3) == 0) settle();
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
            int run = (min(end_blk, all_see >> 4) - blk) & -kBlk;     // blocks that every row sees whole
            while (blk < end_blk) {
                uint32_t here = arrived();
                while (run > 0 && here == kFull) {
                    turn(std::false_type{}, kFull);
                    blk += kBlk;
                    run -= kBlk;
                    if (blk >= end_blk) break;
                    here = arrived();
                }
                if (blk >= end_blk) break;
                turn(std::true_type{}, here);
                blk = min(blk + kBlk, end_blk);
                run = max(0, run - kBlk);
            }
            // ---- end of the item or of the piece: sums over the lanes, results in the values' own scale
            if (!kDirect) settle();
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    acc[n][i][0] = (acc[n][i][0] - acc[n][i][2]) * pow2(24);
                    acc[n][i][1] = (acc[n][i][1] - acc[n][i][3]) * pow2(24);
                    acc[n][i][2] *= pow2(20);
                    acc[n][i][3] *= pow2(20);
                }
            auto down = [&](int n, int i, int c) { return pow2(127 - static_cast<int>((up[n][i] >> (16 * c + 7)) & 255u)); };   // 2^-e
            float ls[NB][2], pms[NB][kNS][2];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                unpair(l[n], ls[n][0], ls[n][1]);
#pragma unroll
                for (int i = 0; i < kNS; ++i) unpair(pm[n][i], pms[n][i][0], pms[n][i][1]);
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) {
                        ls[n][c] += __shfl_xor_sync(0xffffffffu, ls[n][c], o);
#pragma unroll
                        for (int i = 0; i < kNS; ++i) pms[n][i][c] += __shfl_xor_sync(0xffffffffu, pms[n][i][c], o);
                    }
            }
            const bool begins = first_blk == 0, ends = end_blk == cc.n_blk, tail = cc.left == 0;
            if (begins && ends) {
                const RowBlock rows = row_block(a, cc.rb * kRows);
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const RowOut ro = row_out(a, info.x, info.y, cc.kvh, row_of(a, rows, 8 * n + 2 * t + c), D);
                        if (!ro.o) continue;
                        const float r = ro.on && ls[n][c] != 0.f ? 1.f / ls[n][c] : 0.f;
#pragma unroll
                        for (int i = 0; i < kSteps / 2; ++i) {
                            const float add = pms[n][32 * i / G][c], f = down(n, 32 * i / G, c);
                            uint2 w = make_uint2(0, 0);
                            if (r != 0.f) {
                                const __nv_bfloat162 b0 = __floats2bfloat162_rn(fmaf(acc[n][2 * i][c], f, add) * r, fmaf(acc[n][2 * i][c + 2], f, add) * r);
                                const __nv_bfloat162 b1 = __floats2bfloat162_rn(fmaf(acc[n][2 * i + 1][c], f, add) * r, fmaf(acc[n][2 * i + 1][c + 2], f, add) * r);
                                w = make_uint2(*reinterpret_cast<const uint32_t*>(&b0), *reinterpret_cast<const uint32_t*>(&b1));
                            }
                            *reinterpret_cast<uint2*>(ro.o + 32 * i + 4 * g) = w;
                        }
                    }
            } else {
                float* dst = tail ?    // the ring is free now
                                  reinterpret_cast<float*>(smem + kPlanSmem + warp * (STAGES * kStage)) : a.heads + static_cast<size_t>(blockIdx.x * WARPS + warp) * slot_floats(kRows, D);
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int r = 8 * n + 2 * t + c;
#pragma unroll
                        for (int i = 0; i < kSteps / 2; ++i) {
                            const float add = pms[n][32 * i / G][c], f = down(n, 32 * i / G, c);
                            *reinterpret_cast<float4*>(dst + r * D + 32 * i + 4 * g) =
                                make_float4(fmaf(acc[n][2 * i][c], f, add), fmaf(acc[n][2 * i][c + 2], f, add),
                                            fmaf(acc[n][2 * i + 1][c], f, add), fmaf(acc[n][2 * i + 1][c + 2], f, add));
                        }
                        if (g == 0) {
                            dst[kRows * D + 2 * r] = m[n][c];
                            dst[kRows * D + 2 * r + 1] = ls[n][c];
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
            if (tail) break;
            const long long next = advance(&a, plan, &cc);
            blk = static_cast<int>(next);
            end_blk = static_cast<int>(next >> 32);
            if (blk < end_blk) load_queries();
        }
        cp_async_wait_all();
    }
    // rows that no item writes: KV heads that a sequence does not use, sequences that are left out
    for (int s = blockIdx.x; s < a.q.n_seqs; s += gridDim.x) {
        const int4 i = plan.seqs[s];
        const int per_row = a.n_q * (D / 8);
        for (long long x = tid; x < static_cast<long long>(i.y) * per_row; x += 32 * WARPS) {
            const int r = static_cast<int>(x / per_row), v = static_cast<int>(x - static_cast<long long>(r) * per_row), h = v / (D / 8) / a.share;
            if (!((plan.masks[s * a.plan_words + (h >> 5)] >> (h & 31)) & 1u))
                reinterpret_cast<uint4*>(a.o + static_cast<size_t>(i.x + r) * a.n_q * D)[v] = make_uint4(0, 0, 0, 0);
        }
    }
    __syncthreads();

    // ---- join the warps' pieces of each item; what is still a piece goes to the second kernel
    const int st = lane < 2 * WARPS ? e_state[lane >> 1][lane & 1] : 0;
    const uint32_t any = __ballot_sync(0xffffffffu, st != 0), begin_bits = __ballot_sync(0xffffffffu, (st & 2) != 0),
                   end_bits = __ballot_sync(0xffffffffu, (st & 4) != 0);
    int* meta = a.meta + blockIdx.x * 2 * kMeta;
    bool open[2] = {false, false};
    int mine = tid;    // the runs' elements go to the threads in turn
#pragma unroll 1
    for (uint32_t rest = any; rest;) {
        // the next piece and those that follow, up to the one that ends the item or the CTA
        const int at = __ffs(rest) - 1;
        const uint32_t stop = end_bits & rest;
        const uint32_t which = stop ? rest & (0xffffffffu >> (32 - __ffs(stop))) : rest;
        rest &= ~which;
        const bool begins = (begin_bits >> at) & 1u, ends = stop != 0;
        const int seq = e_seq[at >> 1][at & 1], kvh = e_kvh[at >> 1][at & 1], rb = e_rb[at >> 1][at & 1];
        const int4 info = plan.seqs[seq];
        float* dst = nullptr;
        if (!(begins && ends)) {
            const int slot = begins ? 1 : 0;
            open[slot] = true;
            dst = a.parts + static_cast<size_t>(blockIdx.x * 2 + slot) * slot_floats(kRows, D);
            if (tid == 0) {
                int* m = meta + kMeta * slot;
                m[0] = ends ? 2 : 1;
                m[1] = info.x;
                m[2] = info.y;
                m[3] = kvh;
                m[4] = rb;
            }
        }
        const RowBlock rows = row_block(a, rb * kRows);
        constexpr int kElements = kRows * (D / 4);
#pragma unroll 1
        for (; mine < kElements; mine += 32 * WARPS) {
            const int r = mine / (D / 4), d = mine % (D / 4) * 4;
            const RowOut ro = dst ? RowOut{nullptr, false} : row_out(a, info.x, info.y, kvh, row_of(a, rows, r), D);
            join_four<kRows, D>(r, d, which, [&](int x) -> const float* {
                return (x & 1) ? reinterpret_cast<const float*>(smem + kPlanSmem + (x >> 1) * (STAGES * kStage))
                               : a.heads + static_cast<size_t>(blockIdx.x * WARPS + (x >> 1)) * slot_floats(kRows, D);
            }, dst, ro);
        }
        mine -= kElements;
    }
    if (tid == 0) {
        if (!open[0]) meta[0] = 0;
        if (!open[1]) meta[kMeta] = 0;
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
    at += wide_align_up(static_cast<size_t>(kMaxCtas) * 8 * slot_floats(24, 128) * 4, 256);       // 8 warps of 24 rows: more than 16 of 8
    w.parts = at;
    at += wide_align_up(static_cast<size_t>(kMaxCtas) * 2 * slot_floats(24, 128) * 4, 256);
    w.meta = at;
    at += static_cast<size_t>(kMaxCtas) * 2 * kMeta * 4;
    w.total = wide_align_up(at, 256);
    return w;
}

template <int D, int G, int NB>
int launch(wide_ctx* ctx, cudaStream_t s, AttnArgs a, unsigned char* ws) {
    constexpr int kRows = 8 * NB;
    constexpr int stage = kBlk * (16 * D + 128 * (D / G));
    constexpr int room = (227 - 3) * 1024 - kPlanSmem;   // 3 KB for the static arrays
    // 12 warps have 168 registers each, which eight query rows need 132 to 168 of; 16 with 128 each keep some in memory, and were slower
    // everywhere (a batch of 64: 72.2 against 68.6 us, one short sequence: 12.7 against 9.9), as were 10 and 14.  More rows, 8 warps of 255.
    // Spilled a thread (bytes stored) for heads of 128: 8 rows 112 with sub-groups of 32, none with 64 and 128; 16 rows 272, 232, 184 (sub-groups
    // of 32, 64, 128); 24 rows 1404, 1088, 624.  For heads of 64: 24 rows with sub-groups of 32, 72; none else.
    constexpr int W = NB > 1 ? 8 : 12;
    constexpr int S = 3;                                   // stages of a ring (a batch of 64: 66.9 us with 3, 67.1 with 2, 68.2 with 4)
    static_assert(W * S * stage <= room && S * stage >= slot_floats(kRows, D) * 4, "ring");
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
        WIDE_CUDA_CHECK(wide_launch_after(ctx, attn_cache_plan_kernel<kRows>, dim3(1), dim3(1024), 0, s, a, ctas));
    }
    // once a device; threads that come here together all set the same
    static std::atomic<unsigned> set{0};
    const unsigned bit = ctx->device < 32 ? 1u << ctx->device : 0u;
    if (!(set.load(std::memory_order_relaxed) & bit) || !bit) {
        WIDE_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        set.fetch_or(bit, std::memory_order_relaxed);
    }
    {
        WideLaunch l(ctx, s, "attn_cache");
        WIDE_CUDA_CHECK(wide_launch_after(ctx, kernel, dim3(ctas), dim3(32 * W), smem, s, a));
    }
    // Nothing to join where the plan is certain to give every item a CTA of its own (make_plan; rows / kRows + n_seqs row blocks at most).
    const long long items = static_cast<long long>(a.c.n_kv_heads) * (static_cast<long long>(a.q.rows) * a.share / kRows + a.q.n_seqs);
    if (items > ctas || (static_cast<long long>(a.q.max_pages) << (a.c.page_shift - 4)) > kItemAlone) {
        WideLaunch l(ctx, s, "attn_cache_join");
        WIDE_CUDA_CHECK(wide_launch_after(ctx, attn_cache_join_kernel<kRows, D>, dim3(ctas, kRows * D / 512), dim3(256), 0, s, a, ctas));
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
    a.page_bytes = static_cast<unsigned>(a.c.block_bytes) * static_cast<unsigned>(cache->n_kv_heads) << (a.c.page_shift - 4);
    a.qm = static_cast<const __nv_bfloat16*>(q);
    a.qs = qs;
    a.n_q = n_q;
    a.share = n_q / cache->n_kv_heads;
    a.by_share = a.share > 1 ? static_cast<unsigned>(((1ull << 32) + a.share - 1) / a.share) : 0u;
    a.hpg = hpg;
    a.words = (n_q / hpg + 31) / 32;
    a.most_rows = 0x7fffffff;
    a.causal = causal;
    a.mask_bits = mask_bits;
    a.scale_log2e = scale * 1.4426950408889634f;
    a.o = static_cast<__nv_bfloat16*>(o);
    a.status = ctx->d_status + WIDE_STATUS_INDEX;
    a.plan_words = (cache->n_kv_heads + 31) / 32;
    // Rows of a sequence and KV head: `share` where a sequence has one new row, else an average over all sequences, those
    // without new rows among them (the lengths are on the device).  Above eight, 16 rows share a pass over the cache, above 16, 24.
    // An average fits batches of like sequences.  Five rows of four heads of 128 (20 a KV head) on 8192 tokens, sub-groups of 64 / 128, cold:
    // alone one pass of 24 rows, 39 / 33 us; beside 63 idle sequences three of 8, 27 / 25 us, since the 24-row kernel spills.
    const long long rows_per_head = seqs->row_start ? static_cast<long long>(rows) * a.share / seqs->n_seqs : a.share;
    if (rows_per_head <= 8) return launch_shape<1>(ctx, s, a, cache->head_dim, cache->quant_group, static_cast<unsigned char*>(ws));
    if (rows_per_head > 16) return launch_shape<3>(ctx, s, a, cache->head_dim, cache->quant_group, static_cast<unsigned char*>(ws));
    return launch_shape<2>(ctx, s, a, cache->head_dim, cache->quant_group, static_cast<unsigned char*>(ws));
}
