// The work of an attention over the cache: items (sequence, KV head in use, block of query rows) laid end to end on a line that is cut for the
// CTAs, and the joining of items that were cut.  The including file says how many units an item counts on top of its blocks
// (kItemCost), up to how many blocks one CTA may take an item alone (kItemAlone), how many blocks' time it takes to join what is cut (kItemJoin), and with how many
// blocks of room a sequence that is not asked (kItemShort).
#pragma once

#include <math_constants.h>

#include "cache.cuh"
#include "ptx.cuh"

namespace {

using namespace wptx;

constexpr int kMaxCtas = 160;
constexpr int kMeta = 8;           // words of meta of a partial result

struct AttnArgs {
    CacheView c;
    SeqView q;
    const __nv_bfloat16* qm;
    long long qs;
    unsigned page_bytes;
    int n_q, share, hpg, words, causal;
    unsigned by_share;             // 2^32 / share rounded up (0: share is 1): n / share = n * by_share >> 32 for n below 2^32 / share
    const uint32_t* mask_bits;
    float scale_log2e;
    __nv_bfloat16* o;
    int* status;                   // takes WIDE_ERR_BAD_INDEX
    int plan_words;                // words of a sequence's head mask
    unsigned char* plan;           // the plan in the workspace, or NULL: every CTA makes its own in shared memory
    float* heads;                  // partial results of warps whose first item began before their piece; of a portion of an item (wide_attn_tree)
    float* parts;                  // [CTA][2] partial results of CTAs
    int* meta;                     // [CTA][2][kMeta] {0 / 1 / 2: none, more follows, last piece; first row, rows, KV head, row block}
    int most_rows;                 // a sequence with more new rows is left out and reported
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Up to one 128-byte line a thread of the grid.
__device__ __forceinline__ void prefetch_l2(const void* p, size_t bytes) {
    const size_t at = (static_cast<size_t>(blockIdx.x) * blockDim.x + threadIdx.x) * 128;
    if (p && at < bytes) asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const char*>(p) + at));
}

// ------------------------------------------------------------------------------------------------ the plan
// offsets[s] = units of the sequences before s (an item: kItemCost and its 16-key blocks), masks[s] = KV heads in use.
struct Plan {
    long long* offsets;
    int4* seqs;                 // first row, rows, length, row blocks; rows 0 where there is nothing to do
    uint32_t *masks, *groups;   // groups: only on the way to the masks
    int* same;                  // units of every item where each has a CTA of its own, else 0
};
__device__ __forceinline__ Plan plan_at(unsigned char* p, int n_seqs, int plan_words) {
    int4* q = reinterpret_cast<int4*>(p);
    long long* o = reinterpret_cast<long long*>(q + n_seqs);
    uint32_t* m = reinterpret_cast<uint32_t*>(o + n_seqs + 1);
    return Plan{o, q, m + 2, m + 2 + n_seqs * plan_words, reinterpret_cast<int*>(m)};
}
size_t plan_bytes(int n_seqs, int plan_words, int words) {
    return 24 * static_cast<size_t>(n_seqs) + 16 + 4 * static_cast<size_t>(n_seqs) * (plan_words + words);
}

// Two rounds of loads (lengths, masks; one thread a sequence), then arithmetic.  Up to 16 new rows are looked at
// for the KV heads in use; of more rows all heads are taken.
template <int ROWS>
__device__ void make_plan(const AttnArgs& a, const Plan& p, long long* part, int ctas, bool report) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
    const int per = (a.q.n_seqs + blockDim.x - 1) / blockDim.x;
    const int s0 = min(a.q.n_seqs, tid * per), s1 = min(a.q.n_seqs, s0 + per);
    const bool direct = a.share == a.hpg;      // a group is the query heads of one KV head
    for (int s = s0; s < s1; ++s) {
        const SeqInfo i = wide_seq_info(a.q, s, a.c.page_shift);
        if ((i.bad || i.n_rows > a.most_rows) && report) atomicExch(a.status, WIDE_ERR_BAD_INDEX);
        const bool some = i.n_rows > 0 && i.n_rows <= a.most_rows && i.len > 0;
        const int looked = a.mask_bits && i.n_rows <= 16 ? i.n_rows : 0;
        p.seqs[s] = make_int4(i.row0, i.n_rows, i.len, some ? (i.n_rows * a.share + ROWS - 1) / ROWS : 0);
        uint32_t* out = direct ? p.masks + s * a.plan_words : p.groups + s * a.words;
        for (int w = 0; w < a.words; ++w) {      // groups that any new row uses
            uint32_t m = some && looked == 0 ? 0xffffffffu : 0u;
            if (some)
                for (int r = 0; r < looked; ++r) m |= a.mask_bits[static_cast<size_t>(i.row0 + r) * a.words + w];
            const int left = a.c.n_kv_heads - 32 * w;
            out[w] = direct && left < 32 ? m & ((1u << left) - 1u) : m;
        }
    }
    if (!direct) {
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
    }
    // Where there are few items, none of them long, a CTA takes one item: nothing is left to join between CTAs, and that
    // costs more than uneven CTAs do.  (One sequence of 200 tokens, 4 heads: 15.7 us with an even cut, 14.6 us so, when this was added.)
    int most = 0;
    long long items = 0;
    for (int s = s0; s < s1; ++s) {
        int used = 0;
        for (int w = 0; w < a.plan_words; ++w) used += __popc(p.masks[s * a.plan_words + w]);
        const int4 i = p.seqs[s];
        p.offsets[s] = static_cast<long long>(used) * i.w;
        items += p.offsets[s];
        if (used && i.w) most = max(most, (i.z + 15) >> 4);
    }
    const int few = __syncthreads_and(items <= ctas && most <= kItemAlone);
    int same = 0;
    if (few) {      // then these sums fit 32 bits
        const int n = __reduce_add_sync(0xffffffffu, static_cast<int>(items)), longest = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) part[warp] = static_cast<long long>(n) << 32 | longest;
        __syncthreads();
        int sum = 0;
        for (int w = 0; w < n_warps; ++w) {
            sum += static_cast<int>(part[w] >> 32);
            same = max(same, static_cast<int>(part[w]));
        }
        // (an item alone, same blocks, against an even cut, sum * (same + kItemCost) / ctas, and the joining)
        const bool brief = (static_cast<long long>(a.q.max_pages) << (a.c.page_shift - 4)) <= kItemShort;
        same = sum <= ctas && (brief || same * (ctas - sum) <= sum * kItemCost + kItemJoin * ctas) ? same + kItemCost : 0;
        __syncthreads();
    }
    if (tid == 0) *p.same = same;
    long long sum = 0;
    for (int s = s0; s < s1; ++s) {
        const long long n = p.offsets[s] * (same ? same : ((p.seqs[s].z + 15) >> 4) + kItemCost);
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
__global__ void __launch_bounds__(1024) attn_cache_plan_kernel(AttnArgs a, int ctas) {
    __shared__ long long part[32];
    grid_dep_launch();
    grid_dep_wait();
    make_plan<ROWS>(a, plan_at(a.plan, a.q.n_seqs, a.plan_words), part, ctas, true);
}

// The part of an item that lies in a piece of the line: blocks [blk, end).  left: units of the piece behind it.
struct Cursor {
    int seq, kvh, rb;      // the item
    int blk, end, left;
    int n_blk, n_rb;       // blocks of an item of this sequence, row blocks of it
    int each;              // units of an item
};

__device__ __forceinline__ int next_head(const AttnArgs& a, const Plan& p, int seq, int from) {
    for (int w = from >> 5; w < a.plan_words; ++w) {
        uint32_t m = p.masks[seq * a.plan_words + w];
        if (w == from >> 5) m &= 0xffffffffu << (from & 31);
        if (m) return 32 * w + __ffs(m) - 1;
    }
    return -1;
}

// the cursor's item from unit `pos` on
__device__ __forceinline__ void take(Cursor& k, int pos) {
    const int to = min(k.each, pos + k.left);
    k.left -= to - pos;
    k.blk = max(0, pos - kItemCost);
    k.end = min(k.n_blk, max(0, to - kItemCost));
}

// to the next item of the piece that has blocks in it; the caller knows that units are left
__device__ __forceinline__ void next_item(const AttnArgs& a, const Plan& p, Cursor& k) {
    do {
        if (++k.rb >= k.n_rb) {
            k.rb = 0;
            k.kvh = next_head(a, p, k.seq, k.kvh + 1);
            if (k.kvh < 0) {
                do ++k.seq;
                while (k.seq + 1 < a.q.n_seqs && p.offsets[k.seq + 1] == p.offsets[k.seq]);
                const int4 i = p.seqs[k.seq];
                k.n_blk = (i.z + 15) >> 4;
                k.n_rb = i.w;
                k.each = p.same[0] ? p.same[0] : k.n_blk + kItemCost;
                k.kvh = next_head(a, p, k.seq, 0);
            }
        }
        take(k, 0);
    } while (k.blk >= k.end && k.left > 0);
}

// units [u, u + n) of the line
__device__ __forceinline__ Cursor locate(const AttnArgs& a, const Plan& p, long long u, int n) {
    Cursor k;
    int lo = 0, hi = a.q.n_seqs - 1;   // the last sequence that starts at or before u: it holds u
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.offsets[mid] <= u) lo = mid;
        else hi = mid - 1;
    }
    k.seq = lo;
    const int4 i = p.seqs[lo];
    k.n_blk = (i.z + 15) >> 4;
    k.n_rb = i.w;
    k.left = n;
    const long long r = u - p.offsets[lo];
    const int each = p.same[0] ? p.same[0] : k.n_blk + kItemCost;
    k.each = each;
    int nth, pos;
    if (r <= 0x7fffffffLL) {
        nth = static_cast<int>(r) / each;
        pos = static_cast<int>(r) - nth * each;
    } else {
        const long long item = r / each;
        nth = static_cast<int>(item);          // heads * row blocks: far below 2^31
        pos = static_cast<int>(r - item * each);
    }
    k.rb = 0;
    if (k.n_rb > 1) {
        k.rb = nth % k.n_rb;
        nth /= k.n_rb;
    }
    k.kvh = next_head(a, p, lo, 0);
    for (; nth > 0; --nth) k.kvh = next_head(a, p, lo, k.kvh + 1);
    take(k, pos);
    if (k.blk >= k.end && k.left > 0) next_item(a, p, k);
    return k;
}

// Row block `rb` of a KV head: its rows are (new token, query head of the KV head) pairs, token by token.  Row rr of the
// block is token `tok` of the sequence, query head `sub` of the KV head.
struct Row {
    int tok, sub;
};
struct RowBlock {
    int tok0, rem;     // of the block's first row
};
__device__ __forceinline__ RowBlock row_block(const AttnArgs& a, int first) {
    RowBlock b;
    b.tok0 = first / a.share;
    b.rem = first - b.tok0 * a.share;
    return b;
}
__device__ __forceinline__ Row row_of(const AttnArgs& a, const RowBlock& b, int rr) {
    const unsigned n = b.rem + rr, t = a.by_share ? __umulhi(n, a.by_share) : n;
    return Row{b.tok0 + static_cast<int>(t), static_cast<int>(n - t * a.share)};
}

// What the epilogues need of a row: where its output goes (nullptr: the row does not exist), whether its group is on.
struct RowOut {
    __nv_bfloat16* o;
    bool on;
};
__device__ __forceinline__ RowOut row_out(const AttnArgs& a, int row0, int n_rows, int kvh, const Row& w, int head_dim) {
    RowOut r;
    const int h = kvh * a.share + w.sub;
    // (the comparison with all rows: what the second kernel is told comes from the workspace, which another call may be using by mistake)
    r.o = w.tok < n_rows && static_cast<unsigned>(row0 + w.tok) < static_cast<unsigned>(a.q.rows) ? a.o + (static_cast<size_t>(row0 + w.tok) * a.n_q + h) * head_dim : nullptr;
    r.on = r.o && (!a.mask_bits || wide_mask_bit(a.mask_bits, a.words, row0 + w.tok, h / a.hpg));
    return r;
}

__host__ __device__ constexpr int slot_floats(int rows, int D) { return rows * (D + 4); }   // rows of D values, then m and l of each

// Items that more than one CTA had a piece of: block c joins the one that begins in CTA c and goes on in the next.
// A warp takes half a row's channels (a whole row of 64): lane e reads the maximum and sum of piece e.
template <int ROWS, int D>
__global__ void __launch_bounds__(256) attn_cache_join_kernel(const __grid_constant__ AttnArgs a, int ctas) {
    grid_dep_wait();
    const int c = blockIdx.x, lane = threadIdx.x & 31, unit = threadIdx.x >> 5;
    // one round of loads: what does CTA c leave open, how far does it go (CTAs c + 1, ...:
    // the first piece of each belongs to the item, up to the one that ends it)
    const int* mine = a.meta + (2 * c + 1) * kMeta;
    const int4 meta = *reinterpret_cast<const int4*>(mine);
    const int rb = mine[4];
    int st = c + 1 + lane < ctas ? a.meta[2 * (c + 1 + lane) * kMeta] : 0;
    if (meta.x != 1 || static_cast<unsigned>(meta.w) >= static_cast<unsigned>(a.c.n_kv_heads)) return;
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
        st = k + lane < ctas ? a.meta[2 * (k + lane) * kMeta] : 0;
    }
    auto piece = [&](int i) -> const float* {
        return a.parts + static_cast<size_t>(i == 0 ? 2 * c + 1 : 2 * (c + i)) * slot_floats(ROWS, D);
    };
    constexpr int kHalves = D / 64;
    const RowBlock rows = row_block(a, rb * ROWS);
    for (int u = unit + 8 * blockIdx.y; u < ROWS * kHalves; u += 8 * gridDim.y) {
        const int r = u / kHalves, d = u % kHalves * 64 + 2 * lane;
        const RowOut ro = row_out(a, meta.y, meta.z, meta.w, row_of(a, rows, r), D);
        if (!ro.o) continue;
        float m = -CUDART_INF_F, l = 0.f;
        float2 x = make_float2(0.f, 0.f);
        for (int e0 = 0; e0 < n; e0 += 32) {
            // all pieces' values are asked for together with their maxima and sums
            const int last = min(32, n - e0);
            const float2 ml = lane < last ? *reinterpret_cast<const float2*>(piece(e0 + lane) + ROWS * D + 2 * r) : make_float2(-CUDART_INF_F, 0.f);
            float2 v[32];
#pragma unroll
            for (int e = 0; e < 32; ++e)
                v[e] = e < last ? *reinterpret_cast<const float2*>(piece(e0 + e) + r * D + d) : make_float2(0.f, 0.f);
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
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                const float we = __shfl_sync(0xffffffffu, w, e);
                x = make_float2(fmaf(v[e].x, we, x.x), fmaf(v[e].y, we, x.y));
            }
        }
        const float inv = ro.on && l != 0.f ? 1.f / l : 0.f;
        __nv_bfloat162 b = __floats2bfloat162_rn(0.f, 0.f);
        if (inv != 0.f) b = __floats2bfloat162_rn(x.x * inv, x.y * inv);
        *reinterpret_cast<__nv_bfloat162*>(ro.o + d) = b;
    }
}

}  // namespace
