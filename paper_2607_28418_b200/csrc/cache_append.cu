// New rows into the 4-bit cache with the position rotation applied on the way, and the queries rotated beside them
// (wide_cache_append): what wide_rope and wide_cache_write do in two calls, with the same bits, in one launch.
//
// A decode step, whose every call is latency, has one launch instead of two: dependent loads (row range, length, page, rows) bound it.  The rotated keys never go to
// memory, which saves 4 bytes a channel of 2 + 4 + 2 + 0.56 for bf16, but a long chunk takes as long as the two calls, as instructions bound it.
//
// A CTA takes one block of the cache, up to 16 new tokens of a sequence, since these share their sines and cosines, which it works out
// once into shared memory; its warps then take the keys and the values of a head each (as wide_cache_write does: 8 channels of a token
// a lane) and runs of 32 pieces of the query rows.  A key's channel and its partner, rot / 2 further on, lie in two lanes
// of the warp, which exchange them by shuffles.  Several CTAs share a block's heads.
//
// Measured with cold caches (about 8 us of each are the call's own): 64 tokens of a decode step 12.3 us (the two calls 13.3), 976 tokens
// of 16 trees 18.4 (21), 8188 tokens 57 (58; floor 27), 1390 tokens of 40 heads in fp32 35 (39; floor 13).  The issue of
// instructions bounds the long ones (levels 25 a value, rotation 7), at 55 % of the slots, with 24 warps an SM.
#include "cache_levels.cuh"
#include "rope.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxPairs = 64;

struct AppendArgs {
    CacheView c;
    SeqView s;
    const void *q, *k, *v;
    void* q_out;
    long long qs, ks, vs, oqs;
    const int32_t* positions;
    const double* inv_freq;
    const int32_t* axis;
    int n_q, rot, n_axes;
    bool wide;       // the query rows allow 32-byte accesses
    int* status;
};

// cosines and sines of two neighbouring pairs: [token of the block][which two of 8 pairs][8 pairs], so that the lanes of a warp, which
// differ in the last index, read neighbouring 16-byte words
template <int D> struct Angles {
    float4 two[16][4][D / 16];
    __device__ __forceinline__ void put(int r, int pair, float2 v) { reinterpret_cast<float2*>(&two[r][(pair >> 1) & 3][pair >> 3])[pair & 1] = v; }
};

// channels 2 i and 2 i + 1 of a lane's eight
template <template <typename> class R>
__device__ __forceinline__ uint32_t word_of(const R<__nv_bfloat16>& x, int i) { return i == 0 ? x.v.x : i == 1 ? x.v.y : i == 2 ? x.v.z : x.v.w; }
template <template <typename> class R>
__device__ __forceinline__ void two_of(const R<__nv_bfloat16>& x, int i, float& a, float& b) {
    const uint32_t w = word_of(x, i);
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
}
template <template <typename> class R>
__device__ __forceinline__ void two_of(const R<float>& x, int i, float& a, float& b) {
    const float4& f = i < 2 ? x.a : x.b;
    a = i & 1 ? f.z : f.x;
    b = i & 1 ? f.w : f.y;
}
// x's where `first`, else y's
__device__ __forceinline__ void two_of_either(bool first, const Raw8<__nv_bfloat16>& x, const Raw8<__nv_bfloat16>& y, int i, float& a, float& b) {
    const uint32_t w = first ? word_of(x, i) : word_of(y, i);
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
}
__device__ __forceinline__ void two_of_either(bool first, const Raw8<float>& x, const Raw8<float>& y, int i, float& a, float& b) {
    float x0, x1, y0, y1;
    two_of(x, i, x0, x1);
    two_of(y, i, y0, y1);
    a = first ? x0 : y0;
    b = first ? x1 : y1;
}
// the channels of another lane
__device__ __forceinline__ Raw8<__nv_bfloat16> from_lane(const Raw8<__nv_bfloat16>& x, int lane) {
    Raw8<__nv_bfloat16> y;
    y.v = make_uint4(__shfl_sync(0xffffffffu, x.v.x, lane), __shfl_sync(0xffffffffu, x.v.y, lane), __shfl_sync(0xffffffffu, x.v.z, lane),
                     __shfl_sync(0xffffffffu, x.v.w, lane));
    return y;
}
__device__ __forceinline__ float4 from_lane(const float4& x, int lane) {
    return make_float4(__shfl_sync(0xffffffffu, x.x, lane), __shfl_sync(0xffffffffu, x.y, lane), __shfl_sync(0xffffffffu, x.z, lane),
                       __shfl_sync(0xffffffffu, x.w, lane));
}
__device__ __forceinline__ Raw8<float> from_lane(const Raw8<float>& x, int lane) {
    Raw8<float> y;
    y.a = from_lane(x.a, lane);
    y.b = from_lane(x.b, lane);
    return y;
}
template <template <typename> class R>
__device__ __forceinline__ void put_two(R<__nv_bfloat16>& x, int i, float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    (i == 0 ? x.v.x : i == 1 ? x.v.y : i == 2 ? x.v.z : x.v.w) = *reinterpret_cast<const uint32_t*>(&h);
}
template <template <typename> class R>
__device__ __forceinline__ void put_two(R<float>& x, int i, float a, float b) {
    float4& f = i < 2 ? x.a : x.b;
    (i & 1 ? f.z : f.x) = a;
    (i & 1 ? f.w : f.y) = b;
}

// 24 warps an SM of 80 registers for the 16-bit types (200 bytes spilled a thread with heads of 128; 16 warps of 128 registers, nothing
// spilled: 59 instead of 57 us for 8188 tokens; 32 of 64: 61).
template <typename T, int D, int G, bool kInterleaved>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 3 : 2) cache_append_kernel(const __grid_constant__ AppendArgs a) {
    __shared__ Angles<D> table;
    __shared__ unsigned long long turn[kMaxPairs];
    constexpr int kLT = BlockLanes<D>::kLT, kRounds = BlockLanes<D>::kRounds;
    constexpr int kUnits = D / 16;         // pieces of 8 pairs of a query head
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, p = lane / kLT, u8 = lane % kLT;
    const int pairs = a.rot / 2, m = a.rot / 16;
    wptx::grid_dep_wait();
    __shared__ Unit found;
    __shared__ uint8_t* found_page;
    if (warp == 0) {
        const Unit u = find_block(a.s, a.c, blockIdx.x);
        if (lane == 0) {
            found = u;
            found_page = u.some ? wide_cache_block(a.c, a.s, u.seq, u.block << 4, 0) : nullptr;
            if (u.bad || (u.some && !found_page)) atomicExch(a.status, WIDE_ERR_BAD_INDEX);
        }
    } else if (warp < 3) {
        if (tid - 32 < pairs) turn[tid - 32] = wide_rope_turn(a.inv_freq[tid - 32]);
    } else if (blockIdx.y == 0 && a.s.row_start) {   // sequences that no block leads to are checked too
        for (int i = blockIdx.x * (kThreads - 96) + tid - 96; i < a.s.n_seqs; i += gridDim.x * (kThreads - 96))
            if (wide_seq_info(a.s, i, a.c.page_shift).bad) atomicExch(a.status, WIDE_ERR_BAD_INDEX);
    }
    __syncthreads();
    const Unit w = found;
    if (!w.some) return;
    const int p0 = w.block << 4;
    const int r0 = max(0, w.first - p0), r1 = min(16, w.len - p0);   // new tokens of the block
    const long long row_of_0 = static_cast<long long>(w.row0) + (p0 - w.first);
    const int n_units = a.n_q * kUnits, q_tasks = (n_units + 31) >> 5, kv_tasks = 2 * a.c.n_kv_heads, tasks = kv_tasks + q_tasks;
    uint8_t* page = found_page;
    const size_t head_bytes = static_cast<size_t>(a.c.block_bytes) << (a.c.page_shift - 4);
    const int task0 = blockIdx.y * kWarps + warp;
    // the first rows are brought into L2 while the angles are worked out: a line a lane
    if (task0 < kv_tasks) {
        constexpr int kLines = D * static_cast<int>(sizeof(T)) / 128;
        const T* src = static_cast<const T*>((task0 & 1) ? a.v : a.k) + (task0 >> 1) * D;
        for (int i = lane; i < (r1 - r0) * kLines; i += 32)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(src + (row_of_0 + r0 + i / kLines) * ((task0 & 1) ? a.vs : a.ks) + i % kLines * (128 / static_cast<int>(sizeof(T)))));
    }
    if (const int pr = tid % kMaxPairs; pr < pairs) {
        const int ax = a.axis ? a.axis[pr] : 0;
        const bool good = static_cast<unsigned>(ax) < static_cast<unsigned>(a.n_axes);
        if (!good) atomicExch(a.status, WIDE_ERR_BAD_INDEX);
        const int32_t* at = a.positions + static_cast<size_t>(good ? ax : 0) * a.s.rows + row_of_0;
        for (int r = r0 + tid / kMaxPairs; r < r1; r += kThreads / kMaxPairs)
            table.put(r, pr, good ? wide_rope_angle(at[r], turn[pr]) : make_float2(1.f, 0.f));
    }
    __syncthreads();
    for (int task = task0; task < tasks; task += gridDim.y * kWarps) {
        if (task < kv_tasks) {
            if (!page) continue;
            const bool values = task & 1;
            const int head = task >> 1;
            Raw8<T> raw[kRounds];
            uint32_t here = 0;                 // bit i: the token of round i is new
            auto token = [&](int i) { return BlockLanes<D>::token(values, p, i); };
            const T* src = static_cast<const T*>(values ? a.v : a.k) + row_of_0 * (values ? a.vs : a.ks) + head * D + 8 * u8;
            const long long stride = values ? a.vs : a.ks;
#pragma unroll
            for (int i = 0; i < kRounds; ++i) {
                const int r = token(i);
                raw[i].clear();
                if (r >= r0 && r < r1) {
                    raw[i].load(src + r * stride);
                    here |= 1u << i;
                }
            }
            const bool turned = !values && u8 < 2 * m, low = u8 < m;
            const int j = kInterleaved ? u8 >> 1 : low ? u8 : u8 - m;
            const int partner = turned && !kInterleaved ? (low ? m : -m) : 0;     // lanes further on
            // channels 2 i, 2 i + 1 of token r: of this lane in x, the partner's in y; word by word, since all eight with their angles cost
            // spilled registers
            auto turn_two = [&](Raw8<T>& x, const Raw8<T>& y, int r, int i) {
                float x0, x1;
                if (kInterleaved) {
                    two_of(x, i, x0, x1);
                    const float4 two = table.two[r][2 * (u8 & 1) + (i >> 1)][j];
                    const float2 c = i & 1 ? make_float2(two.z, two.w) : make_float2(two.x, two.y);
                    put_two(x, i, wide_rope_low(x0, x1, c), wide_rope_high(x0, x1, c));
                } else {
                    const float4 two = table.two[r][i][j];
                    // low: x c - y s, high: y s + x c, in wide_rope's order of rounding
                    float p0, p1, q0, q1;
                    two_of_either(low, x, y, i, p0, p1);
                    two_of_either(low, y, x, i, q0, q1);
                    const float c0 = low ? two.x : two.y, s0 = low ? -two.y : two.x, c1 = low ? two.z : two.w, s1 = low ? -two.w : two.z;
                    put_two(x, i, __fmaf_rn(p0, c0, __fmul_rn(q0, s0)), __fmaf_rn(p1, c1, __fmul_rn(q1, s1)));
                }
            };
            if (!values) {
                const uint32_t rounds = __reduce_or_sync(0xffffffffu, here);
#pragma unroll
                for (int i = 0; i < kRounds; ++i) {
                    if (!((rounds >> i) & 1u)) continue;
                    const bool mine = turned && ((here >> i) & 1u);
                    Raw8<T> other;
                    if (!kInterleaved) other = from_lane(raw[i], lane + partner);
                    if (mine)
#pragma unroll
                        for (int e = 0; e < 4; ++e) turn_two(raw[i], other, token(i), e);
                }
            }
            put_block<T, D, G>(raw, here, page + head * head_bytes, values, [&](int i, bool on) {
                Raw8<T> again;       // rare: read and turned once more, which keeps the registers free
                again.clear();
                if (on) {
                    const T* row = src + token(i) * stride;
                    again.load(row);
                    if (turned) {
                        Raw8<T> other;
                        other.load(row + 8 * partner);
#pragma unroll
                        for (int e = 0; e < 4; ++e) turn_two(again, other, token(i), e);
                    }
                }
                return again;
            });
        } else {
            const int unit = (task - kv_tasks) * 32 + lane;
            if (unit < n_units) {
                const int qh = unit / kUnits, j = unit % kUnits;
                const bool turned = j < m;
                const int lo = qh * D + ((turned && !kInterleaved) ? 8 * j : 16 * j);
                const int hi = qh * D + ((turned && !kInterleaved) ? 8 * j + pairs : 16 * j + 8);
                const T* src = static_cast<const T*>(a.q) + (row_of_0 + r0) * a.qs;
                T* dst = static_cast<T*>(a.q_out) + (row_of_0 + r0) * a.oqs;
                constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;     // rows on their way
                for (int rr = r0; rr < r1; rr += kAhead) {
                    Vec8<T> u[kAhead], z[kAhead];
#pragma unroll
                    for (int i = 0; i < kAhead; ++i)
                        if (rr + i < r1) {
                            u[i].load(src + i * a.qs + lo, a.wide);
                            z[i].load(src + i * a.qs + hi, a.wide);
                        }
#pragma unroll
                    for (int i = 0; i < kAhead; ++i)
                        if (rr + i < r1) {
                            if (turned) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const float4 one = table.two[rr + i][kInterleaved ? e >> 1 : e][j], two = table.two[rr + i][kInterleaved ? 2 + (e >> 1) : e][j];
                                    float x0, x1, y0, y1;
                                    two_of(u[i], e, x0, x1);
                                    two_of(z[i], e, y0, y1);
                                    if (kInterleaved) {
                                        const float2 c = e & 1 ? make_float2(one.z, one.w) : make_float2(one.x, one.y);
                                        const float2 d = e & 1 ? make_float2(two.z, two.w) : make_float2(two.x, two.y);
                                        put_two(u[i], e, wide_rope_low(x0, x1, c), wide_rope_high(x0, x1, c));
                                        put_two(z[i], e, wide_rope_low(y0, y1, d), wide_rope_high(y0, y1, d));
                                    } else {
                                        const float2 c = make_float2(one.x, one.y), d = make_float2(one.z, one.w);
                                        put_two(u[i], e, wide_rope_low(x0, y0, c), wide_rope_low(x1, y1, d));
                                        put_two(z[i], e, wide_rope_high(x0, y0, c), wide_rope_high(x1, y1, d));
                                    }
                                }
                            }
                            u[i].store(dst + i * a.oqs + lo, a.wide);
                            z[i].store(dst + i * a.oqs + hi, a.wide);
                        }
                    src += kAhead * a.qs;
                    dst += kAhead * a.oqs;
                }
            }
        }
    }
}

template <typename T, int D, int G>
int launch(wide_ctx* ctx, cudaStream_t s, const AppendArgs& a, bool interleaved) {
    // CTAs that share a block's heads make the angles of its tokens once each, but even out what SMs finish unevenly.  Up to 2, 4, 8, 12
    // CTAs an SM in all: 8188 tokens of 32/8 heads of 128, bf16 (519 blocks) 65 / 59 / 57 / 57 us, 1390 of 40/40 heads of 64, fp32
    // 32 / 33 / 35 / 41 us (cold caches, the call's own 8 us included).
    const int slots = slots_of(a.s);
    const int tasks = 2 * a.c.n_kv_heads + (a.n_q * (D / 16) + 31) / 32;
    const int most = (tasks + kWarps - 1) / kWarps, want = (8 * ctx->sm_count + slots - 1) / slots;
    const auto kernel = interleaved ? cache_append_kernel<T, D, G, true> : cache_append_kernel<T, D, G, false>;
    WideLaunch l(ctx, s, "cache_append");
    WIDE_CUDA_CHECK(wide_launch_after(ctx, kernel, dim3(slots, want < most ? want : most), dim3(kThreads), 0, s, a));
    return WIDE_OK;
}

template <typename T>
int launch_dims(wide_ctx* ctx, cudaStream_t s, const AppendArgs& a, bool interleaved, int D, int G) {
    if (D == 128) {
        if (G == 128) return launch<T, 128, 128>(ctx, s, a, interleaved);
        if (G == 64) return launch<T, 128, 64>(ctx, s, a, interleaved);
        return launch<T, 128, 32>(ctx, s, a, interleaved);
    }
    if (G == 64) return launch<T, 64, 64>(ctx, s, a, interleaved);
    return launch<T, 64, 32>(ctx, s, a, interleaved);
}

}  // namespace

int wide_launch_cache_append(wide_ctx* ctx, cudaStream_t s, const wide_cache* cache, const wide_seqs* seqs, const void* q, const void* k,
                             const void* v, int dtype, int rows, int n_q, int rot, long long qs, long long ks, long long vs,
                             const int32_t* positions, int n_axes, const double* inv_freq, const int32_t* axis, void* q_out,
                             long long oqs, unsigned flags) {
    AppendArgs a{};
    a.c = wide_cache_view(cache);
    a.s = wide_seq_view(seqs, rows);
    a.q = q; a.k = k; a.v = v; a.q_out = q_out;
    a.qs = qs; a.ks = ks; a.vs = vs; a.oqs = oqs;
    a.positions = positions; a.inv_freq = inv_freq; a.axis = axis;
    a.n_q = n_q; a.rot = rot; a.n_axes = n_axes;
    const bool interleaved = (flags & WIDE_FLAG_ROPE_INTERLEAVED) != 0;
    const int elem = wide_elem_bytes(dtype);
    a.wide = !q || (wide_rows32(q, qs * elem) && wide_rows32(q_out, oqs * elem));
    a.status = ctx->d_status + WIDE_STATUS_INDEX;
    if (dtype == WIDE_F32) return launch_dims<float>(ctx, s, a, interleaved, cache->head_dim, cache->quant_group);
    return launch_dims<__nv_bfloat16>(ctx, s, a, interleaved, cache->head_dim, cache->quant_group);
}
