// New rows into the 4-bit cache with the position rotation applied on the way, and the queries rotated beside them
// (wide_cache_append): what wide_rope and wide_cache_write do in two calls, with the same bits, in one launch.
//
// The rotated keys never go to memory: per token and KV head that saves 4 bytes a channel of 2 + 4 + 2 + 0.56 for bf16, and a decode step,
// whose every call is latency, has one launch instead of two.  HBM bounds a long chunk, dependent loads (row range, length,
// page, rows) a step.
//
// A CTA takes one block of the cache, up to 16 new tokens of a sequence, since these share their sines and cosines, which it works out
// once into shared memory; its warps then take the keys and the values of a head each (as wide_cache_write does: 8 channels of a token
// a lane) and runs of 32 pieces of the query rows.  A key's channel and its partner, rot / 2 further on, lie in two lanes
// of the warp, which exchange them by shuffles.  Where there are fewer blocks than SMs, several CTAs share a block's heads.
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
    bool interleaved;
    bool wide;       // the query rows allow 32-byte accesses
    int* status;
};

// cosines and sines of two neighbouring pairs: [token of the block][which two of 8 pairs][8 pairs], so that the lanes of a warp, which
// differ in the last index, read neighbouring 16-byte words
template <int D> struct Angles {
    float4 two[16][4][D / 16];
    __device__ __forceinline__ void put(int r, int pair, float2 v) { reinterpret_cast<float2*>(&two[r][(pair >> 1) & 3][pair >> 3])[pair & 1] = v; }
};

// the channels of another lane
__device__ __forceinline__ void from_lane(const Raw8<__nv_bfloat16>& x, int lane, float (&y)[8]) {
    Raw8<__nv_bfloat16> z;
    z.v = make_uint4(__shfl_sync(0xffffffffu, x.v.x, lane), __shfl_sync(0xffffffffu, x.v.y, lane), __shfl_sync(0xffffffffu, x.v.z, lane),
                     __shfl_sync(0xffffffffu, x.v.w, lane));
    z.get(y);
}
__device__ __forceinline__ void from_lane(const Raw8<float>& x, int lane, float (&y)[8]) {
    float z[8];
    x.get(z);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = __shfl_sync(0xffffffffu, z[e], lane);
}
__device__ __forceinline__ void put_back(Raw8<__nv_bfloat16>& x, const float (&y)[8]) {
    Vec8<__nv_bfloat16> z;
    z.set(y);
    x.v = z.v;
}
__device__ __forceinline__ void put_back(Raw8<float>& x, const float (&y)[8]) {
    x.a = make_float4(y[0], y[1], y[2], y[3]);
    x.b = make_float4(y[4], y[5], y[6], y[7]);
}

template <int D>
__device__ __forceinline__ void angles_of(const Angles<D>& t, int r, int j, float2 (&c)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float4 two = t.two[r][e][j];
        c[2 * e] = make_float2(two.x, two.y);
        c[2 * e + 1] = make_float2(two.z, two.w);
    }
}

template <typename T, int D, int G>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 3 : 2) cache_append_kernel(const __grid_constant__ AppendArgs a) {
    __shared__ Angles<D> table;
    __shared__ unsigned long long turn[kMaxPairs];
    constexpr int kLT = BlockLanes<D>::kLT, kRounds = BlockLanes<D>::kRounds;
    constexpr int kUnits = D / 16;         // pieces of 8 pairs of a query head
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, p = lane / kLT, u8 = lane % kLT;
    const int pairs = a.rot / 2, m = a.rot / 16;
    wptx::grid_dep_wait();
    const Unit w = find_block(a.s, a.c, blockIdx.x);
    if (w.bad && tid == 0) atomicExch(a.status, WIDE_ERR_BAD_INDEX);
    if (blockIdx.y == 0) report_bad(a.s, a.c.page_shift, a.status);
    if (!w.some) return;
    const int p0 = w.block << 4;
    const int r0 = max(0, w.first - p0), r1 = min(16, w.len - p0);   // new tokens of the block
    const long long row_of_0 = static_cast<long long>(w.row0) + (p0 - w.first);
    const int n_units = a.n_q * kUnits, q_tasks = (n_units + 31) >> 5, kv_tasks = 2 * a.c.n_kv_heads, tasks = kv_tasks + q_tasks;
    uint8_t* page = wide_cache_block(a.c, a.s, w.seq, p0, 0);
    if (!page && tid == 0) atomicExch(a.status, WIDE_ERR_BAD_INDEX);
    const size_t head_bytes = static_cast<size_t>(a.c.block_bytes) << (a.c.page_shift - 4);
    bool ready = false;
    for (int task = blockIdx.y * kWarps + warp;; task += gridDim.y * kWarps) {
        const bool kv = task < kv_tasks && page, values = task & 1;
        const int head = task >> 1;
        Raw8<T> raw[kRounds];
        uint32_t here = 0;                 // bit i: the token of round i is new
        auto token = [&](int i) { return BlockLanes<D>::token(values, p, i); };
        if (kv) {
            const T* src = static_cast<const T*>(values ? a.v : a.k) + head * D + 8 * u8;
            const long long stride = values ? a.vs : a.ks;
#pragma unroll
            for (int i = 0; i < kRounds; ++i) {
                const int r = token(i);
                raw[i].clear();
                if (r >= r0 && r < r1) {
                    raw[i].load(src + (row_of_0 + r) * stride);
                    here |= 1u << i;
                }
            }
        }
        if (!ready) {      // the angles, while the first rows are on their way
            ready = true;
            if (tid < pairs) turn[tid] = wide_rope_turn(a.inv_freq[tid]);
            __syncthreads();
            for (int i = tid; i < (r1 - r0) * pairs; i += kThreads) {
                const int rr = i / pairs, pr = i - rr * pairs;
                const int ax = a.axis ? a.axis[pr] : 0;
                float2 v = make_float2(1.f, 0.f);
                if (static_cast<unsigned>(ax) < static_cast<unsigned>(a.n_axes))
                    v = wide_rope_angle(a.positions[static_cast<size_t>(ax) * a.s.rows + row_of_0 + r0 + rr], turn[pr]);
                else
                    atomicExch(a.status, WIDE_ERR_BAD_INDEX);
                table.put(r0 + rr, pr, v);
            }
            __syncthreads();
        }
        if (task >= tasks) break;
        if (kv) {
            if (!values) {
                const uint32_t rounds = __reduce_or_sync(0xffffffffu, here);
                const bool turned = u8 < 2 * m, low = u8 < m;
                const int j = a.interleaved ? u8 >> 1 : low ? u8 : u8 - m;
                const int partner = turned ? (low ? lane + m : lane - m) : lane;
#pragma unroll
                for (int i = 0; i < kRounds; ++i) {
                    if (!((rounds >> i) & 1u)) continue;
                    const int r = token(i);
                    float x[8];
                    raw[i].get(x);
                    if (a.interleaved) {
                        if (turned && ((here >> i) & 1u)) {
                            const float4 c0 = table.two[r][2 * (u8 & 1)][j], c1 = table.two[r][2 * (u8 & 1) + 1][j];
                            const float2 c[4] = {{c0.x, c0.y}, {c0.z, c0.w}, {c1.x, c1.y}, {c1.z, c1.w}};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float u = x[2 * e], v = x[2 * e + 1];
                                x[2 * e] = wide_rope_low(u, v, c[e]);
                                x[2 * e + 1] = wide_rope_high(u, v, c[e]);
                            }
                            put_back(raw[i], x);
                        }
                    } else {
                        float y[8];
                        from_lane(raw[i], partner, y);
                        if (turned && ((here >> i) & 1u)) {
                            float2 c[8];
                            angles_of<D>(table, r, j, c);
#pragma unroll
                            for (int e = 0; e < 8; ++e) x[e] = low ? wide_rope_low(x[e], y[e], c[e]) : wide_rope_high(y[e], x[e], c[e]);
                            put_back(raw[i], x);
                        }
                    }
                }
            }
            put_block<T, D, G>(raw, here, page + head * head_bytes, values, [&](int i, bool) {
                Raw8<T> x;
                x.clear();
#pragma unroll
                for (int e = 0; e < kRounds; ++e)
                    if (e == i) x = raw[e];
                return x;
            });
        } else if (task >= kv_tasks) {
            const int unit = (task - kv_tasks) * 32 + lane;
            if (unit < n_units) {
                const int qh = unit / kUnits, j = unit % kUnits;
                const bool turned = j < m;
                const int lo = qh * D + ((turned && !a.interleaved) ? 8 * j : 16 * j);
                const int hi = qh * D + ((turned && !a.interleaved) ? 8 * j + pairs : 16 * j + 8);
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
                                float x[8], y[8];
                                u[i].get(x);
                                z[i].get(y);
                                float2 c[8];
                                angles_of<D>(table, rr + i, j, c);
                                if (a.interleaved) {
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        const float x0 = x[2 * e], x1 = x[2 * e + 1], y0 = y[2 * e], y1 = y[2 * e + 1];
                                        x[2 * e] = wide_rope_low(x0, x1, c[e]);
                                        x[2 * e + 1] = wide_rope_high(x0, x1, c[e]);
                                        y[2 * e] = wide_rope_low(y0, y1, c[4 + e]);
                                        y[2 * e + 1] = wide_rope_high(y0, y1, c[4 + e]);
                                    }
                                } else {
#pragma unroll
                                    for (int e = 0; e < 8; ++e) {
                                        const float x0 = x[e], y0 = y[e];
                                        x[e] = wide_rope_low(x0, y0, c[e]);
                                        y[e] = wide_rope_high(x0, y0, c[e]);
                                    }
                                }
                                u[i].set(x);
                                z[i].set(y);
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
int launch(wide_ctx* ctx, cudaStream_t s, const AppendArgs& a) {
    const int slots = slots_of(a.s);
    const int tasks = 2 * a.c.n_kv_heads + (a.n_q * (D / 16) + 31) / 32;
    const int most = (tasks + kWarps - 1) / kWarps, want = (2 * ctx->sm_count + slots - 1) / slots;
    WideLaunch l(ctx, s, "cache_append");
    WIDE_CUDA_CHECK(wide_launch_after(ctx, cache_append_kernel<T, D, G>, dim3(slots, want < most ? want : most), dim3(kThreads), 0, s, a));
    return WIDE_OK;
}

template <typename T>
int launch_dims(wide_ctx* ctx, cudaStream_t s, const AppendArgs& a, int D, int G) {
    if (D == 128) {
        if (G == 128) return launch<T, 128, 128>(ctx, s, a);
        if (G == 64) return launch<T, 128, 64>(ctx, s, a);
        return launch<T, 128, 32>(ctx, s, a);
    }
    if (G == 64) return launch<T, 64, 64>(ctx, s, a);
    return launch<T, 64, 32>(ctx, s, a);
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
    a.interleaved = (flags & WIDE_FLAG_ROPE_INTERLEAVED) != 0;
    const int elem = wide_elem_bytes(dtype);
    a.wide = !q || (wide_rows32(q, qs * elem) && wide_rows32(q_out, oqs * elem));
    a.status = ctx->d_status + WIDE_STATUS_INDEX;
    if (dtype == WIDE_F32) return launch_dims<float>(ctx, s, a, cache->head_dim, cache->quant_group);
    return launch_dims<__nv_bfloat16>(ctx, s, a, cache->head_dim, cache->quant_group);
}
