// Rotary positions with one or several axes (wide_rope): pair i of every head of token t turns by
// positions[axis[i], t] * inv_freq[i].
//
// Moves bytes: every channel is read and written once, so HBM is the bound; the sines and cosines
// of a token are worked out once by the CTA and serve all of its heads from shared memory.
// The angle must not lose the low bits of a far position (fp32: position 10^6 times frequency 1 is off by
// 0.03 rad).  So a frequency becomes a 64-bit fixed-point number of turns per position, the product with the
// integer position wraps modulo one turn for free in 64-bit integer arithmetic (error: position * 2^-53 of the
// frequency), and only the reduced angle, in half turns, is rounded to fp32 for sincospif.
#include "internal.h"
#include "ptx.cuh"
#include "rope.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 64;
constexpr int kMaxTile = 4;      // tokens of a CTA (16384 tokens of 80 heads, bf16: 133 us with 1, 119 with 2, 113 with 4, 117 with 8)

struct RopeArgs {
    const void *q, *k;
    void *q_out, *k_out;
    long long qs, ks, oqs, oks;
    const int32_t* positions;
    const double* inv_freq;
    const int32_t* axis;
    int tokens, n_q, n_kv, rot, n_axes, tile;
    bool interleaved, inverse;
    bool wide;       // all rows allow 32-byte accesses
    int* status;
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs a) {
    __shared__ unsigned long long turn[kMaxPairs];          // turns per position, 64-bit fraction
    __shared__ __align__(16) float2 cs[kMaxTile][kMaxPairs];
    const int pairs = a.rot / 2, tid = threadIdx.x;
    const int t0 = blockIdx.x * a.tile, nt = min(a.tile, a.tokens - t0);
    // A unit is 8 pairs of one head: two 8-channel pieces, rot / 2 apart or neighbours.  A thread has the same pairs of
    // every (kThreads / kUnits)-th head of the tile's tokens in turn.
    constexpr int kUnits = D / 16, kStep = kThreads / kUnits;
    const int heads = a.n_q + a.n_kv, j = tid % kUnits;
    const bool turned = 16 * j < a.rot;
    const int lo = (turned && !a.interleaved) ? 8 * j : 16 * j;
    const int hi = (turned && !a.interleaved) ? 8 * j + pairs : 16 * j + 8;
    int t = 0, head = tid / kUnits;
    auto wrap = [&]() {
        while (head >= heads) {
            head -= heads;
            ++t;
        }
    };
    auto from = [&]() {
        const long long row = t0 + t;
        return head < a.n_q ? static_cast<const T*>(a.q) + row * a.qs + head * D : static_cast<const T*>(a.k) + row * a.ks + (head - a.n_q) * D;
    };
    wrap();
    wptx::grid_dep_wait();
    // the first unit is on its way while the angles are worked out, each later one while its predecessor turns
    Vec8<T> u, w;
    if (t < nt) {
        const T* src = from();
        u.load(src + lo, a.wide);
        w.load(src + hi, a.wide);
    }
    if (tid < pairs) turn[tid] = wide_rope_turn(a.inv_freq[tid]);
    __syncthreads();
    for (int i = tid; i < nt * pairs; i += kThreads) {
        const int tt = i / pairs, p = i - tt * pairs;
        const int ax = a.axis ? a.axis[p] : 0;
        float2 v = make_float2(1.f, 0.f);
        if (static_cast<unsigned>(ax) < static_cast<unsigned>(a.n_axes)) {
            v = wide_rope_angle(a.positions[static_cast<size_t>(ax) * a.tokens + t0 + tt], turn[p]);
            if (a.inverse) v.y = -v.y;
        } else {
            atomicExch(a.status, WIDE_ERR_BAD_INDEX);
        }
        cs[tt][p] = v;
    }
    __syncthreads();
    while (t < nt) {
        T* dst = (head < a.n_q ? static_cast<T*>(a.q_out) + (t0 + t) * a.oqs + head * D : static_cast<T*>(a.k_out) + (t0 + t) * a.oks + (head - a.n_q) * D);
        const int tt = t;
        Vec8<T> x8 = u, y8 = w;
        head += kStep;
        wrap();
        if (t < nt) {
            const T* src = from();
            u.load(src + lo, a.wide);
            w.load(src + hi, a.wide);
        }
        if (turned) {
            float x[8], y[8];
            x8.get(x);
            y8.get(y);
            float2 c[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 two = *reinterpret_cast<const float4*>(&cs[tt][8 * j + 2 * e]);
                c[2 * e] = make_float2(two.x, two.y);
                c[2 * e + 1] = make_float2(two.z, two.w);
            }
            if (a.interleaved) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = x[2 * e], s = x[2 * e + 1], p2 = y[2 * e], s2 = y[2 * e + 1];
                    x[2 * e] = wide_rope_low(p, s, c[e]);
                    x[2 * e + 1] = wide_rope_high(p, s, c[e]);
                    y[2 * e] = wide_rope_low(p2, s2, c[4 + e]);
                    y[2 * e + 1] = wide_rope_high(p2, s2, c[4 + e]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = x[e], s = y[e];
                    x[e] = wide_rope_low(p, s, c[e]);
                    y[e] = wide_rope_high(p, s, c[e]);
                }
            }
            x8.set(x);
            y8.set(y);
        }
        x8.store(dst + lo, a.wide);
        y8.store(dst + hi, a.wide);
    }
}

}  // namespace

int wide_launch_rope(wide_ctx* ctx, cudaStream_t s, const void* q, const void* k, int dtype, int tokens, int n_q, int n_kv,
                     int head_dim, int rot, long long qs, long long ks, const int32_t* positions, int n_axes,
                     const double* inv_freq, const int32_t* axis, void* q_out, void* k_out, long long oqs, long long oks,
                     unsigned flags) {
    RopeArgs a;
    a.q = q; a.k = k; a.q_out = q_out; a.k_out = k_out;
    a.qs = qs; a.ks = ks; a.oqs = oqs; a.oks = oks;
    a.positions = positions; a.inv_freq = inv_freq; a.axis = axis;
    a.tokens = tokens; a.n_q = n_q; a.n_kv = n_kv; a.rot = rot; a.n_axes = n_axes;
    a.interleaved = (flags & WIDE_FLAG_ROPE_INTERLEAVED) != 0;
    a.inverse = (flags & WIDE_FLAG_ROPE_INVERSE) != 0;
    const int elem = wide_elem_bytes(dtype);
    a.wide = wide_rows32(q, qs * elem) && wide_rows32(q_out, oqs * elem) && (!k || (wide_rows32(k, ks * elem) && wide_rows32(k_out, oks * elem)));
    a.status = ctx->d_status + WIDE_STATUS_INDEX;
    a.tile = tokens >= 8 * ctx->sm_count ? kMaxTile : 1;
    const int grid = (tokens + a.tile - 1) / a.tile;
    WideLaunch l(ctx, s, "rope");
    if (dtype == WIDE_F32) {
        if (head_dim == 128) WIDE_CUDA_CHECK(wide_launch_after(ctx, rope_kernel<float, 128>, dim3(grid), dim3(kThreads), 0, s, a));
        else WIDE_CUDA_CHECK(wide_launch_after(ctx, rope_kernel<float, 64>, dim3(grid), dim3(kThreads), 0, s, a));
    } else {
        if (head_dim == 128) WIDE_CUDA_CHECK(wide_launch_after(ctx, rope_kernel<__nv_bfloat16, 128>, dim3(grid), dim3(kThreads), 0, s, a));
        else WIDE_CUDA_CHECK(wide_launch_after(ctx, rope_kernel<__nv_bfloat16, 64>, dim3(grid), dim3(kThreads), 0, s, a));
    }
    return WIDE_OK;
}
