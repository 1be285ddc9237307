// Dense linear layer with its epilogue (wide_linear):  y[t, n] = act(sum_k x[t, k] w[n, k] + bias[n]) + residual[t, n].
//
// Weights are the 128-row operand of the tensor cores, tokens the other: D [128 output channels (TMEM lanes)][tokens (columns)] in fp32,
// so that a single token costs no more than the weights' bytes.  An epilogue warp has 32 channels of all the tile's tokens; it turns
// them round through its own part of shared memory, so that rows of y are read and written in runs of 64 or 128 bytes.
//
// Few tokens (linear_kernel): the weights' bytes bound it, and N / 128 tiles are fewer than SMs.  A cluster of CTAs shares a tile: each takes a
// part of K, and each joins the parts of some of the tokens over distributed shared memory, in the order of K, so results do not
// depend on timing.  One token 4096 -> 6144: 18.5 us with cold caches, 12.9 in a stream of calls (floor 7.7); 64 tokens 4096 -> 128256: 195 us, 82% of
// the memory's rate.
//
// Many tokens (linear_pair_kernel): pairs of SMs, below.  4096 tokens 4096 -> 14336: 299 us alone (1.61 PFLOP/s, the rate that the library's product reaches alone), 330 to 360 in a
// stream of calls, where the power cap holds the clocks down; short of that rate where the last round of tiles leaves SMs idle (2048 tokens 4096 -> 4096: 56 us,
// 1.23), and far from it with 129 to 1000 tokens, whose tiles are fewer than the pairs (256 tokens 4096 -> 6144: 29 us, the library 21.5).
#include <cuda.h>

#include <algorithm>
#include <atomic>

#include "internal.h"
#include "ptx.cuh"

namespace {

using namespace wptx;

constexpr int kM = 128;                 // output channels of a tile
constexpr int kBK = 64;                 // bf16 numbers of a 128-byte swizzle row
constexpr int kABytes = kM * kBK * 2;
constexpr int kThreads = 192;           // TMA, MMA, four epilogue warps
// fp32 outputs: after so many steps of kBK a sum goes on in the other accumulator, and the epilogue warps add the pieces up.  The tensor cores cut a sum
// off at every addition, towards zero, so that a long one drifts: 2-norm of the error 4.4e-6 at K = 4096 in one piece, 1.0e-6 in pieces of 16
// steps, 7e-7 of 12, 4.8e-7 of 8, whatever K.  With few tokens it costs nothing; 4096 tokens 4096 -> 14336 take 307, 338, 371, 394 us.  bf16 outputs,
// whose rounding is 1.7e-3 (2-norm), keep one piece up to kWhole steps: 65536 products of one sign lose 2.4e-4 there, a million would lose 2^-8.
constexpr int kChain = 12, kWhole = 1024;

struct LinearArgs {
    int T, N, nk;                       // nk: steps of kBK
    int tiles_n, split;
    const __nv_bfloat16* bias;
    const void* residual;
    void* y;
    long long rs, ys;                   // row strides in elements
    int act, out_f32;
    int* status;
    unsigned long long wait_ns;
};

__device__ __forceinline__ float reciprocal(float x) {       // within 1 unit of the last place; 0 for x above 2^126
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// v / (1 + exp(-z)).  Divided by 1 + exp(-z) as it stands, it would be 0 from z = -87 on, where the divisor passes 2^126, though the result is a normal number down to -92.
// EXACT keeps fp32's digits (8 units of the last place), with an exponential up to 1 (and a rounded quotient: 333 tokens 1000 -> 5003 with SiLU 24.7 us instead of
// 14).  For bf16 the fast exponential does, though its error grows with z up to 2^-16; divisor and dividend are taken times 2^-43, so that
// the divisor stays below 2^126 as far as there are results.
template <bool EXACT>
__device__ __forceinline__ float times_sigmoid(float v, float z) {
    if (EXACT) {
        const float e = expf(-fabsf(z)), r = reciprocal(1.f + e);
        return v * (z >= 0.f ? r : e * r);
    }
    constexpr float kUnit = 1.1368683772161603e-13f;
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fmaf(z, -1.4426950408889634f, -43.f)));
    return v * (kUnit * reciprocal(kUnit + e));
}
template <int ACT, bool EXACT>
__device__ __forceinline__ float activate(float v) {
    if (ACT == WIDE_ACT_SILU) return times_sigmoid<EXACT>(v, v);
    if (ACT == WIDE_ACT_GELU) return 0.5f * v * erfcf(-0.70710678118654752f * v);
    if (ACT == WIDE_ACT_GELU_TANH) return times_sigmoid<EXACT>(v, 1.5957691216057307f * fmaf(0.044715f * v * v, v, v));     // v (1 + tanh u) / 2 = v / (1 + exp(-2 u))
    return v;
}
template <bool EXACT>
__device__ __forceinline__ float activate(float v, int act) {
    switch (act) {
        case WIDE_ACT_SILU: return activate<WIDE_ACT_SILU, EXACT>(v);
        case WIDE_ACT_GELU: return activate<WIDE_ACT_GELU, EXACT>(v);
        case WIDE_ACT_GELU_TANH: return activate<WIDE_ACT_GELU_TANH, EXACT>(v);
        default: return v;
    }
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// (of converged warps only: an epilogue's lanes leave their loops after different numbers of tokens)
__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// the address in CTA `rank` of the cluster that `addr` is in this one
__device__ __forceinline__ uint32_t map_rank(uint32_t addr, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
__device__ __forceinline__ float4 ld_cluster(uint32_t a) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}

// four neighbouring outputs of a row from channel f on: the residual, rounding
__device__ __forceinline__ void put(const LinearArgs& a, long long t, int f, float (&x)[4]) {
    const int n = min(4, a.N - f);
    if (a.out_f32) {
        float* y = static_cast<float*>(a.y) + t * a.ys + f;
        const float* r = static_cast<const float*>(a.residual) + t * a.rs + f;
        if (n == 4) {
            if (a.residual) {
                const float4 z = *reinterpret_cast<const float4*>(r);
                x[0] += z.x, x[1] += z.y, x[2] += z.z, x[3] += z.w;
            }
            *reinterpret_cast<float4*>(y) = make_float4(x[0], x[1], x[2], x[3]);
        } else {
            for (int e = 0; e < n; ++e) y[e] = x[e] + (a.residual ? r[e] : 0.f);
        }
    } else {
        __nv_bfloat16* y = static_cast<__nv_bfloat16*>(a.y) + t * a.ys + f;
        const __nv_bfloat16* r = static_cast<const __nv_bfloat16*>(a.residual) + t * a.rs + f;
        if (n == 4) {
            if (a.residual) {
                const uint2 z = *reinterpret_cast<const uint2*>(r);
                x[0] += __uint_as_float(z.x << 16), x[1] += __uint_as_float(z.x & 0xFFFF0000u);
                x[2] += __uint_as_float(z.y << 16), x[3] += __uint_as_float(z.y & 0xFFFF0000u);
            }
            const __nv_bfloat162 p = __floats2bfloat162_rn(x[0], x[1]), q = __floats2bfloat162_rn(x[2], x[3]);
            *reinterpret_cast<uint2*>(y) = make_uint2(*reinterpret_cast<const uint32_t*>(&p), *reinterpret_cast<const uint32_t*>(&q));
        } else {
            for (int e = 0; e < n; ++e) y[e] = __float2bfloat16_rn(x[e] + (a.residual ? __bfloat162float(r[e]) : 0.f));
        }
    }
}

__device__ __forceinline__ void finish(const LinearArgs& a, long long t, int f, float4 v, const float (&bias)[4]) {
    float x[4] = {v.x + bias[0], v.y + bias[1], v.z + bias[2], v.w + bias[3]};
    if (a.act != WIDE_ACT_NONE) {
        if (a.out_f32) {
#pragma unroll 1
            for (int e = 0; e < 4; ++e) {       // (a loop, as the code of four exact activations of each kind slows every call of few tokens down by a tenth)
                const float y = activate<true>(x[0], a.act);
                x[0] = x[1], x[1] = x[2], x[2] = x[3], x[3] = y;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = activate<false>(x[e], a.act);
        }
    }
    put(a, t, f, x);
}

// Stages such that two CTAs fit on an SM: with one, a cluster of four or eight often has to wait for SMs of its own (128 tokens, 4096 x 4096: 37
// us with one, 22.5 with two; 48 tokens 24.6 and 18.4).
template <int NT>
struct Small {
    static constexpr int kStages = NT == 16 ? 6 : NT == 32 ? 5 : NT == 64 ? 4 : 3, kStage = kABytes + NT * kBK * 2, kSmem = kStages * kStage + 1024;
};

// A tile of 128 channels and all tokens, at most NT, a cluster: weights are read once.
template <int NT, bool CHAIN>
__global__ void __launch_bounds__(kThreads) linear_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x,
                                                          const __grid_constant__ LinearArgs a) {
    constexpr int kStages = Small<NT>::kStages, kStage = Small<NT>::kStage;
    constexpr uint32_t kCols = CHAIN ? 2 * NT : NT < 32 ? 32 : NT;
    static_assert(kStages * kStage >= NT * kM * 4, "the parts of a tile take the place of the stages");
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kStages + 4];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t full = smem_u32(bars), empty = smem_u32(bars + kStages), done = smem_u32(bars + 2 * kStages), taken = smem_u32(bars + 2 * kStages + 2);
    volatile int* abort_flag = &abort_word;
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(done + 8 * s, 1);
            mbar_init(taken + 8 * s, 4);
        }
        abort_word = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_w);
        prefetch_tmap(&tm_x);
    }
    grid_dep_wait();
    // (Tensor memory is taken after the kernel before has ended and before the next may come: no two wait for each other's.)
    if (warp == 1) {
        tmem_alloc(smem_u32(&tmem_slot), kCols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    const int rank = a.split > 1 ? static_cast<int>(cluster_rank()) : 0;
    const int tile = blockIdx.x / a.split;
    const int k0 = static_cast<int>(static_cast<long long>(a.nk) * rank / a.split), k1 = static_cast<int>(static_cast<long long>(a.nk) * (rank + 1) / a.split);
    grid_dep_launch();

    if (warp == 0) {
        if (lane == 0) {
            const uint64_t once = l2_policy_evict_first();
            for (int k = k0; k < k1; ++k) {
                const int i = k - k0, s = i % kStages;
                if (!mbar_wait(empty + 8 * s, ((i / kStages) & 1) ^ 1u, a.wait_ns, abort_flag)) break;
                mbar_arrive_expect_tx(full + 8 * s, kStage);
                const uint32_t at = smem_u32(base + s * kStage);
                tma_load_2d_hint(at, &tm_w, k * kBK, tile * kM, full + 8 * s, once);
                tma_load_2d(at + kABytes, &tm_x, k * kBK, 0, full + 8 * s);
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            bool ok = true;
            for (int k = k0; k < k1 && ok; ++k) {
                const int i = k - k0, s = i % kStages, piece = CHAIN ? i / kChain : 0;
                if (CHAIN && i % kChain == 0) {
                    if (piece > 0) umma_commit(done + 8 * ((piece - 1) & 1));
                    if (piece >= 2 && !(ok = mbar_wait(taken + 8 * (piece & 1), ((piece >> 1) & 1) ^ 1, a.wait_ns, abort_flag))) break;
                }
                ok = mbar_wait(full + 8 * s, (i / kStages) & 1, a.wait_ns, abort_flag);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t at = smem_u32(base + s * kStage);
                const uint64_t wd = umma_desc_sw128(at), xd = umma_desc_sw128(at + kABytes);
#pragma unroll
                for (int e = 0; e < kBK / 16; ++e) umma_bf16(tmem + (piece & 1) * NT, wd + 2 * e, xd + 2 * e, umma_idesc_bf16(kM, NT), ((CHAIN ? i % kChain : i) | e) ? 1u : 0u);
                umma_commit(empty + 8 * s);
            }
            if (ok) umma_commit(done + (CHAIN ? 8 * (((k1 - k0 - 1) / kChain) & 1) : 0));
        }
    }
    __syncwarp();
    // ---- epilogue: warps 2..5, of the TMEM lanes that a warp's number gives it
    const int quarter = warp & 3;
    float* parts = reinterpret_cast<float*>(base);      // [token][128]: every stage has been read when `done` completes
    bool ok = true;
    if (warp >= 2) {
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
        if constexpr (CHAIN) {
            float sum[NT];
            const int pieces = (k1 - k0 + kChain - 1) / kChain;
            for (int c = 0; c < pieces; ++c) {
                if (!(ok = mbar_wait_warp(done + 8 * (c & 1), (c >> 1) & 1, a.wait_ns, abort_flag))) break;
                tc_fence_after_sync();
#pragma unroll
                for (int t = 0; t < NT; t += 16) {
                    uint32_t r[16];
                    tmem_ld_32x16(lanes + (c & 1) * NT + t, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum[t + e] = c == 0 ? __uint_as_float(r[e]) : sum[t + e] + __uint_as_float(r[e]);
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(taken + 8 * (c & 1));
            }
            if (ok) {
#pragma unroll
                for (int t = 0; t < NT; ++t) parts[t * kM + quarter * 32 + lane] = sum[t];
            }
        } else {
            ok = mbar_wait_warp(done, 0, a.wait_ns, abort_flag);
            tc_fence_after_sync();
            if (ok) {
#pragma unroll 1
                for (int c = 0; c < NT; c += 16) {
                    uint32_t r[16];
                    tmem_ld_32x16(lanes + c, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; ++e) parts[(c + e) * kM + quarter * 32 + lane] = __uint_as_float(r[e]);
                }
            }
        }
        if (!ok && lane == 0) atomicExch(a.status, WIDE_ERR_TIMEOUT);
        __syncwarp();
    }
    if (a.split > 1) {
        cluster_arrive();
        cluster_wait();
    }
    if (warp >= 2 && ok) {
        const int t0 = NT * rank / a.split, t1 = NT * (rank + 1) / a.split;      // the tokens that this CTA joins
        const int f = tile * kM + quarter * 32 + (lane & 7) * 4;
        float bias[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[e] = a.bias && f + e < a.N ? __bfloat162float(a.bias[f + e]) : 0.f;
        const uint32_t mine = smem_u32(parts) + (quarter * 32 + (lane & 7) * 4) * 4;
        if (f < a.N) {
            for (int t = t0 + (lane >> 3); t < t1 && t < a.T; t += 4) {
                float4 v;
                if (a.split == 1) {
                    v = *reinterpret_cast<const float4*>(parts + t * kM + quarter * 32 + (lane & 7) * 4);
                } else {
                    v = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int p = 0; p < a.split; ++p) {
                        const float4 z = ld_cluster(map_rank(mine + t * kM * 4, p));
                        v = make_float4(v.x + z.x, v.y + z.y, v.z + z.z, v.w + z.w);
                    }
                }
                finish(a, t, f, v, bias);
            }
        }
    }
    if (a.split > 1) {       // no CTA leaves while its part may be read
        cluster_arrive();
        cluster_wait();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) let_copies_land();
    if (warp == 1) tmem_dealloc(tmem, kCols);
}

// ------------------------------------------------------------------------------------------------ many tokens
// Pairs of CTAs (cta_group::2) take tiles of 256 channels and 256 tokens: each brings 128 rows of both operands for a product that reads
// the two SMs' shared memory, 7.8 bytes a kFLOP from L2, where 128 x 256 tiles of one SM need 11.7 and end at 1.0 PFLOP/s.  A CTA has its 128 channels
// (TMEM lanes) of all 256 tokens in one of two accumulators, so the epilogue of a tile runs under the next one's products.  Persistent;
// tiles go by bands of 16 token tiles, channels within them, so that a band's tokens stay in L2.
// Tiles of 128 tokens fill SMs that 256 leave idle (256 tokens, 4096 -> 6144: 34 us with 256, 30 with 128; 512, 4096 -> 4096: 32, 28).
constexpr int kPairEpi = 8;                                     // epilogue warps: two for each quarter of the lanes
constexpr int kPairThreads = 64 + 32 * kPairEpi;
constexpr int kBand = 16;
template <int PT>
struct Pair {
    static constexpr int kStages = PT == 256 ? 6 : 8, kStage = kABytes + PT * kBK;     // (half of the tokens a CTA)
    static constexpr int kSmem = kStages * kStage + kPairEpi * 32 * 32 * 4 + 1024;
};

// 32 tokens of a warp's 32 channels, which lie in its shared memory as [token][channel]: a lane has channels f .. f + 3 of every fourth token.  Bias and
// activation are a short loop of their own, in place: unrolled among the loads and stores below, the activation of 32 values was
// more code than the instruction cache holds (333 tokens 1000 -> 5003 with GELU: 25.5 us against 16.8).
template <int ACT, bool EXACT>
__device__ __forceinline__ void activate_block(float* block, int lane, const float (&bias)[4]) {
#pragma unroll 1
    for (int j = 0; j < 8; j += 2) {
        float4* at = reinterpret_cast<float4*>(block + (4 * j + (lane >> 3)) * 32 + (lane & 7) * 4);
        const float4 v = at[0], w = at[32];
        at[0] = make_float4(activate<ACT, EXACT>(v.x + bias[0]), activate<ACT, EXACT>(v.y + bias[1]), activate<ACT, EXACT>(v.z + bias[2]), activate<ACT, EXACT>(v.w + bias[3]));
        at[32] = make_float4(activate<ACT, EXACT>(w.x + bias[0]), activate<ACT, EXACT>(w.y + bias[1]), activate<ACT, EXACT>(w.z + bias[2]), activate<ACT, EXACT>(w.w + bias[3]));
    }
}
__device__ __noinline__ void activate_any(float* block, int lane, int act, int exact, float b0, float b1, float b2, float b3) {
    const float bias[4] = {b0, b1, b2, b3};
    if (act == WIDE_ACT_GELU) activate_block<WIDE_ACT_GELU, true>(block, lane, bias);       // (the same for both types)
    else if (act == WIDE_ACT_SILU && exact) activate_block<WIDE_ACT_SILU, true>(block, lane, bias);
    else if (act == WIDE_ACT_SILU) activate_block<WIDE_ACT_SILU, false>(block, lane, bias);
    else if (exact) activate_block<WIDE_ACT_GELU_TANH, true>(block, lane, bias);
    else activate_block<WIDE_ACT_GELU_TANH, false>(block, lane, bias);
}
// All eight pieces of a lane together, from token t on, so that their loads overlap; `bias` is still to be added.
__device__ __forceinline__ void finish_block(const LinearArgs& a, long long t, int f, const float* block, int lane, const float (&bias)[4]) {
    float x[8][4];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float4 v = *reinterpret_cast<const float4*>(block + (4 * j + (lane >> 3)) * 32 + (lane & 7) * 4);
        x[j][0] = v.x + bias[0], x[j][1] = v.y + bias[1], x[j][2] = v.z + bias[2], x[j][3] = v.w + bias[3];
    }
    const long long row = t + (lane >> 3);
    if (a.out_f32) {
        if (a.residual) {
            const float* r = static_cast<const float*>(a.residual) + row * a.rs + f;
            float4 z[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = *reinterpret_cast<const float4*>(r + 4 * j * a.rs);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j][0] += z[j].x, x[j][1] += z[j].y, x[j][2] += z[j].z, x[j][3] += z[j].w;
        }
        float* y = static_cast<float*>(a.y) + row * a.ys + f;
#pragma unroll
        for (int j = 0; j < 8; ++j) *reinterpret_cast<float4*>(y + 4 * j * a.ys) = make_float4(x[j][0], x[j][1], x[j][2], x[j][3]);
    } else {
        if (a.residual) {
            const __nv_bfloat16* r = static_cast<const __nv_bfloat16*>(a.residual) + row * a.rs + f;
            uint2 z[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = *reinterpret_cast<const uint2*>(r + 4 * j * a.rs);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j][0] += __uint_as_float(z[j].x << 16), x[j][1] += __uint_as_float(z[j].x & 0xFFFF0000u);
                x[j][2] += __uint_as_float(z[j].y << 16), x[j][3] += __uint_as_float(z[j].y & 0xFFFF0000u);
            }
        }
        __nv_bfloat16* y = static_cast<__nv_bfloat16*>(a.y) + row * a.ys + f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(x[j][0], x[j][1]), q = __floats2bfloat162_rn(x[j][2], x[j][3]);
            *reinterpret_cast<uint2*>(y + 4 * j * a.ys) = make_uint2(*reinterpret_cast<const uint32_t*>(&p), *reinterpret_cast<const uint32_t*>(&q));
        }
    }
}

// As tma_load_2d, the bytes counted by the even CTA's barrier of the pair (the same address with its rank cleared).
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* m, int c0, int c1, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar & 0xFEFFFFFFu), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void umma_bf16_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Arrives on the barrier at this address in both CTAs once the pair's products so far are done.
__device__ __forceinline__ void umma_commit_pair(uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(bar), "h"(static_cast<uint16_t>(3))
        : "memory");
}
__device__ __forceinline__ void arrive_rank0(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(map_rank(bar, 0)) : "memory");
}

template <int PT, bool CHAIN>
__global__ void __launch_bounds__(kPairThreads, 1) __cluster_dims__(2, 1, 1)
linear_pair_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ LinearArgs a) {
    constexpr int kPairStages = Pair<PT>::kStages, kPairStage = Pair<PT>::kStage, kPairT = PT;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kPairStages + 4];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = static_cast<int>(cluster_rank());
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t full = smem_u32(bars), empty = smem_u32(bars + kPairStages), tfull = smem_u32(bars + 2 * kPairStages), tempty = smem_u32(bars + 2 * kPairStages + 2);
    volatile int* abort_flag = &abort_word;
    if (tid == 0) {
        for (int s = 0; s < kPairStages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(tfull + 8 * s, 1);
            mbar_init(tempty + 8 * s, 2 * kPairEpi);
        }
        abort_word = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_w);
        prefetch_tmap(&tm_x);
    }
    grid_dep_wait();
    // (Tensor memory is taken after the kernel before has ended and before the next may come: no two wait for each other's.)
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(2u * PT) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_arrive();
    cluster_wait();            // the other CTA's barriers and tensor memory are there
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    grid_dep_launch();
    const int tiles_t = (a.T + kPairT - 1) / kPairT, tiles_n = (a.N + 2 * kM - 1) / (2 * kM);
    const long long tiles = static_cast<long long>(tiles_t) * tiles_n;
    const int pairs = gridDim.x >> 1;
    struct At {
        int t, n;
    };
    auto tile_at = [&](long long i) {
        const long long per_band = static_cast<long long>(kBand) * tiles_n;
        const int band = static_cast<int>(i / per_band), in = static_cast<int>(i - band * per_band);
        const int wide = min(kBand, tiles_t - band * kBand);
        return At{band * kBand + in % wide, in / wide};
    };
    bool ok = true;
    if (warp == 0) {
        // ------------------------------------------------------------------ TMA: 128 rows of each operand
        if (lane == 0) {
            int it = 0;
            for (long long i = blockIdx.x >> 1; i < tiles && ok; i += pairs) {
                const At at = tile_at(i);
                const int row_w = at.n * 2 * kM + rank * kM, row_x = at.t * kPairT + rank * (kPairT / 2);
                for (int k = 0; k < a.nk; ++k, ++it) {
                    const int s = it % kPairStages;
                    if (!(ok = mbar_wait(empty + 8 * s, ((it / kPairStages) & 1) ^ 1u, a.wait_ns, abort_flag))) break;
                    if (rank == 0) mbar_arrive_expect_tx(full + 8 * s, 2 * kPairStage);     // both CTAs' bytes
                    const uint32_t to = smem_u32(base + s * kPairStage);
                    tma_load_2d_pair(to, &tm_w, k * kBK, row_w, full + 8 * s);
                    tma_load_2d_pair(to + kABytes, &tm_x, k * kBK, row_x, full + 8 * s);
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ products, by the even CTA
        if (rank == 0) {
            int it = 0, n = 0;
            for (long long i = blockIdx.x >> 1; i < tiles && ok; i += pairs, ++n) {       // n: accumulators filled
                if (n >= 2 && !(ok = mbar_wait_warp(tempty + 8 * (n & 1), ((n >> 1) & 1) ^ 1u, a.wait_ns, abort_flag))) break;
                tc_fence_after_sync();
                for (int k = 0; k < a.nk; ++k, ++it) {
                    const int s = it % kPairStages;
                    if (CHAIN && k > 0 && k % kChain == 0) {
                        umma_commit_pair(tfull + 8 * (n & 1));
                        ++n;
                        if (n >= 2 && !(ok = mbar_wait_warp(tempty + 8 * (n & 1), ((n >> 1) & 1) ^ 1u, a.wait_ns, abort_flag))) break;
                        tc_fence_after_sync();
                    }
                    if (!(ok = mbar_wait_warp(full + 8 * s, (it / kPairStages) & 1, a.wait_ns, abort_flag))) break;
                    tc_fence_after_sync();
                    const uint32_t from = smem_u32(base + s * kPairStage);
                    const uint64_t wd = umma_desc_sw128(from), xd = umma_desc_sw128(from + kABytes);
#pragma unroll
                    for (int e = 0; e < kBK / 16; ++e)
                        umma_bf16_pair(tmem + (n & 1) * kPairT, wd + 2 * e, xd + 2 * e, umma_idesc_bf16(2 * kM, kPairT), ((CHAIN ? k % kChain : k) | e) ? 1u : 0u);
                    umma_commit_pair(empty + 8 * s);
                }
                if (ok) umma_commit_pair(tfull + 8 * (n & 1));
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue: 32 channels of half of the tokens a warp
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        float* mine = reinterpret_cast<float*>(base + kPairStages * kPairStage) + (warp - 2) * 32 * 32;      // [token][channel]
        int n = 0;
        for (long long i = blockIdx.x >> 1; i < tiles; i += pairs, ++n) {
            const At at = tile_at(i);
            const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + half * (kPairT / 2);
            const int f = at.n * 2 * kM + rank * kM + quarter * 32 + (lane & 7) * 4;
            float bias[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) bias[e] = a.bias && f + e < a.N ? __bfloat162float(a.bias[f + e]) : 0.f;
            float left[4];          // of the bias, behind the activation
#pragma unroll
            for (int e = 0; e < 4; ++e) left[e] = a.act == WIDE_ACT_NONE ? bias[e] : 0.f;
            auto finish_32 = [&](int c) {          // the tokens from c on of this warp's half, which lie in its shared memory
                __syncwarp();
                const int t0 = at.t * kPairT + half * (kPairT / 2) + c;
                if (a.act != WIDE_ACT_NONE && t0 < a.T) activate_any(mine, lane, a.act, a.out_f32, bias[0], bias[1], bias[2], bias[3]);
                if (f + 3 < a.N && t0 + 32 <= a.T) {
                    finish_block(a, t0, f, mine, lane, left);
                } else if (f < a.N) {
#pragma unroll 1
                    for (int e = lane >> 3; e < 32 && t0 + e < a.T; e += 4) {
                        const float4 v = *reinterpret_cast<const float4*>(mine + e * 32 + (lane & 7) * 4);
                        float x[4] = {v.x + left[0], v.y + left[1], v.z + left[2], v.w + left[3]};
                        put(a, static_cast<long long>(t0) + e, f, x);
                    }
                }
                __syncwarp();
            };
            if constexpr (CHAIN) {
                float sum[kPairT / 2];
                for (int k = 0; k < a.nk; k += kChain, ++n) {
                    if (!(ok = mbar_wait_warp(tfull + 8 * (n & 1), (n >> 1) & 1, a.wait_ns, abort_flag))) break;
                    tc_fence_after_sync();
#pragma unroll
                    for (int c = 0; c < kPairT / 2; c += 16) {
                        uint32_t r[16];
                        tmem_ld_32x16(lanes + (n & 1) * kPairT + c, r);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) sum[c + e] = k == 0 ? __uint_as_float(r[e]) : sum[c + e] + __uint_as_float(r[e]);
                    }
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) arrive_rank0(tempty + 8 * (n & 1));
                }
                if (!ok) break;
                --n;
#pragma unroll
                for (int c = 0; c < kPairT / 2; c += 32) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) mine[e * 32 + lane] = sum[c + e];
                    finish_32(c);
                }
            } else {
                if (!(ok = mbar_wait_warp(tfull + 8 * (n & 1), (n >> 1) & 1, a.wait_ns, abort_flag))) break;
                tc_fence_after_sync();
#pragma unroll 1
                for (int c = 0; c < kPairT / 2; c += 32) {
                    uint32_t r[32];
                    tmem_ld_32x32(lanes + (n & 1) * kPairT + c, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; ++e) mine[e * 32 + lane] = __uint_as_float(r[e]);
                    finish_32(c);
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) arrive_rank0(tempty + 8 * (n & 1));
            }
        }
    }
    if (!ok && lane == 0) atomicExch(a.status, WIDE_ERR_TIMEOUT);
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) let_copies_land();
    cluster_arrive();
    cluster_wait();            // no CTA leaves while the other may still reach into it
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2u * PT) : "memory");
}

// bf16 rows `stride` bytes apart, box [rows, 64 columns], 128-byte swizzle
bool make_map(const wide_ctx* ctx, CUtensorMap* map, const void* base, long long rows, long long cols, long long stride, uint32_t box_rows) {
    typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                               const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(stride)};
    const cuuint32_t box[2] = {kBK, box_rows}, each[2] = {1, 1};
    return reinterpret_cast<Encode>(ctx->encode_tiled)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, each,
                                                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Once a device and kernel; threads that come here together all set the same.
template <typename K>
bool allow_smem(const wide_ctx* ctx, K kernel, int bytes, std::atomic<unsigned>& set) {
    const unsigned bit = ctx->device < 32 ? 1u << ctx->device : 0u;
    if (bit && (set.load(std::memory_order_relaxed) & bit)) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    set.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

template <int NT, bool CHAIN>
int launch_small(wide_ctx* ctx, cudaStream_t s, LinearArgs a, const void* x, long long xs, const void* w, int K) {
    CUtensorMap tm_w, tm_x;
    if (!make_map(ctx, &tm_w, w, a.N, K, 2LL * K, kM) || !make_map(ctx, &tm_x, x, a.T, K, 2 * xs, NT)) return WIDE_ERR_CUDA;
    static std::atomic<unsigned> set{0};
    if (!allow_smem(ctx, linear_kernel<NT, CHAIN>, Small<NT>::kSmem, set)) return WIDE_ERR_CUDA;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(a.tiles_n * a.split));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Small<NT>::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = a.split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ctx->prof ? 1 : 2;
    WideLaunch l(ctx, s, "linear");
    WIDE_CUDA_CHECK(cudaLaunchKernelEx(&cfg, linear_kernel<NT, CHAIN>, tm_w, tm_x, a));
    return WIDE_OK;
}

// T <= NT
template <int NT>
int launch(wide_ctx* ctx, cudaStream_t s, LinearArgs a, const void* x, long long xs, const void* w, int K) {
    a.split = 1;
    // CTAs for three quarters of the SMs at least, as long as each keeps 8 steps of K (one token, 4096 x 4096: 4 parts 16.4 us, 8 parts 18.4)
    while (a.split < 8 && 4LL * a.tiles_n * a.split < 3 * ctx->sm_count && a.nk / (2 * a.split) >= 8) a.split *= 2;
    return a.nk > (a.out_f32 ? kChain : kWhole) * a.split ? launch_small<NT, true>(ctx, s, a, x, xs, w, K) : launch_small<NT, false>(ctx, s, a, x, xs, w, K);
}

template <int PT>
long long pair_tiles(const LinearArgs& a) {
    return static_cast<long long>((a.T + PT - 1) / PT) * ((a.N + 2 * kM - 1) / (2 * kM));
}

template <int PT, bool CHAIN>
int launch_pairs(wide_ctx* ctx, cudaStream_t s, LinearArgs a, const void* x, long long xs, const void* w, int K) {
    CUtensorMap tm_w, tm_x;
    if (!make_map(ctx, &tm_w, w, a.N, K, 2LL * K, kM) || !make_map(ctx, &tm_x, x, a.T, K, 2 * xs, PT / 2)) return WIDE_ERR_CUDA;
    static std::atomic<unsigned> set{0};
    if (!allow_smem(ctx, linear_pair_kernel<PT, CHAIN>, Pair<PT>::kSmem, set)) return WIDE_ERR_CUDA;
    const int pairs = static_cast<int>(std::min<long long>(pair_tiles<PT>(a), ctx->sm_count / 2));
    WideLaunch l(ctx, s, "linear_pair");
    WIDE_CUDA_CHECK(wide_launch_after(ctx, linear_pair_kernel<PT, CHAIN>, dim3(2 * pairs), dim3(kPairThreads), Pair<PT>::kSmem, s, tm_w, tm_x, a));
    return WIDE_OK;
}

}  // namespace

int wide_launch_linear(wide_ctx* ctx, cudaStream_t s, const void* x, int T, int K, long long xs, const void* w, int N, const void* bias, int act,
                       const void* residual, long long rs, void* y, int out_dtype, long long ys) {
    LinearArgs a{};
    a.T = T;
    a.N = N;
    a.nk = (K + kBK - 1) / kBK;
    a.tiles_n = (N + kM - 1) / kM;
    a.bias = static_cast<const __nv_bfloat16*>(bias);
    a.residual = residual;
    a.y = y;
    a.rs = rs;
    a.ys = ys;
    a.act = act;
    a.out_f32 = out_dtype == WIDE_F32;
    a.status = ctx->d_status;
    a.wait_ns = ctx->wait_ns;
    if (T <= 16) return launch<16>(ctx, s, a, x, xs, w, K);
    if (T <= 32) return launch<32>(ctx, s, a, x, xs, w, K);
    if (T <= 64) return launch<64>(ctx, s, a, x, xs, w, K);
    if (T <= 128) return launch<128>(ctx, s, a, x, xs, w, K);
    // Rounds of the pairs; a tile of 128 tokens takes 0.65 to 0.8 of one of 256, not half, as it reads shared memory at twice the rate for its
    // products (1024 tokens, 4096 -> 6144, three rounds of 128: 62 us, two of 256: 54).
    const long long pairs = ctx->sm_count / 2, wide = (pair_tiles<256>(a) + pairs - 1) / pairs, narrow = (pair_tiles<128>(a) + pairs - 1) / pairs;
    const bool chain = a.nk > (a.out_f32 ? kChain : kWhole);
    if (8 * narrow < 10 * wide) return chain ? launch_pairs<128, true>(ctx, s, a, x, xs, w, K) : launch_pairs<128, false>(ctx, s, a, x, xs, w, K);
    return chain ? launch_pairs<256, true>(ctx, s, a, x, xs, w, K) : launch_pairs<256, false>(ctx, s, a, x, xs, w, K);
}
