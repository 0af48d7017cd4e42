// qless_token_loss of one to four tokens, alone or with dH: one pass over W.
//
// Bound: memory, W is read once (the tile kernels read it for the logits and again for dH).  A workgroup takes a contiguous share of the
// vocabulary, a thread 8 KU columns of all its rows, so that a row that has been multiplied with the tokens for its logits is
// still in registers when its probability is known: batches of RB rows (16 to 32 KB) are requested one ahead, their logits summed over the
// workgroup, and acc = acc exp(m_before - m) + sum_v exp(z_v - m) W_v (v not the target) with the running maximum m, all in fp32.  The vector units take
// 4 + 4 T operations for two columns of a row, a third of the memory's time for one token and about as long for four.  The workgroups' maxima,
// sums and rows of acc are joined by a second kernel, which adds the target's part.
#include "token_loss.h"
#include "score.h"
#include <type_traits>

namespace qless {

constexpr int kSingleGroups = 2048;            // at most

struct SingleArgs {
    const uint16_t *H; int64_t ldH;
    const uint16_t *W; int64_t ldW;
    const int64_t *target; const float *weight;
    int32_t T, D, V, share;                    // share: rows of W of a workgroup
    float *hit;                                // [T]
    float2 *part;                              // [groups][T]
    float *planes;                             // [groups][T][Dp]
    int64_t Dp;
    float *nll, *lse;
    uint16_t *dH; int64_t ldDH;
};

__device__ inline float low_half(uint32_t x) { return __uint_as_float(x << 16); }
__device__ inline float high_half(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }

// The sum over the wavefront, in its last lane.
template <int CTRL, int ROWS> __device__ inline float dpp_add(float x) {
    return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, ROWS, 0xF, false));
}
__device__ inline float wave_sum_last(float x) {
    x = dpp_add<0x111, 0xF>(x); x = dpp_add<0x112, 0xF>(x); x = dpp_add<0x114, 0xF>(x); x = dpp_add<0x118, 0xF>(x);
    x = dpp_add<0x142, 0xA>(x);
    return dpp_add<0x143, 0xC>(x);
}

template <int TT, int KU, int NW, bool DH>
__global__ void __launch_bounds__(64 * NW, 2)
loss_single_kernel(SingleArgs a) {
    constexpr int RB = (TT == 4 || TT * KU == 8 ? 4 : 8) / KU, N = RB * TT;        // as registers allow
    __shared__ __attribute__((aligned(16))) float s_part[2][NW][N];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int v0 = (int)blockIdx.x * a.share, v1 = v0 + a.share < a.V ? v0 + a.share : a.V;
    int64_t y[TT];
    float h[TT][KU][8], acc[TT][KU][8], top[TT], sum[TT];
    int col[KU];
#pragma unroll
    for (int k = 0; k < KU; ++k) col[k] = (tid + 64 * NW * k) * 8;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        y[t] = t < a.T ? a.target[t] : -1;
        if (y[t] >= a.V) y[t] = -1;
        top[t] = -INFINITY; sum[t] = 0.0f;
#pragma unroll
        for (int k = 0; k < KU; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                acc[t][k][i] = 0.0f;
                h[t][k][i] = y[t] >= 0 && col[k] < a.D ? low_half(a.H[t * a.ldH + col[k] + i]) : 0.0f;
            }
    }
    uint4 now[RB][KU], next[RB][KU];
    auto request = [&](uint4 (&x)[RB][KU], int v) {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const uint16_t *row = a.W + (int64_t)(v + r < v1 ? v + r : v1 - 1) * a.ldW;
#pragma unroll
            for (int k = 0; k < KU; ++k) x[r][k] = *(const uint4 *)(row + (col[k] < a.D ? col[k] : 0));
        }
    };
    int buffer = 0;
    auto batch = [&](uint4 (&x)[RB][KU], int v) {
        float z[N];                                        // [row][token]
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < KU; ++k) {
                    const uint32_t w[4] = {x[r][k].x, x[r][k].y, x[r][k].z, x[r][k].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) s = __builtin_fmaf(high_half(w[i]), h[t][k][2 * i + 1], __builtin_fmaf(low_half(w[i]), h[t][k][2 * i], s));
                }
                z[r * TT + t] = wave_sum_last(s);
            }
        if (lane == 63)
#pragma unroll
            for (int i = 0; i < N; ++i) s_part[buffer][wave][i] = z[i];
        __syncthreads();                                   // (the other buffer's readers have passed the barrier before this one)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            z[i] = s_part[buffer][0][i];
#pragma unroll
            for (int w = 1; w < NW; ++w) z[i] += s_part[buffer][w][i];
        }
        buffer ^= 1;
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            float m = top[t];
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                if (v + r >= v1) z[r * TT + t] = -INFINITY;
                m = fmaxf(m, z[r * TT + t]);
            }
            const float ref = m == -INFINITY ? 0.0f : m, shrink = top[t] == -INFINITY ? 0.0f : __expf(top[t] - ref);
            top[t] = m;
            sum[t] *= shrink;
            float p[RB];
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                p[r] = __expf(z[r * TT + t] - ref);
                if (v + r == y[t] && v + r < v1) {         // the same for the workgroup
                    p[r] = 0.0f;
                    if (tid == 0) a.hit[t] = z[r * TT + t];
                }
                sum[t] += p[r];
            }
            if (!DH) continue;
#pragma unroll
            for (int k = 0; k < KU; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[t][k][i] *= shrink;
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int k = 0; k < KU; ++k) {
                    const uint32_t w[4] = {x[r][k].x, x[r][k].y, x[r][k].z, x[r][k].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        acc[t][k][2 * i] = __builtin_fmaf(p[r], low_half(w[i]), acc[t][k][2 * i]);
                        acc[t][k][2 * i + 1] = __builtin_fmaf(p[r], high_half(w[i]), acc[t][k][2 * i + 1]);
                    }
                }
        }
    };
    if (v0 < v1) request(now, v0);
    for (int v = v0; v < v1; v += 2 * RB) {
        if (v + RB < v1) request(next, v + RB);
        batch(now, v);
        if (v + RB >= v1) break;
        if (v + 2 * RB < v1) request(now, v + 2 * RB);
        batch(next, v + RB);
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        if (t >= a.T) break;
        if (tid == 0) a.part[(int64_t)blockIdx.x * a.T + t] = make_float2(top[t], sum[t]);
        if (!DH) continue;
        float *out = a.planes + ((int64_t)blockIdx.x * a.T + t) * a.Dp;
#pragma unroll
        for (int k = 0; k < KU; ++k)
            if (col[k] < a.D) {
                *(float4 *)(out + col[k]) = make_float4(acc[t][k][0], acc[t][k][1], acc[t][k][2], acc[t][k][3]);
                *(float4 *)(out + col[k] + 4) = make_float4(acc[t][k][4], acc[t][k][5], acc[t][k][6], acc[t][k][7]);
            }
    }
}

// Grid (tokens, 16 columns, or one workgroup where dH is null): the workgroups' parts of a token joined, four columns a thread, 64 threads sharing the planes, the first of which are
// requested before the parts are (1 x 2048 x 32000: 5.6 us; with 16 threads, and none ahead, 8.3).
__global__ void __launch_bounds__(256)
loss_single_join_kernel(SingleArgs a, int groups) {
    __shared__ float s_top[4], s_sum[4], s_factor[kSingleGroups];
    __shared__ float4 s_acc[16];
    constexpr int AHEAD = 8;
    const int tid = threadIdx.x, t = blockIdx.x, sub = tid >> 2;
    const int64_t y = a.target[t];
    const bool live = y >= 0 && y < a.V;
    const int c = (int)blockIdx.y * 16 + (tid & 3) * 4;
    uint16_t *out = a.dH + t * a.ldDH + c;
    if (!live) {
        if (tid < 4 && a.dH)
#pragma unroll
            for (int u = 0; u < 4; ++u) if (c + u < a.D) out[u] = 0;
        if (tid == 0 && blockIdx.y == 0) {
            a.nll[t] = 0.0f;
            if (a.lse) a.lse[t] = 0.0f;
        }
        return;
    }
    const bool on = a.dH && c < a.D;                               // D is a multiple of eight
    auto plane = [&](int g) { return on && g < groups ? *(const float4 *)(a.planes + ((int64_t)g * a.T + t) * a.Dp + c) : make_float4(0.0f, 0.0f, 0.0f, 0.0f); };
    float4 ahead[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ahead[i] = plane(sub + 64 * i);
    uint16_t of_target[4] = {0, 0, 0, 0};
    if (on) __builtin_memcpy(of_target, __builtin_assume_aligned(a.W + y * a.ldW + c, 8), 8);
    const float hit = a.hit[t], w = a.weight ? a.weight[t] : 1.0f;
    float top = -INFINITY, sum = 0.0f;
    for (int g = tid; g < groups; g += 256) {
        const float2 x = a.part[(int64_t)g * a.T + t];
        s_factor[g] = x.x;
        join_pair(top, sum, x.x, x.y);
    }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
        const float o = __shfl_xor(top, d, 64), p = __shfl_xor(sum, d, 64);
        join_pair(top, sum, o, p);
    }
    if ((tid & 63) == 0) { s_top[tid >> 6] = top; s_sum[tid >> 6] = sum; }
    __syncthreads();
    top = s_top[0]; sum = s_sum[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) join_pair(top, sum, s_top[i], s_sum[i]);
    const float ref = top == -INFINITY ? 0.0f : top;
    for (int g = tid; g < groups; g += 256) s_factor[g] = __expf(s_factor[g] - ref);
    __syncthreads();
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    auto add = [&](float f, const float4 &x) {
        s.x = __builtin_fmaf(f, x.x, s.x); s.y = __builtin_fmaf(f, x.y, s.y); s.z = __builtin_fmaf(f, x.z, s.z); s.w = __builtin_fmaf(f, x.w, s.w);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (sub + 64 * i < groups) add(s_factor[sub + 64 * i], ahead[i]);
#pragma unroll 4
    for (int g = sub + 64 * AHEAD; g < groups; g += 64) add(s_factor[g], plane(g));
#pragma unroll
    for (int d = 4; d < 64; d *= 2) {
        s.x += __shfl_xor(s.x, d, 64); s.y += __shfl_xor(s.y, d, 64); s.z += __shfl_xor(s.z, d, 64); s.w += __shfl_xor(s.w, d, 64);
    }
    if ((tid & 63) < 4) s_acc[(tid >> 6) * 4 + (tid & 3)] = s;
    __syncthreads();
    if (tid >= 4) return;
#pragma unroll
    for (int g = 1; g < 4; ++g) {
        const float4 x = s_acc[g * 4 + tid];
        s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
    }
    const TokenResult it = token_result(top, sum, hit, w);
    if (tid == 0 && blockIdx.y == 0) {
        a.nll[t] = it.nll;
        if (a.lse) a.lse[t] = it.lse;
    }
    if (!on) return;
    const float f[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int u = 0; u < 4; ++u)
        out[u] = __builtin_bit_cast(uint16_t, (__bf16)__builtin_fmaf(it.pull, low_half(of_target[u]), it.scale * f[u]));
}

static int64_t single_dp(int32_t D) { return ((int64_t)D + 7) / 8 * 8; }
static int single_units(int32_t D) { return D <= 2048 ? 1 : D <= 4096 ? 2 : 4; }
static int single_waves(int32_t D) { return D <= 512 ? 1 : D <= 1024 ? 2 : 4; }
static int single_groups(int32_t D) {          // two wavefronts a SIMD
    const int g = 8 * compute_units() / single_waves(D);
    return g < kSingleGroups ? g : kSingleGroups;
}

// Registers: tokens and sums of 16 KU T floats next to 64 of the rows.  Three and four tokens gain where a thread's columns are sixteen, the
// vector work then hides behind memory (4 x 4096 x 131072 415 -> 309 us, 4 x 1024 x 50257 54 -> 77), and where launches count.  The loss alone
// is one read of W for the tile kernels too: one token 1 x 4096 x 32000 58 -> 46 us, with cold caches 123 -> 99; two tokens 2 x 2496 x 25064 30 -> 35, 66 -> 63.
bool single_serves(int64_t T, int32_t D, int32_t V, bool want_dH) {
    if (T < 1 || T > 4 || D > 8192 || T * single_units(D) > 8) return false;
    return T == 1 || (want_dH && (T == 2 || (D > 2048 && D <= 4096))) || (int64_t)V * D <= (4 << 20);
}
static int single_share(int32_t D, int32_t V) {            // rows of W of a workgroup: a batch at least
    const int groups = single_groups(D), share = (V + groups - 1) / groups, batch = 8 / single_units(D);
    return share < batch ? batch : share;
}
static int single_used(int32_t D, int32_t V) { return (V + single_share(D, V) - 1) / single_share(D, V); }       // workgroups that have rows
static size_t single_parts(int64_t T, int32_t D, int32_t V) { return ((size_t)single_used(D, V) * T * 8 + 255) & ~(size_t)255; }
size_t single_workspace(int64_t T, int32_t D, int32_t V, bool want_dH) {
    if (!single_serves(T, D, V, want_dH)) return 0;
    return 256 + single_parts(T, D, V) + (want_dH ? (size_t)single_used(D, V) * T * single_dp(D) * 4 : 0);
}

template <int TT, int KU, int NW>
static void launch_single_as(const SingleArgs &a, int groups, hipStream_t st) {
    if (a.dH) hipLaunchKernelGGL((loss_single_kernel<TT, KU, NW, true>), dim3((unsigned)groups), dim3(64 * NW), 0, st, a);
    else hipLaunchKernelGGL((loss_single_kernel<TT, KU, NW, false>), dim3((unsigned)groups), dim3(64 * NW), 0, st, a);
    hipLaunchKernelGGL(loss_single_join_kernel, dim3((unsigned)a.T, a.dH ? (unsigned)((a.D + 15) / 16) : 1), dim3(256), 0, st, a, groups);
}

qless_status launch_single(const uint16_t *H, int64_t ldH, const uint16_t *W, int64_t ldW, int T, int32_t D, int32_t V, const int64_t *target,
                           const float *weight, float *nll, float *lse, uint16_t *dH, int64_t ldDH, void *ws, hipStream_t st) {
    const int used = single_used(D, V), units = single_units(D);
    unsigned char *base = (unsigned char *)ws;
    SingleArgs a{H, ldH, W, ldW, target, weight, T, D, V, single_share(D, V), (float *)base, (float2 *)(base + 256),
                 (float *)(base + 256 + single_parts(T, D, V)), single_dp(D), nll, lse, dH, ldDH};
    auto by_tokens = [&](auto ku, auto waves) {
        constexpr int KU = decltype(ku)::value, NW = decltype(waves)::value;
        if (T == 1) launch_single_as<1, KU, NW>(a, used, st);
        else if (T == 2) launch_single_as<2, KU, NW>(a, used, st);
        else if constexpr (KU <= 2) launch_single_as<4, KU, NW>(a, used, st);
    };
    using std::integral_constant;
    switch (units * 4 + single_waves(D)) {
        case 5: by_tokens(integral_constant<int, 1>(), integral_constant<int, 1>()); break;
        case 6: by_tokens(integral_constant<int, 1>(), integral_constant<int, 2>()); break;
        case 8: by_tokens(integral_constant<int, 1>(), integral_constant<int, 4>()); break;
        case 12: by_tokens(integral_constant<int, 2>(), integral_constant<int, 4>()); break;
        default: by_tokens(integral_constant<int, 4>(), integral_constant<int, 4>()); break;
    }
    return launch_status();
}

}  // namespace qless
