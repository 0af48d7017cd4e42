// qless_token_loss: softmax cross entropy of tokens over a vocabulary, from the last hidden states H and the head's weights W, with
// its gradients, a piece of the T x V logits at a time.
//   z = H W^T,  lse_t = log sum_v exp z_tv,  nll_t = lse_t - z_t,target,  delta_tv = w_t (exp(z_tv - lse_t) - [v = target_t]),
//   dH = delta W,  dW = delta^T H.
// Tokens without a target in the vocabulary are left out: the others' rows of H are gathered first (bounded by T on the host, counted
// on the device), and the products are of these.  (How dH's is cut is planned from T: see LossPlan::splits.)
//
// Loss alone: the tiles of logits end with the maximum and the sum of their exponentials, which are joined.
// dH: a piece of the vocabulary at a time, one pass over it, as with the running softmax of an attention: planes = planes 2^(R_before - R) +
// p W, dH = w / s planes + w (p_target - 1) W_target at the end.  The tiles end with p = 2^(z log2 e - r), r the whole number above their
// own maximum, as bfloat16, with the sum of the others' p in fp32; a small kernel finds R, the greatest r of a token so far; and
// the product with W takes 2^(r - R) off the exponents of its operand, exactly.  So fp32 logits pass through memory only where D is cut in parts, and p is
// rounded once.  (With fp32 logits in memory and a kernel that turned them into p, 4096 x 4096 x 131072 took 7.9 ms.)
// dW needs the sums first, and its operand's factors are not of its entries but of its tokens.  Where the whole vocabulary is one piece,
// its logits are kept until delta is formed from them; else a second pass forms them again.
//
// The target's entry, the largest of a row, never passes through the bfloat16 operand, and its exponential enters no sum: it is added in fp32, to dH in the last kernel,
// to dW behind the product, from the tokens ordered by target.  (Rounded with the rest it made gradients of few tokens up to 0.4 %
// wrong.)  Up to 32 tokens, where the products wait for W anyway, the rest goes in as the sum of two bfloat16 numbers.
#include "product.h"
#include "score.h"
#include "token_loss.h"
#include <cmath>
#include <type_traits>

namespace qless {

struct LossTokens {                        // workspace views, by live token (padded to whole tiles)
    uint16_t *H;                           // [Tp][Dp] bfloat16: gathered rows, zeros behind them
    int32_t *count;                        // live tokens
    int32_t *token, *target;               // [Tp]
    int32_t *place;                        // [T]: live index of a token, or -1
    float *weight, *lse, *hit;             // [Tp]; hit: the target's logit
    float *top, *sum, *shrink;             // [Tp] R, sum of the others' 2^(z log2 e - R), 2^ the last change of R (few tokens: of exp and m)
    float *pull;                           // [Tp] w (p_target - 1)
    float2 *part;                          // [parts][Tp] maximum, sum of the others' exp(z - maximum); or r, sum of the others' p
    uint32_t *shift;                       // [parts][Tp] R - r, for two exponents
    int32_t *order, *order_target, *start; // [Tp] live tokens by target, and their targets; [Vp / 64 + 1]: where each 64 entries begin there
    float *logits;                         // [Tp][piece]
    uint16_t *delta;                       // [Tp][piece]
    uint16_t *pack;                        // [piece][Dp] where W cannot be read as it lies
    float *planes;                         // [splits][Tp][Dp] partial dH
    float *raw;                            // [raw][Tp][Vp] partial logits of small vocabularies
};
struct LossPlan {
    int64_t T, Tp, Dp, Vp, piece, parts;
    int32_t D, V, tile_n, tile_m, per_part, splits, raw;   // splits: of dH's product, as fill the chip if all tokens are live (8192 x 4096 x 32000, 90 % masked: 980 us, not 380)
    bool one_pass;                         // dW without a second pass
    size_t off[20], total;
};

constexpr int kGather = 1024;              // entries of a part where partial logits are added
constexpr int kFew = 32;                   // tokens up to which the rest of delta is two terms: rows t and t + kFew of delta and H

constexpr int64_t kMostEntries = 1 << 22;  // of a piece: 32-bit offsets into a tile's rows of delta
constexpr int64_t kMostTokens = (1 << 24) - 256;           // 256 threads for each of them, up to whole tiles
constexpr int64_t kMostTiles = (1 << 23) - 8;              // of 512 threads
constexpr int kLossThreads = 1024;

// A row of D numbers, or none, and zeros up to ld (a multiple of 64), eight elements a thread.
__device__ inline void copy_row(const uint16_t *x, bool there, int32_t D, uint16_t *out, int64_t ld) {
    for (int64_t c = threadIdx.x * 8; c < ld; c += 256 * 8) {
        uint16_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0;
        if (there && c + 8 <= D) __builtin_memcpy(v, x + c, 16);
        else if (there)
#pragma unroll
            for (int i = 0; i < 8; ++i) if (c + i < D) v[i] = x[c + i];
        __builtin_memcpy(__builtin_assume_aligned(out + c, 16), v, 16);
    }
}

// The live tokens numbered in their order: a workgroup a thousand tokens, whose place follows from a count of the targets before them.
__global__ void __launch_bounds__(kLossThreads)
loss_live_kernel(const int64_t *target, const float *weight, int64_t T, int32_t V, LossTokens w, float *nll, float *lse) {
    __shared__ int32_t s_before[kLossThreads / 64], s_wave[kLossThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t t0 = (int64_t)blockIdx.x * kLossThreads, t = t0 + tid;
    int32_t earlier = 0;
    for (int64_t i = tid; i < t0; i += kLossThreads) {
        const int64_t y = target[i];
        earlier += y >= 0 && y < V;
    }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) earlier += __shfl_xor(earlier, d, 64);
    const int64_t y = t < T ? target[t] : -1;
    const bool live = y >= 0 && y < V;
    const uint64_t votes = __ballot(live);
    if (lane == 0) { s_before[wave] = earlier; s_wave[wave] = __popcll(votes); }
    __syncthreads();
    int32_t at = __popcll(votes & (((uint64_t)1 << lane) - 1)), all = 0;
#pragma unroll
    for (int i = 0; i < kLossThreads / 64; ++i) {
        at += s_before[i] + (i < wave ? s_wave[i] : 0);
        all += s_before[i] + s_wave[i];
    }
    if (t < T) {
        w.place[t] = live ? at : -1;
        if (live) {
            w.token[at] = (int32_t)t;
            w.target[at] = (int32_t)y;
            w.weight[at] = weight ? weight[t] : 1.0f;
        } else {
            nll[t] = 0.0f;
            if (lse) lse[t] = 0.0f;
        }
    }
    if (tid == 0 && t0 + kLossThreads >= T) *w.count = all;
}

// The same for at most 64 tokens, together with the rows of H: a workgroup a row of the gathered ones.
__global__ void __launch_bounds__(256)
loss_start_kernel(const int64_t *target, const float *weight, int T, int32_t V, LossTokens w, float *nll, float *lse,
                  const uint16_t *H, int64_t ldH, int32_t D, int64_t Dp, int few) {
    const int lane = threadIdx.x & 63, r = blockIdx.x, of = few && r >= kFew ? r - kFew : r;
    const int64_t y = lane < T ? target[lane] : -1;
    const bool live = y >= 0 && y < V;
    const uint64_t votes = __ballot(live);
    const int at = __popcll(votes & (((uint64_t)1 << lane) - 1)), count = __popcll(votes);
    if (r == 0 && threadIdx.x < 64) {
        if (lane < T) {
            w.place[lane] = live ? at : -1;
            if (live) {
                w.token[at] = lane;
                w.target[at] = (int32_t)y;
                w.weight[at] = weight ? weight[lane] : 1.0f;
            } else {
                nll[lane] = 0.0f;
                if (lse) lse[lane] = 0.0f;
            }
        }
        if (lane == 0) *w.count = count;
    }
    const int from = of < count ? __ffsll((unsigned long long)__ballot(live && at == of)) - 1 : 0;
    copy_row(H + from * ldH, of < count, D, w.H + r * Dp, Dp);
}

// The same for at most 1024 tokens: four in a thread, every workgroup counts them all (65 x 512 x 2000 with dH: 38.1 -> 36.9 us; 512 x 2048 x 151936 661 -> 656).
__global__ void __launch_bounds__(256)
loss_start_many_kernel(const int64_t *target, const float *weight, int T, int32_t V, LossTokens w, float *nll, float *lse,
                       const uint16_t *H, int64_t ldH, int32_t D, int64_t Dp) {
    __shared__ int s_wave[4], s_from;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = blockIdx.x;
    int64_t y[4];
    int mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[i] = 4 * tid + i < T ? target[4 * tid + i] : -1;
        if (y[i] >= V) y[i] = -1;
        mine += y[i] >= 0;
    }
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(upto, d, 64);
        if (lane >= d) upto += o;
    }
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    int at = upto - mine, count = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        at += i < wave ? s_wave[i] : 0;
        count += s_wave[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = 4 * tid + i;
        if (t >= T) continue;
        if (y[i] >= 0 && at == r) s_from = t;
        if (r == 0) {
            w.place[t] = y[i] >= 0 ? at : -1;
            if (y[i] >= 0) {
                w.token[at] = t;
                w.target[at] = (int32_t)y[i];
                w.weight[at] = weight ? weight[t] : 1.0f;
            } else {
                nll[t] = 0.0f;
                if (lse) lse[t] = 0.0f;
            }
        }
        at += y[i] >= 0;
    }
    if (r == 0 && tid == 0) *w.count = count;
    if (r >= (count + 255) / 256 * 256) return;            // the whole workgroup
    __syncthreads();
    copy_row(H + (int64_t)(r < count ? s_from : 0) * ldH, r < count, D, w.H + r * Dp, Dp);
}

// Rows of bfloat16 copied to rows of ld with zeros behind their D elements; `from` null: row r,
// else the row that it names, and zeros from *count up to whole tiles.
__global__ void __launch_bounds__(256)
loss_rows_kernel(const uint16_t *X, int64_t ldX, int32_t D, const int32_t *from, const int32_t *count, int64_t rows, uint16_t *out, int64_t ld) {
    const int64_t r = blockIdx.x;
    const int64_t n = count ? *count : rows;
    if (r >= (n + 255) / 256 * 256) return;
    copy_row(X + (r < n ? (from ? (int64_t)from[r] : r) * ldX : 0), r < n, D, out + r * ld, ld);
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- what the tiles of logits end with: rows m are vocabulary entries, columns n tokens
// The maximum, the sum of the exponentials without the target's, and the target's logit.  STORE: the logits too, for a delta kernel, -infinity the target's
template <bool STORE> struct LossStats {
    struct Args { const int32_t *target; float *hit; float2 *part; int64_t Tp, first; int32_t V; float *logits; int64_t ld; };
    template <int FM, int FN>
    static __device__ inline void run(const Args &a, unsigned char *lds, f32x16 (&acc)[FM][FN], int64_t m, int64_t n, int, int64_t live) {
        const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
        const int64_t part = ((STORE ? 0 : a.first) + m) / (32 * FM);
        const int v0 = (int)(a.first + m) + 4 * half, over = a.V - v0;         // entries from here on
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int64_t t = n + 32 * j + l32;
            const int y = t < live ? a.target[t] - v0 : -1;
            const bool here = y >= 0 && y < 32 * FM && (y & 4) == 0;
            if (over < 32 * FM) {                           // the end of the vocabulary
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[i][j][v] = 32 * i + 8 * (v >> 2) + (v & 3) < over ? acc[i][j][v] : -INFINITY;
            }
            float top = acc[0][j][0];
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) top = fmaxf(top, acc[i][j][v]);
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float ref = (top == -INFINITY ? 0.0f : top) * kLog2e;
            if (__any(here)) {
                float hit = 0.0f;
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const bool it = y == 32 * i + 8 * (v >> 2) + (v & 3);
                        hit = it ? acc[i][j][v] : hit;
                        acc[i][j][v] = it ? -INFINITY : acc[i][j][v];
                    }
                if (here) a.hit[t] = hit;
            }
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) sum += exp2_of(__builtin_fmaf(acc[i][j][v], kLog2e, -ref));
            sum += __shfl_xor(sum, 32, 64);
            if (half == 0 && t < live) a.part[part * a.Tp + t] = make_float2(top, sum);
        }
        if (STORE)
            by_rows<FM, FN>(lds, acc, [&](int r, int c, f32x4 x) {
                if (n + r < live) *(f32x4 *)(a.logits + (n + r) * a.ld + m + c) = x;
            });
    }
};

// p = 2^(z log2 e - r) of a piece, without the targets' entries, as bfloat16, r and the sums
struct LossPower {
    struct Args { const int32_t *target; float *hit; float2 *part; int64_t Tp, first; int32_t V; uint16_t *out; int64_t ld; };
    template <int FM, int FN>
    static __device__ inline void run(const Args &a, unsigned char *lds, f32x16 (&acc)[FM][FN], int64_t m, int64_t n, int, int64_t live) {
        const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
        const int v0 = (int)(a.first + m) + 4 * half, over = a.V - v0;         // entries from here on
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int64_t t = n + 32 * j + l32;
            const int y = t < live ? a.target[t] - v0 : -1;
            const bool here = y >= 0 && y < 32 * FM && (y & 4) == 0;
            if (over < 32 * FM) {                           // the end of the vocabulary
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[i][j][v] = 32 * i + 8 * (v >> 2) + (v & 3) < over ? acc[i][j][v] : -INFINITY;
            }
            float top = acc[0][j][0];
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) top = fmaxf(top, acc[i][j][v]);
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float r = top == -INFINITY ? 0.0f : ceilf(top * kLog2e);
            if (__any(here)) {
                float hit = 0.0f;
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const bool it = y == 32 * i + 8 * (v >> 2) + (v & 3);
                        hit = it ? acc[i][j][v] : hit;
                        acc[i][j][v] = it ? -INFINITY : acc[i][j][v];
                    }
                if (here) a.hit[t] = hit;
            }
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    acc[i][j][v] = exp2_of(__builtin_fmaf(acc[i][j][v], kLog2e, -r));
                    sum += acc[i][j][v];
                }
            sum += __shfl_xor(sum, 32, 64);
            if (half == 0 && t < live) a.part[m / (32 * FM) * a.Tp + t] = make_float2(top == -INFINITY ? -INFINITY : r, sum);
        }
        by_rows<FM, FN>(lds, acc, [&](int row, int c, f32x4 x) {
            uint16_t d[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) d[u] = __builtin_bit_cast(uint16_t, (__bf16)x[u]);
            if (n + row < live) __builtin_memcpy(__builtin_assume_aligned(a.out + (n + row) * a.ld + m + c, 8), d, 8);
        });
    }
};

// the second pass of dW: delta without the targets' entries, of a piece
template <bool FEW> struct LossDelta {
    struct Args { const int32_t *target; const float *lse, *weight; uint16_t *delta; int64_t ld, first; int32_t V; };
    template <int FM, int FN>
    static __device__ inline void run(const Args &a, unsigned char *lds, f32x16 (&acc)[FM][FN], int64_t m, int64_t n, int, int64_t live) {
        by_rows<FM, FN>(lds, acc, [&](int r, int c, f32x4 z) {
            const int64_t t = n + r;
            const bool on = t < live;
            const float lse = on ? a.lse[t] : 0.0f, w = on ? a.weight[t] : 0.0f;
            const int c0 = (int)m + c, y = on ? a.target[t] - (int)a.first - c0 : -1, over = on ? a.V - (int)a.first - c0 : 0;
            uint16_t d[4], rest[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float x = u < over && u != y ? w * __expf(z[u] - lse) : 0.0f;
                d[u] = __builtin_bit_cast(uint16_t, (__bf16)x);
                rest[u] = __builtin_bit_cast(uint16_t, (__bf16)(x - __uint_as_float((uint32_t)d[u] << 16)));
            }
            uint16_t *out = a.delta + t * a.ld + c0;
            __builtin_memcpy(__builtin_assume_aligned(out, 8), d, 8);
            if (FEW) __builtin_memcpy(__builtin_assume_aligned(out + kFew * a.ld, 8), rest, 8);
        });
    }
};

// rows m are columns of dH, columns n tokens; pieces after the first add to what is there, shrunk.  FEW: columns kFew on are the second
// terms of the first ones.
template <bool FEW> struct LossPlane {
    struct Args { float *planes; int64_t Tp, Dp; const float *shrink; };
    template <int FM, int FN>
    static __device__ inline void run(const Args &a, unsigned char *lds, f32x16 (&acc)[FM][FN], int64_t m, int64_t n, int split, int64_t live) {
        static_assert(!FEW || FN * 32 == 2 * kFew, "both terms in one wavefront");
        if (FEW)
#pragma unroll
            for (int i = 0; i < FM; ++i) acc[i][0] += acc[i][FN - 1];
        auto store = [&](int r, int c, f32x4 x) {
            const int64_t t = n + r;
            if (t >= live || m + c >= a.Dp) return;
            float *out = a.planes + (split * a.Tp + t) * a.Dp + m + c;
            if (a.shrink) x += *(const f32x4 *)out * a.shrink[t];
            *(f32x4 *)out = x;
        };
        if (FEW) {
            f32x16 first[FM][1];
#pragma unroll
            for (int i = 0; i < FM; ++i) first[i][0] = acc[i][0];
            by_rows<FM, 1>(lds, first, store);
        } else {
            by_rows<FM, FN>(lds, acc, store);
        }
    }
};

// rows m are columns of dW, columns n vocabulary entries; the targets' entries of delta are added here in fp32, one token after the other (1 us each where a
// wavefront's 64 entries are the targets of thousands)
struct LossHead {
    struct Args {
        uint16_t *dW; int64_t ld, first; int32_t V, D;
        const int32_t *order, *order_target, *start; const float *pull; const uint16_t *H; int64_t Dp;
    };
    template <int FM, int FN>
    static __device__ inline void run(const Args &a, unsigned char *lds, f32x16 (&acc)[FM][FN], int64_t m, int64_t n, int, int64_t) {
        static_assert(FN == 2, "64 entries a wavefront");
        const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
        const int block = __builtin_amdgcn_readfirstlane((int)((a.first + n) / 64));
        const int lo = a.start[block], hi = a.start[block + 1];
        for (int x0 = lo; x0 < hi; x0 += 64) {             // in the order of target and token; 64 of them in the lanes
            const bool on = x0 + lane < hi;
            const int rows = on ? a.order[x0 + lane] : 0, cols = on ? a.order_target[x0 + lane] & 63 : 0;
            const float pulls = on ? a.pull[rows] : 0.0f;
            for (int x = 0; x < 64 && x0 + x < hi; ++x) {
                const int r = __builtin_amdgcn_readlane(rows, x), col = __builtin_amdgcn_readlane(cols, x);
                const float pull = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(pulls), x)), f = l32 == (col & 31) ? pull : 0.0f;
                const uint16_t *h = a.H + r * a.Dp + m + 4 * half;
                auto add = [&](int j) {
#pragma unroll
                    for (int i = 0; i < FM; ++i)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            uint16_t y[4] = {0, 0, 0, 0};
                            if (m + 32 * i + 8 * q + 4 * half < a.Dp) __builtin_memcpy(y, __builtin_assume_aligned(h + 32 * i + 8 * q, 8), 8);
#pragma unroll
                            for (int u = 0; u < 4; ++u) acc[i][j][4 * q + u] = __builtin_fmaf(f, __uint_as_float((uint32_t)y[u] << 16), acc[i][j][4 * q + u]);
                        }
                };
                if (col < 32) add(0); else add(1);
            }
        }
        by_rows<FM, FN>(lds, acc, [&](int r, int c, f32x4 y) {
            const int64_t v = a.first + n + r, d = m + c;
            if (v >= a.V) return;
            uint16_t x[4], *out = a.dW + v * a.ld + d;
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = __builtin_bit_cast(uint16_t, (__bf16)y[u]);
            if (d + 4 <= a.D) __builtin_memcpy(out, x, 8);
            else
#pragma unroll
                for (int u = 0; u < 4; ++u) if (d + u < a.D) out[u] = x[u];
        });
    }
};

// lse and nll of TOK tokens from their parts, 256 / TOK threads each.
template <int TOK>
__global__ void __launch_bounds__(256)
loss_join_kernel(LossTokens w, int64_t Tp, int64_t parts, float *nll, float *lse) {
    constexpr int LANES = 256 / TOK;
    __shared__ float s_top[256], s_sum[256];
    const int tok = threadIdx.x % TOK, part = threadIdx.x / TOK;
    const int64_t t = (int64_t)blockIdx.x * TOK + tok;
    const int64_t live = *w.count;
    if ((int64_t)blockIdx.x * TOK >= live) return;          // the whole workgroup
    float top = -INFINITY, sum = 0.0f;
    for (int64_t p = part; p < parts && t < live; p += LANES) {
        const float2 x = w.part[p * Tp + t];
        join_pair(top, sum, x.x, x.y);
    }
    s_top[threadIdx.x] = top; s_sum[threadIdx.x] = sum;
    __syncthreads();
    for (int h = LANES / 2; h > 0; h /= 2) {
        if (part < h) {
            const int o = threadIdx.x + h * TOK;
            join_pair(s_top[threadIdx.x], s_sum[threadIdx.x], s_top[o], s_sum[o]);
        }
        __syncthreads();
    }
    if (part == 0 && t < live) {
        const TokenResult it = token_result(s_top[tok], s_sum[tok], w.hit[t], w.weight[t]);
        const int64_t at = w.token[t];
        w.lse[t] = it.lse;
        w.pull[t] = it.pull;
        nll[at] = it.nll;
        if (lse) lse[at] = it.lse;
    }
}

// A token's logits of a piece become an operand of the products; the target's is -infinity there.  Grid (tokens, shares of the row).
//   RUN      p = exp(z - m), m the maximum so far; top, sum, shrink go on (one share)
//   else     delta = w exp(z - lse), with its loss (the piece is the vocabulary; the parts hold sums)
//   FEW      in two terms, rows t and t + kFew
// Rows behind the live tokens, up to a whole stage, are zeros.
template <bool RUN, bool FEW>
__global__ void __launch_bounds__(256)
loss_delta_kernel(LossTokens w, int64_t Tp, int64_t parts, int64_t first, int64_t width, int64_t ld, float *nll, float *lse) {
    __shared__ float s_top[4], s_sum[4];
    const int64_t t = blockIdx.x, live = *w.count;
    if (t >= (FEW ? kFew : (live + 63) / 64 * 64)) return;
    const int tid = threadIdx.x;
    const int64_t share = (width / 4 + gridDim.y - 1) / gridDim.y * 4, c0 = share * blockIdx.y, c1 = c0 + share < width ? c0 + share : width;
    uint16_t *out = w.delta + t * ld;
    auto put = [&](int64_t c, const float (&x)[4]) {
        uint16_t d[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) d[u] = __builtin_bit_cast(uint16_t, (__bf16)x[u]);
        __builtin_memcpy(__builtin_assume_aligned(out + c, 8), d, 8);
        if (FEW) {
#pragma unroll
            for (int u = 0; u < 4; ++u) d[u] = __builtin_bit_cast(uint16_t, (__bf16)(x[u] - __uint_as_float((uint32_t)d[u] << 16)));
            __builtin_memcpy(__builtin_assume_aligned(out + kFew * ld + c, 8), d, 8);
        }
    };
    if (t >= live) {
        const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int64_t c = c0 + 4 * tid; c < c1; c += 1024) put(c, zero);
        return;
    }
    const float *z = w.logits + t * ld;
    if (RUN) {
        const float before = first ? w.top[t] : -INFINITY, sum_before = first ? w.sum[t] : 0.0f;
        float top = before;
        for (int64_t p = tid; p < parts; p += 256) top = fmaxf(top, w.part[p * Tp + t].x);
#pragma unroll
        for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
        if ((tid & 63) == 0) s_top[tid >> 6] = top;
        __syncthreads();
        top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
        const float ref = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
        for (int64_t c = 4 * tid; c < width; c += 1024) {
            const float4 v = *(const float4 *)(z + c);
            const float f[4] = {v.x, v.y, v.z, v.w};
            float x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                x[u] = __expf(f[u] - ref);
                sum += x[u];
            }
            put(c, x);
        }
#pragma unroll
        for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d, 64);
        if ((tid & 63) == 0) s_sum[tid >> 6] = sum;
        __syncthreads();
        if (tid == 0) {
            const float shrink = before == -INFINITY ? 0.0f : __expf(before - ref);
            w.top[t] = top;
            w.sum[t] = sum_before * shrink + ((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]));
            w.shrink[t] = shrink;
        }
        return;
    }
    float top = -INFINITY, sum = 0.0f;
    for (int64_t p = tid; p < parts; p += 256) {
        const float2 x = w.part[p * Tp + t];
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
    const TokenResult it = token_result(top, sum, w.hit[t], w.weight[t]);
    if (tid == 0 && blockIdx.y == 0) {
        const int64_t at = w.token[t];
        w.pull[t] = it.pull;
        nll[at] = it.nll;
        if (lse) lse[at] = it.lse;
    }
    for (int64_t c = c0 + 4 * tid; c < c1; c += 1024) {
        const float4 v = *(const float4 *)(z + c);
        const float f[4] = {v.x, v.y, v.z, v.w};
        float x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = it.scale * __expf(f[u] - top);
        put(c, x);
    }
}

// Partial logits added, with what the tiles' epilogue leaves of whole ones: a workgroup kGather entries of a token.
enum { SUMS = 0, LOGITS = 1, POWERS = 2 };
template <int WHAT>
__global__ void __launch_bounds__(256)
loss_gather_kernel(LossTokens w, int64_t Tp, int64_t Vp, int raw, int32_t V) {
    __shared__ float s_top[4], s_sum[4];
    const int64_t t = blockIdx.x;
    if (t >= *w.count) return;
    const int c = (int)blockIdx.y * kGather + 4 * (int)threadIdx.x, y = w.target[t] - c;
    f32x4 z = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (c < Vp) {
        z = *(const f32x4 *)(w.raw + t * Vp + c);
#pragma unroll 4
        for (int s = 1; s < raw; ++s) z += *(const f32x4 *)(w.raw + (s * Tp + t) * Vp + c);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (c + u >= V) z[u] = -INFINITY;
    }
    float top = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (u == y) {
            w.hit[t] = z[u];
            z[u] = -INFINITY;
        }
    if (WHAT == LOGITS && c < Vp) *(f32x4 *)(w.logits + t * Vp + c) = z;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
    if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    float ref = top == -INFINITY ? 0.0f : top, p[4];
    if (WHAT == POWERS) ref = ceilf(ref * kLog2e);
#pragma unroll
    for (int u = 0; u < 4; ++u) p[u] = WHAT == POWERS ? exp2_of(__builtin_fmaf(z[u], kLog2e, -ref)) : __expf(z[u] - ref);
    if (WHAT == POWERS && c < Vp) {
        uint16_t d[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) d[u] = __builtin_bit_cast(uint16_t, (__bf16)p[u]);
        __builtin_memcpy(__builtin_assume_aligned(w.delta + t * Vp + c, 8), d, 8);
    }
    float sum = (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
    for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d, 64);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) w.part[(int64_t)blockIdx.y * Tp + t] = make_float2(WHAT == POWERS && top != -INFINITY ? ref : top, (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]));
}

// R of a piece: TOK tokens a workgroup.  Where the maximum is not a number's, the sum is not one either.
template <int TOK>
__global__ void __launch_bounds__(1024)
loss_shift_kernel(LossTokens w, int64_t Tp, int64_t parts, int first) {
    constexpr int LANES = 1024 / TOK, WAVES = 16;           // a wavefront's 64 / TOK threads of a token are joined in registers
    __shared__ float s_top[WAVES][TOK], s_sum[WAVES][TOK];
    const int64_t live = *w.count, t = (int64_t)blockIdx.x * TOK + threadIdx.x % TOK;
    if ((int64_t)blockIdx.x * TOK >= live) return;          // the whole workgroup
    const int lane = threadIdx.x / TOK, tok = threadIdx.x % TOK, wave = threadIdx.x >> 6;
    const int64_t mine = t < live ? parts : 0;
    const float before = t < live && !first ? w.top[t] : -INFINITY;
    float top = before;
#pragma unroll 4
    for (int64_t p = lane; p < mine; p += LANES) top = fmaxf(top, w.part[p * Tp + t].x);
#pragma unroll
    for (int d = TOK; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
    if ((threadIdx.x & 63) < TOK) s_top[wave][tok] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) top = fmaxf(top, s_top[i][tok]);
    float sum = 0.0f;
#pragma unroll 4
    for (int64_t p = lane; p < mine; p += LANES) {
        const float2 x = w.part[p * Tp + t];
        const float by = fminf(top - x.x, 255.0f);          // of a part without entries, or numbers: 255
        sum += x.y * exp2_of(x.x - top);
        w.shift[p * Tp + t] = (uint32_t)(int)by * 0x00800080u;
    }
#pragma unroll
    for (int d = TOK; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
    if ((threadIdx.x & 63) < TOK) s_sum[wave][tok] = sum;
    __syncthreads();
    if (lane == 0 && t < live) {
        for (int i = 1; i < WAVES; ++i) sum += s_sum[i][tok];
        const float shrink = before == -INFINITY ? 0.0f : exp2_of(before - top);
        w.top[t] = top;
        w.sum[t] = (first ? 0.0f : w.sum[t] * shrink) + sum;
        w.shrink[t] = shrink;
    }
}

// The live tokens in the order of target and token, and where each 64 vocabulary entries begin there: 16 threads count what comes before
// a token (or before 64 entries).  T (T + V / 64) comparisons, next to the 2 T D V operations of the products (2048 x 2048 x 50257: 10 of 1400 us; 2^16 tokens
// 1.1 ms, 2^19 59 ms).
__global__ void __launch_bounds__(256)
loss_order_kernel(LossTokens w, int64_t T, int64_t blocks64) {
    const int live = *w.count, sub = threadIdx.x & 15;
    const int64_t token_groups = (T + 15) / 16;
    const bool by_token = blockIdx.x < token_groups;
    const int64_t i = (by_token ? blockIdx.x : blockIdx.x - token_groups) * 16 + (threadIdx.x >> 4);
    if (by_token ? i >= live : i >= blocks64) return;      // whole rows of 16 lanes
    const int mine = by_token ? w.target[i] : (int)(i * 64);
    int before = 0;
#pragma unroll 8
    for (int j = sub; j < live; j += 16) {
        const int y = w.target[j];
        before += y < mine || (by_token && y == mine && j < i);
    }
#pragma unroll
    for (int d = 8; d > 0; d /= 2) before += __shfl_xor(before, d, 16);
    if (sub != 0) return;
    if (by_token) { w.order[before] = (int32_t)i; w.order_target[before] = mine; }
    else w.start[i] = before;
}

// dH of a token: the sum of its planes (times w / s where they run), and the target's part; or zeros.  SG threads share the planes
// of four columns, in a fixed order.
template <int SG>
__global__ void __launch_bounds__(256)
loss_hidden_kernel(LossTokens w, int64_t Tp, int64_t Dp, int32_t D, int splits, int run, const uint16_t *W, int64_t ldW,
                   uint16_t *dH, int64_t ld, float *nll, float *lse) {
    constexpr int COLS = 256 / SG;
    __shared__ float4 s_sum[SG > 1 ? 256 : 1];
    const int64_t t = blockIdx.x, r = w.place[t];
    const int col = threadIdx.x % COLS, sg = threadIdx.x / COLS;
    float scale = 1.0f, pull = 0.0f;
    const uint16_t *row = W;
    if (r >= 0) {
        row += w.target[r] * ldW;
        if (run) {
            float one, all;
            if (run == 2) {                                 // token_result with powers of two
                const float top = w.top[r], others = w.sum[r], at = __builtin_fmaf(w.hit[r], kLog2e, -top), mine = exp2_of(at), total = others + mine;
                one = others < mine ? log1pf(others / mine) : kLn2 * (log2f(total) - at);
                all = one + w.hit[r];
                scale = w.weight[r] / total;
                pull = -scale * others;
            } else {
                const TokenResult it = token_result(w.top[r], w.sum[r], w.hit[r], w.weight[r]);
                one = it.nll;
                all = it.lse;
                scale = it.scale;
                pull = it.pull;
            }
            if (threadIdx.x == 0 && blockIdx.y == 0) {
                nll[t] = one;
                if (lse) lse[t] = all;
                w.lse[r] = all;
                w.pull[r] = pull;
            }
        } else {
            pull = w.pull[r];
        }
    }
    for (int64_t c0 = (int64_t)blockIdx.y * COLS * 4; c0 < D; c0 += (int64_t)gridDim.y * COLS * 4) {     // the same for the workgroup
        const int64_t c = c0 + col * 4;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (r >= 0 && c < D) {
#pragma unroll 4
            for (int p = sg; p < splits; p += SG) {
                const float4 y = *(const float4 *)(w.planes + ((int64_t)p * Tp + r) * Dp + c);
                s.x += y.x; s.y += y.y; s.z += y.z; s.w += y.w;
            }
        }
        if (SG > 1) {
            s_sum[threadIdx.x] = s;
            __syncthreads();
            if (sg == 0)
#pragma unroll
                for (int g = 1; g < SG; ++g) {
                    const float4 y = s_sum[g * COLS + col];
                    s.x += y.x; s.y += y.y; s.z += y.z; s.w += y.w;
                }
            __syncthreads();
        }
        if (sg != 0 || c >= D) continue;
        uint16_t x[4] = {0, 0, 0, 0};
        if (r >= 0) {
            uint16_t v[4] = {0, 0, 0, 0};
            if (c + 4 <= D) __builtin_memcpy(v, row + c, 8);
            else
#pragma unroll
                for (int u = 0; u < 4; ++u) if (c + u < D) v[u] = row[c + u];
            const float f[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = __builtin_bit_cast(uint16_t, (__bf16)__builtin_fmaf(pull, __uint_as_float((uint32_t)v[u] << 16), scale * f[u]));
        }
        uint16_t *out = dH + t * ld + c;
        if (c + 4 <= D) __builtin_memcpy(out, x, 8);
        else
#pragma unroll
            for (int u = 0; u < 4; ++u) if (c + u < D) out[u] = x[u];
    }
}

typedef ProductShape<256, 256, 2, 4, 2> Loss256;
typedef ProductShape<128, 256, 2, 4, 3> LossHalf;
typedef ProductShape<256, 128, 4, 2, 3> Loss128;
typedef ProductShape<256, 64, 4, 2, 4> Loss64;
typedef ProductShape<256, 64, 4, 2, 3> LossShift;          // with room for shifts
typedef ProductShape<256, 64, 8, 1, 4> LossTerms;          // both terms of few tokens in a wavefront
typedef ProductShape<256, 32, 8, 1, 4> Loss32;
typedef ProductShape<128, 128, 2, 2, 2> LossSmall;         // dW where larger tiles do not fill the chip

static int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// Everything of a call that follows from its sizes.
static LossPlan loss_plan(int64_t T, int32_t D, int32_t V, bool want_dH, bool want_dW) {
    LossPlan p{};
    p.T = T; p.D = D; p.V = V;
    p.tile_n = T <= 32 ? 32 : T <= 64 ? 64 : T <= 128 ? 128 : 256;
    p.Tp = up_to(T > 0 ? T : 1, p.tile_n < 64 ? 64 : p.tile_n);
    p.Dp = up_to(D, 64);
    p.Vp = up_to(V, 256);
    const bool gradient = want_dH || want_dW;
    // A piece: p, or logits and delta, of up to 1.5 GB (they come from memory at any size that is worth its additions to the planes, and more
    // tiles fill their last round better).  With dW one piece saves the second pass.  Few tokens: one piece.
    const int64_t budget = (int64_t)1536 << 20, cus = compute_units();
    const int64_t ntiles = (T + p.tile_n - 1) / p.tile_n;
    // The tiles of logits where few fill the chip: rounds of tiles of 128 entries, at 0.64 of the larger ones' time each (256 x 4096 x 32000,
    // loss alone: 102 -> 79 us), or D in parts, whose partial logits another kernel adds in 8 us and their bytes' time (256 x 8192 x 4000: 157 -> 52 us).  A
    // stage of 64 columns takes 1.6 us in a tile of 256 tokens; with few tokens 0.5, and half of the chip reads W as fast as all
    // of it (1 x 4096 x 32000 in two parts 49 -> 53 us).
    const int64_t tiles_m = p.Vp / 256 * (ntiles > 0 ? ntiles : 1);
    const double rounds = (double)((tiles_m + cus - 1) / cus), half_rounds = 0.64 * (double)((2 * tiles_m + cus - 1) / cus);
    const bool halves = p.tile_n == 256 && half_rounds < rounds, narrow = p.tile_n <= 64;
    p.tile_m = halves ? 128 : 256;
    p.raw = 1;
    int64_t raw = cus / tiles_m > 0 ? cus / tiles_m : 1;
    if (raw > p.Dp / 64 / 4) raw = p.Dp / 64 / 4 > 0 ? p.Dp / 64 / 4 : 1;
    const double saved = (double)(p.Dp / 64) * (narrow ? 0.5 : p.tile_n == 128 ? 0.8 : 1.6) * ((halves ? 0.64 : 1.0) - 1.0 / (double)raw);
    if (raw >= (narrow ? 3 : 2) && saved > 8.0 + (double)T * (double)p.Vp * 8.0 * (double)raw / 5e6) {
        p.raw = (int32_t)raw;
        p.tile_m = 256;
    }
    p.one_pass = T <= kFew || (want_dW && p.Tp * p.Vp * 6 <= budget);
    const int64_t bytes = p.one_pass ? 6 : 2;               // of an entry of a piece
    int64_t piece = p.Vp;
    if (!p.one_pass && p.Tp * p.Vp * bytes > budget) {
        // whole rounds of tiles of the chip, if all tokens are live
        int64_t m = budget / (bytes * p.Tp) / 256;
        if (m < 8) m = 8;
        const int64_t rounds = m * ntiles / cus;
        if (rounds > 0) m = rounds * cus / ntiles > 0 ? rounds * cus / ntiles : 1;
        piece = m * 256;
        if (piece > p.Vp) piece = p.Vp;
    }
    if (piece > kMostEntries) piece = kMostEntries;
    p.piece = piece;
    // (raw: its parts are larger.)  Where dH runs along powers of two the parts are a piece's
    p.per_part = p.tile_m == 128 ? 64 : p.tile_n == 256 ? 128 : p.tile_n == 32 ? 32 : 64;
    p.parts = (want_dH && !p.one_pass ? piece : p.Vp) / p.per_part;
    const int64_t tiles = ((D + 255) / 256) * ntiles, stages = piece / 64;
    int64_t splits = tiles > 0 ? cus / tiles : 1;
    // a stage takes 1.3 us, a plane its bytes' time twice (512 x 512 x 2000: 45 us with eight stages a split at least, 42 with four; 1024 x 1024 x 5000: 61 and 68, so by both)
    const int64_t worth = (int64_t)sqrt((double)stages * 1.3 * 5e6 / (8.0 * (double)(T > 0 ? T : 1) * (double)p.Dp));
    if (splits > stages / 4) splits = stages / 4;
    if (splits > worth) splits = worth;
    if (splits < 1) splits = 1;
    p.splits = (int32_t)splits;
    size_t at = 0;
    int i = 0;
    auto take = [&](size_t bytes) { p.off[i++] = at; at = (at + bytes + 255) & ~(size_t)255; };
    take((size_t)p.Tp * p.Dp * 2);                          // 0 H
    take(256);                                              // 1 count
    for (int j = 0; j < 10; ++j) take((size_t)p.Tp * 4);    // 2 token, target, place, weight, lse, hit, top, sum, shrink, pull
    take((size_t)p.parts * p.Tp * 8);                       // 12 part
    take(want_dW ? (size_t)p.Tp * 8 : 0);                   // 13 order, order_target
    take(want_dW ? (size_t)(p.Vp / 64 + 1) * 4 : 0);        // 14 start
    // 15: a piece's logits and delta, or p; where W has to be packed, shorter pieces with the packed rows behind them: room for 64 MB of them all
    const size_t each = (size_t)p.Tp * (gradient ? bytes : 0) + (size_t)p.Dp * 2;
    size_t whole = gradient ? (size_t)p.Tp * piece * bytes : 0, packed = each * p.Vp;
    if (packed > ((size_t)64 << 20)) packed = (size_t)64 << 20;
    if (packed < each * 256) packed = each * 256;
    take(whole > packed ? whole : packed);
    take(want_dH ? (size_t)p.splits * p.Tp * p.Dp * 4 : 0); // 16 planes
    take(p.raw > 1 ? (size_t)p.raw * p.Tp * p.Vp * 4 : 0);  // 17 raw
    take(want_dH && T > kFew ? (size_t)(piece / p.per_part) * p.Tp * 4 : 0);      // 18 shift
    p.total = at;
    return p;
}

// FROM: the smallest tile that a call takes
template <class Epilogue, int AK, int BK, int FROM, bool SHIFT = false>
static qless_status loss_product(int tile_n, const ProductArgs &a, const typename Epilogue::Args &e, hipStream_t st) {
    switch (tile_n) {
        case 32:
            if constexpr (FROM == 32) return launch_product<Loss32, AK, BK, Epilogue>(a, e, st);
            return QLESS_ERR_UNSUPPORTED;
        case 64: return launch_product<std::conditional_t<SHIFT, LossShift, Loss64>, AK, BK, Epilogue, false, SHIFT>(a, e, st);
        case 128: return launch_product<Loss128, AK, BK, Epilogue, false, SHIFT>(a, e, st);
        default: return launch_product<Loss256, AK, BK, Epilogue, false, SHIFT>(a, e, st);
    }
}
// the tiles of logits of `entries` from the vocabulary
template <class Epilogue, int FROM>
static qless_status logits_product(const LossPlan &p, ProductArgs a, int64_t entries, const typename Epilogue::Args &e, hipStream_t st) {
    a.mtiles = (int32_t)((entries + p.tile_m - 1) / p.tile_m);
    if (p.tile_m == 128) return launch_product<LossHalf, ALONG, ALONG, Epilogue>(a, e, st);
    return loss_product<Epilogue, ALONG, ALONG, FROM>(p.tile_n, a, e, st);
}

// Sizes that the launches bear: a workgroup for a token, and tiles of dH for all of them at once.
static bool loss_sizes_ok(int64_t T, int32_t D, int32_t V) {
    return D <= 65536 && V <= 0x1FFFFFFF && T <= kMostTokens && (D + 255) / 256 * ((T + 255) / 256) <= kMostTiles;
}

}  // namespace qless

extern "C" size_t qless_token_loss_workspace(int64_t T, int32_t D, int32_t V, int want_dH, int want_dW) {
    using namespace qless;
    if (T < 0 || D < 1 || V < 1 || !loss_sizes_ok(T, D, V)) return 0;
    // (a workspace for more outputs serves fewer, which may keep the parts of a whole vocabulary where more pass a piece at a time)
    size_t most = single_workspace(T, D, V, want_dH != 0);
    for (int some = 0; some < 4; ++some) {
        if (((some & 1) && !want_dH) || ((some & 2) && !want_dW)) continue;
        const size_t total = loss_plan(T, D, V, (some & 1) != 0, (some & 2) != 0).total;
        if (total > most) most = total;
    }
    return most;
}

extern "C" qless_status qless_token_loss(const void *H, int64_t ldH, const void *W, int64_t ldW, qless_dtype dt, int64_t T, int32_t D, int32_t V,
                                         const int64_t *target, const float *weight, float *nll, float *lse, void *dH, int64_t ldDH,
                                         void *dW, int64_t ldDW, void *ws, size_t ws_bytes, void *stream) {
    using namespace qless;
    if (T < 0 || D < 1 || V < 1 || (T > 1 && (ldH < D || (dH && ldDH < D))) || (V > 1 && (ldW < D || (dW && ldDW < D)))) return QLESS_ERR_INVALID_ARG;
    if (dt != QLESS_BF16 || !loss_sizes_ok(T, D, V)) return QLESS_ERR_UNSUPPORTED;
    if (T == 0 && !dW) return QLESS_OK;
    if (!W || (T > 0 && (!H || !target || !nll))) return QLESS_ERR_INVALID_ARG;
    if (!ws || ws_bytes < qless_token_loss_workspace(T, D, V, dH != nullptr, dW != nullptr) || ((uintptr_t)ws & 15) != 0) return QLESS_ERR_WORKSPACE;
    const qless_status ready = device_ready();
    if (ready != QLESS_OK) return ready;
    const hipStream_t st = (hipStream_t)stream;
    // W is read where it lies if its rows are whole 16-byte chunks; else a piece at a time is packed into the workspace
    const bool packs = ((uintptr_t)W & 15) != 0 || (ldW % 8 != 0 && V > 1) || D % 8 != 0 || ldW * 2 >= ((int64_t)1 << 23);
    if (!dW && !packs && single_serves(T, D, V, dH != nullptr))
        return launch_single((const uint16_t *)H, ldH, (const uint16_t *)W, V > 1 ? ldW : D, (int)T, D, V, target, weight, nll, lse, (uint16_t *)dH, ldDH, ws, st);
    const LossPlan p = loss_plan(T, D, V, dH != nullptr, dW != nullptr);
    unsigned char *base = (unsigned char *)ws;
    auto ints = [&](int i) { return (int32_t *)(base + p.off[i]); };
    auto floats = [&](int i) { return (float *)(base + p.off[i]); };
    LossTokens w{};
    w.H = (uint16_t *)(base + p.off[0]); w.count = ints(1);
    w.token = ints(2); w.target = ints(3); w.place = ints(4);
    w.weight = floats(5); w.lse = floats(6); w.hit = floats(7); w.top = floats(8); w.sum = floats(9); w.shrink = floats(10); w.pull = floats(11);
    w.part = (float2 *)(base + p.off[12]); w.order = ints(13); w.order_target = w.order + p.Tp; w.start = ints(14);
    w.logits = floats(15); w.planes = floats(16); w.raw = floats(17); w.shift = (uint32_t *)ints(18);

    const bool gradient = dH || dW, few = T <= kFew;
    const int64_t bytes = p.one_pass ? 6 : 2;
    int64_t piece = p.piece;
    if (!gradient) {                                        // the vocabulary at once, but for more tiles than a launch takes
        const int64_t most = kMostTiles / ((T + p.tile_n - 1) / p.tile_n) * p.tile_m / 256 * 256;
        piece = p.Vp < most ? p.Vp : most;
    }
    if (packs) {
        const int64_t room = (int64_t)((p.off[16] - p.off[15]) / ((size_t)p.Tp * (gradient ? bytes : 0) + (size_t)p.Dp * 2)) / 256 * 256;
        if (piece > room) piece = room;
    }
    // Where dW was to need no second pass but W is packed, its pieces are the plan's pieces' part: dH runs along powers of two then too.
    const bool one_pass = gradient && p.one_pass && piece == p.Vp, power = dH && !few && !one_pass;
    w.delta = few || one_pass ? (uint16_t *)(w.logits + p.Tp * piece) : (uint16_t *)w.logits;
    w.pack = gradient ? (uint16_t *)((unsigned char *)w.logits + p.Tp * piece * bytes) : (uint16_t *)w.logits;
    auto rows_of = [&](int64_t v0) { return V - v0 < piece ? V - v0 : piece; };
    auto head = [&](int64_t v0) {                           // a piece of W by rows of D
        if (!packs) return ProductOperand{(const uint16_t *)W + v0 * ldW, V > 1 ? ldW * 2 : p.Dp * 2, rows_of(v0), (int64_t)D * 2};
        const int64_t n = rows_of(v0);
        hipLaunchKernelGGL(loss_rows_kernel, dim3((unsigned)up_to(n, 256)), dim3(256), 0, st, (const uint16_t *)W + v0 * ldW, ldW, D, nullptr, nullptr, n, w.pack, p.Dp);
        return ProductOperand{w.pack, p.Dp * 2, n, p.Dp * 2};
    };
    const ProductOperand tokens{w.H, p.Dp * 2, p.Tp, p.Dp * 2};
    const bool raw = p.raw > 1 && piece == p.Vp;
    const int per_part = raw ? kGather : p.per_part;
    auto parts_of = [&](int64_t entries) { return (entries + per_part - 1) / per_part; };
    auto hidden_product = [&](const ProductOperand &rows, int64_t n, int64_t v0) {        // dH's planes: rows m columns of W, columns n tokens
        const ProductArgs a{ProductOperand{rows.base, rows.ld, rows.depth, n}, ProductOperand{w.delta, piece * 2, few ? 2 * kFew : p.Tp, up_to(n, 64) * 2},
                            few ? 2 * kFew : T, n, few ? nullptr : w.count, nullptr, (D + 255) / 256, p.splits, nullptr,
                            w.shift, p.Tp, raw ? 4 : per_part == 128 ? 1 : 0};
        const float *shrink = v0 > 0 ? w.shrink : nullptr;
        if (few) return launch_product<LossTerms, ACROSS, ALONG, LossPlane<true>>(a, LossPlane<true>::Args{w.planes, p.Tp, p.Dp, shrink}, st);
        const LossPlane<false>::Args e{w.planes, p.Tp, p.Dp, shrink};
        return power ? loss_product<LossPlane<false>, ACROSS, ALONG, 64, true>(p.tile_n, a, e, st) : loss_product<LossPlane<false>, ACROSS, ALONG, 64>(p.tile_n, a, e, st);
    };
    auto head_product = [&](int64_t n, int64_t v0) {        // dW: rows m columns of H, columns n entries
        ProductArgs a{ProductOperand{w.H, p.Dp * 2, p.Dp * 2, p.Tp}, ProductOperand{w.delta, piece * 2, up_to(n, 64) * 2, few ? 2 * kFew : p.Tp},
                      n, p.Tp, nullptr, w.count, (D + 255) / 256, 1, nullptr, nullptr, 0, 0};             // (without live tokens delta may be unwritten: no stage)
        const LossHead::Args e{(uint16_t *)dW, ldDW, v0, V, D, w.order, w.order_target, w.start, w.pull, w.H, p.Dp};
        if (a.mtiles * ((n + 255) / 256) < compute_units()) {            // 512 x 512 x 2000: 104 -> 86 us; a chip full of the larger ones is 5 % faster
            a.mtiles = (D + 127) / 128;
            return launch_product<LossSmall, ACROSS, ACROSS, LossHead>(a, e, st);
        }
        return launch_product<Loss256, ACROSS, ACROSS, LossHead>(a, e, st);
    };

    if (T <= 64) {
        hipLaunchKernelGGL(loss_start_kernel, dim3((unsigned)p.Tp), dim3(256), 0, st, target, weight, (int)T, V, w, nll, lse, (const uint16_t *)H, ldH, D, p.Dp, few ? 1 : 0);
    } else if (T <= 1024) {
        hipLaunchKernelGGL(loss_start_many_kernel, dim3((unsigned)p.Tp), dim3(256), 0, st, target, weight, (int)T, V, w, nll, lse, (const uint16_t *)H, ldH, D, p.Dp);
    } else {
        hipLaunchKernelGGL(loss_live_kernel, dim3((unsigned)((T + kLossThreads - 1) / kLossThreads)), dim3(kLossThreads), 0, st, target, weight, T, V, w, nll, lse);
        hipLaunchKernelGGL(loss_rows_kernel, dim3((unsigned)p.Tp), dim3(256), 0, st, (const uint16_t *)H, ldH, D, w.token, w.count, p.Tp, w.H, p.Dp);
    }
    if (dW)
        hipLaunchKernelGGL(loss_order_kernel, dim3((unsigned)((T + 15) / 16 + (p.Vp / 64 + 1 + 15) / 16)), dim3(256), 0, st, w, T, p.Vp / 64 + 1);
    qless_status rc = QLESS_OK;
    // first pass: the losses, and dH unless delta comes with dW
    const bool run = few && dH && !one_pass, store = one_pass || run;
    for (int64_t v0 = 0; T > 0 && v0 < V && rc == QLESS_OK; v0 += piece) {
        const int64_t n = rows_of(v0), np = up_to(n, 256), parts = parts_of(np);
        const ProductOperand rows = head(v0);
        const ProductArgs a{rows, tokens, T, p.Dp, w.count, nullptr, 0, raw ? p.raw : 1, nullptr, nullptr, 0, 0};
        if (raw) {
            rc = logits_product<LossPlane<false>, 32>(p, a, np, LossPlane<false>::Args{w.raw, p.Tp, p.Vp, nullptr}, st);
            auto gather = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)T, (unsigned)parts), dim3(256), 0, st, w, p.Tp, p.Vp, p.raw, V); };
            power ? gather(loss_gather_kernel<POWERS>) : store ? gather(loss_gather_kernel<LOGITS>) : gather(loss_gather_kernel<SUMS>);
        } else if (power) {
            rc = logits_product<LossPower, 64>(p, a, np, LossPower::Args{w.target, w.hit, w.part, p.Tp, v0, V, w.delta, piece}, st);
        } else if (store) {
            rc = logits_product<LossStats<true>, 32>(p, a, np, LossStats<true>::Args{w.target, w.hit, w.part, p.Tp, v0, V, w.logits, piece}, st);
        } else {
            rc = logits_product<LossStats<false>, 32>(p, a, np, LossStats<false>::Args{w.target, w.hit, w.part, p.Tp, v0, V, nullptr, 0}, st);
        }
        if (rc != QLESS_OK) break;
        if (power) {
            if (T <= 1024) hipLaunchKernelGGL(loss_shift_kernel<4>, dim3((unsigned)((T + 3) / 4)), dim3(1024), 0, st, w, p.Tp, parts, v0 == 0 ? 1 : 0);
            else hipLaunchKernelGGL(loss_shift_kernel<16>, dim3((unsigned)((T + 15) / 16)), dim3(1024), 0, st, w, p.Tp, parts, v0 == 0 ? 1 : 0);
        } else if (store) {
            int64_t shares = run || T >= 1024 ? 1 : 1024 / T + 1;              // of a row
            if (shares > np / 1024) shares = np / 1024 > 0 ? np / 1024 : 1;
            auto delta = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, dim3((unsigned)up_to(T, few ? kFew : 64), (unsigned)shares), dim3(256), 0, st, w, p.Tp, parts, v0, np, piece, nll, lse);
            };
            run ? delta(loss_delta_kernel<true, true>) : few ? delta(loss_delta_kernel<false, true>) : delta(loss_delta_kernel<false, false>);
        }
        if (dH) rc = hidden_product(rows, n, v0);
        if (rc == QLESS_OK && dW && one_pass) rc = head_product(n, v0);
    }
    if (rc != QLESS_OK) return rc;
    if (T > 0 && !store && !power) {
        const int64_t parts = parts_of(p.Vp);
        if (T <= 64) hipLaunchKernelGGL(loss_join_kernel<1>, dim3((unsigned)T), dim3(256), 0, st, w, p.Tp, parts, nll, lse);
        else hipLaunchKernelGGL(loss_join_kernel<4>, dim3((unsigned)((T + 3) / 4)), dim3(256), 0, st, w, p.Tp, parts, nll, lse);
    }
    if (T > 0 && dH) {
        auto hidden = [&](auto kernel, int cols) {
            int64_t shares = 2048 / T + 1;
            if (shares > (D + cols - 1) / cols) shares = (D + cols - 1) / cols;
            hipLaunchKernelGGL(kernel, dim3((unsigned)T, (unsigned)shares), dim3(256), 0, st, w, p.Tp, p.Dp, D, p.splits, power ? 2 : run ? 1 : 0, (const uint16_t *)W, ldW, (uint16_t *)dH, ldDH, nll, lse);
        };
        if (p.splits >= 16) hidden(loss_hidden_kernel<16>, 64);
        else if (p.splits >= 4) hidden(loss_hidden_kernel<4>, 256);
        else hidden(loss_hidden_kernel<1>, 1024);
    }

    // second pass: delta from the known losses, a piece at a time, and dW
    for (int64_t v0 = 0; dW && (!one_pass || T == 0) && v0 < V && rc == QLESS_OK; v0 += piece) {
        const int64_t n = rows_of(v0);
        const ProductArgs a{head(v0), tokens, T, p.Dp, w.count, nullptr, (int32_t)(up_to(n, 256) / 256), 1, nullptr, nullptr, 0, 0};
        if (few) rc = launch_product<Loss32, ALONG, ALONG, LossDelta<true>>(a, LossDelta<true>::Args{w.target, w.lse, w.weight, w.delta, piece, v0, V}, st);
        else rc = loss_product<LossDelta<false>, ALONG, ALONG, 64>(p.tile_n, a, LossDelta<false>::Args{w.target, w.lse, w.weight, w.delta, piece, v0, V}, st);
        if (rc == QLESS_OK) rc = head_product(n, v0);
    }
    return rc == QLESS_OK ? launch_status() : rc;
}
