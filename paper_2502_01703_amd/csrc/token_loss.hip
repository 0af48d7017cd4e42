// qless_token_loss: softmax cross entropy of tokens over a vocabulary, from the last hidden states H and the head's weights W, with
// its gradients, without the T x V logits.
//   z = H W^T,  lse_t = log sum_v exp z_tv,  nll_t = lse_t - z_t,target,  delta_tv = w_t (exp(z_tv - lse_t) - [v = target_t]),
//   dH = delta W,  dW = delta^T H.
// Tokens without a target in the vocabulary are left out: the others' rows of H are gathered first (bounded by T on the host, counted
// on the device), so that a prompt costs no products.  A first pass over the vocabulary keeps each token's maximum and sum of 256
// logits at a time; a second one, a piece of the vocabulary after another, forms the logits again and leaves delta of the piece as
// bfloat16 in the workspace, which the products for dH and dW read.
#include "product.h"
#include "score.h"

namespace qless {

struct LossTokens {                        // workspace views, by live token (padded to whole tiles)
    uint16_t *H;                           // [Tp][Dp] bfloat16: gathered rows, zeros behind them
    int32_t *count;                        // live tokens
    int32_t *token, *target;               // [Tp]
    int32_t *place;                        // [T]: live index of a token, or -1
    float *weight, *lse, *nll, *hit;       // [Tp]; hit: the target's logit
    float2 *part;                          // [parts][Tp] maximum, sum of exp(z - maximum)
    uint16_t *delta;                       // [Tp][Vc]
    uint16_t *pack;                        // [Vc][Dp] where W cannot be read as it lies
    float *planes;                         // [splits][Tp][Dp] partial dH
};
struct LossPlan {
    int64_t T, Tp, Dp, Vp, Vc, parts;
    int32_t D, V, tile_n, splits;
    bool packed;
    size_t off[12], total;
};

constexpr int kLossThreads = 1024;

// One workgroup numbers the live tokens in their order: eight tokens a thread and pass.
__global__ void __launch_bounds__(kLossThreads)
loss_live_kernel(const int64_t *target, const float *weight, int64_t T, int32_t V, LossTokens w, float *nll, float *lse) {
    __shared__ int32_t s_wave[kLossThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t before = 0;
    for (int64_t t0 = 0; t0 < T; t0 += 8 * kLossThreads) {
        int64_t y[8];
        int32_t mine = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t t = t0 + 8 * tid + i;
            y[i] = t < T ? target[t] : -1;
            mine += y[i] >= 0 && y[i] < V;
        }
        int32_t up = mine;                                 // inclusive sums over the wavefront
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int32_t o = __shfl_up(up, d, 64);
            up += lane >= d ? o : 0;
        }
        __syncthreads();
        if (lane == 63) s_wave[wave] = up;
        __syncthreads();
        int32_t at = before + up - mine;
        for (int i = 0; i < kLossThreads / 64; ++i) {
            if (i < wave) at += s_wave[i];
            before += s_wave[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t t = t0 + 8 * tid + i;
            if (t >= T) break;
            const bool live = y[i] >= 0 && y[i] < V;
            w.place[t] = live ? at : -1;
            if (live) {
                w.token[at] = (int32_t)t;
                w.target[at] = (int32_t)y[i];
                w.weight[at] = weight ? weight[t] : 1.0f;
                ++at;
            } else {
                nll[t] = 0.0f;
                if (lse) lse[t] = 0.0f;
            }
        }
    }
    if (tid == 0) *w.count = before;
}

// Rows of bfloat16 copied to rows of ld (a multiple of 64) with zeros behind their D elements, eight elements a thread; `from` null: row r,
// else the row that it names, and zeros from *count up to whole tiles.
__global__ void __launch_bounds__(256)
loss_rows_kernel(const uint16_t *X, int64_t ldX, int32_t D, const int32_t *from, const int32_t *count, int64_t rows, uint16_t *out, int64_t ld) {
    const int64_t r = blockIdx.x;
    const int64_t n = count ? *count : rows;
    if (r >= (n + 255) / 256 * 256) return;
    const uint16_t *x = r < n ? X + (from ? (int64_t)from[r] : r) * ldX : nullptr;
    for (int64_t c = threadIdx.x * 8; c < ld; c += 256 * 8) {
        uint16_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0;
        if (x && c + 8 <= D) __builtin_memcpy(v, x + c, 16);
        else if (x)
#pragma unroll
            for (int i = 0; i < 8; ++i) if (c + i < D) v[i] = x[c + i];
        __builtin_memcpy(__builtin_assume_aligned(out + r * ld + c, 16), v, 16);
    }
}

// ---- what the tiles of logits end with: rows m are vocabulary entries, columns n tokens
struct LossStats {
    struct Args { const int32_t *target; float *hit; float2 *part; int64_t Tp, first; int32_t V; };
    template <int FM, int FN>
    static __device__ inline void run(const Args &a, f32x16 (&acc)[FM][FN], int64_t m, int64_t n, int, int64_t live) {
        const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
        const int64_t part = (a.first + m) / (32 * FM);
        const int v0 = (int)(a.first + m) + 4 * half, over = a.V - v0;         // entries from here on
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int64_t t = n + 32 * j + l32;
            const int y = t < live ? a.target[t] - v0 : -1;
            float hit = 0.0f;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int at = 32 * i + 8 * (v >> 2) + (v & 3);
                    hit = y == at ? acc[i][j][v] : hit;
                    acc[i][j][v] = at < over ? acc[i][j][v] : -INFINITY;
                }
            if (y >= 0 && y < 32 * FM && (y & 4) == 0) a.hit[t] = hit;
            float top = acc[0][j][0];
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) top = fmaxf(top, acc[i][j][v]);
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float ref = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) sum += __expf(acc[i][j][v] - ref);
            sum += __shfl_xor(sum, 32, 64);
            if (half == 0 && t < live) a.part[part * a.Tp + t] = make_float2(top, sum);
        }
    }
};

struct LossDelta {
    struct Args { const int32_t *target; const float *lse, *nll, *weight; uint16_t *delta; int64_t Tp, ld, first; int32_t V; };
    template <int FM, int FN>
    static __device__ inline void run(const Args &a, f32x16 (&acc)[FM][FN], int64_t m, int64_t n, int, int64_t live) {
        const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int64_t t = n + 32 * j + l32;
            const bool on = t < live;
            const float lse = on ? a.lse[t] : 0.0f, w = on ? a.weight[t] : 0.0f, at_target = on ? w * expm1f(-a.nll[t]) : 0.0f;
            const int64_t y = on ? a.target[t] - a.first : -1;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int64_t c = m + 32 * i + 8 * q + 4 * half;          // of the piece
                    uint16_t d[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        float x = w * __expf(acc[i][j][4 * q + u] - lse);
                        if (y == c + u) x = at_target;
                        if (!on || a.first + c + u >= a.V) x = 0.0f;
                        d[u] = __builtin_bit_cast(uint16_t, (__bf16)x);
                    }
                    __builtin_memcpy(__builtin_assume_aligned(a.delta + t * a.ld + c, 8), d, 8);
                }
        }
    }
};

// rows m are columns of dH, columns n tokens; pieces after the first add to what is there
struct LossPlane {
    struct Args { float *planes; int64_t Tp, Dp; int add; };
    template <int FM, int FN>
    static __device__ inline void run(const Args &a, f32x16 (&acc)[FM][FN], int64_t m, int64_t n, int split, int64_t live) {
        typedef __attribute__((ext_vector_type(4))) float f32x4;
        const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int64_t t = n + 32 * j + l32;
            if (t >= live) continue;
            float *row = a.planes + (split * a.Tp + t) * a.Dp;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int64_t d = m + 32 * i + 8 * q + 4 * half;
                    if (d >= a.Dp) continue;
                    f32x4 x;
#pragma unroll
                    for (int u = 0; u < 4; ++u) x[u] = acc[i][j][4 * q + u];
                    if (a.add) x += *(const f32x4 *)(row + d);
                    *(f32x4 *)(row + d) = x;
                }
        }
    }
};

// rows m are columns of dW, columns n vocabulary entries
struct LossHead {
    struct Args { uint16_t *dW; int64_t ld, first; int32_t V, D; };
    template <int FM, int FN>
    static __device__ inline void run(const Args &a, f32x16 (&acc)[FM][FN], int64_t m, int64_t n, int, int64_t) {
        const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int64_t v = a.first + n + 32 * j + l32;
            if (v >= a.V) continue;
            uint16_t *row = a.dW + v * a.ld;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int64_t d = m + 32 * i + 8 * q + 4 * half;
                    uint16_t x[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) x[u] = __builtin_bit_cast(uint16_t, (__bf16)acc[i][j][4 * q + u]);
                    if (d + 4 <= a.D) __builtin_memcpy(row + d, x, 8);
                    else
#pragma unroll
                        for (int u = 0; u < 4; ++u) if (d + u < a.D) row[d + u] = x[u];
                }
        }
    }
};

// lse and nll of TOK tokens from their parts, 256 / TOK threads each: the running maximum and the sum relative to it, then joined.
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
        const float next = fmaxf(top, x.x);
        if (next == -INFINITY) sum += x.y;                  // 0, or NaN of logits that are not numbers
        else sum = sum * __expf(top - next) + x.y * __expf(x.x - next);
        top = next;
    }
    s_top[threadIdx.x] = top; s_sum[threadIdx.x] = sum;
    __syncthreads();
    for (int h = LANES / 2; h > 0; h /= 2) {
        if (part < h) {
            const int o = threadIdx.x + h * TOK;
            const float a = s_top[threadIdx.x], b = s_top[o], next = fmaxf(a, b);
            if (next == -INFINITY) s_sum[threadIdx.x] += s_sum[o];
            else s_sum[threadIdx.x] = s_sum[threadIdx.x] * __expf(a - next) + s_sum[o] * __expf(b - next);
            s_top[threadIdx.x] = next;
        }
        __syncthreads();
    }
    if (part == 0 && t < live) {
        const float m = s_top[tok], l = logf(s_sum[tok]), all = m + l, one = l + (m - w.hit[t]);   // near 0 the loss keeps its digits
        w.lse[t] = all; w.nll[t] = one;
        const int64_t at = w.token[t];
        nll[at] = one;
        if (lse) lse[at] = all;
    }
}

// dH of a token: the sum of its planes, or zeros.
__global__ void __launch_bounds__(256)
loss_hidden_kernel(LossTokens w, int64_t Tp, int64_t Dp, int32_t D, int splits, uint16_t *dH, int64_t ld) {
    const int64_t t = blockIdx.x, r = w.place[t];
    for (int64_t c = threadIdx.x * 4; c < D; c += 256 * 4) {
        uint16_t x[4] = {0, 0, 0, 0};
        if (r >= 0) {
            float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (int p = 0; p < splits; ++p) {
                const float4 y = *(const float4 *)(w.planes + ((int64_t)p * Tp + r) * Dp + c);
                s.x += y.x; s.y += y.y; s.z += y.z; s.w += y.w;
            }
            const float f[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = __builtin_bit_cast(uint16_t, (__bf16)f[u]);
        }
        uint16_t *out = dH + t * ld + c;
        if (c + 4 <= D) __builtin_memcpy(out, x, 8);
        else
#pragma unroll
            for (int u = 0; u < 4; ++u) if (c + u < D) out[u] = x[u];
    }
}

typedef ProductShape<256, 256, 2, 4, 2> LossWide;          // many tokens
typedef ProductShape<256, 32, 8, 1, 4> LossFew;

static int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// Everything of a call that follows from its sizes.
static LossPlan loss_plan(int64_t T, int32_t D, int32_t V, bool gradient) {
    LossPlan p{};
    p.T = T; p.D = D; p.V = V;
    p.tile_n = T <= 32 ? 32 : 256;
    p.Tp = up_to(T > 0 ? T : 1, 256);
    p.Dp = up_to(D, 64);
    p.Vp = up_to(V, 256);
    p.parts = p.Vp / 256 * (p.tile_n == 32 ? LossFew::WY : LossWide::WY);
    // a piece: 256 MB of delta
    int64_t Vc = ((int64_t)256 << 20) / (2 * p.Tp) / 256 * 256;
    if (Vc < 256) Vc = 256;
    if (Vc > p.Vp) Vc = p.Vp;
    p.Vc = Vc;
    const int64_t tiles = ((D + 255) / 256) * ((T + p.tile_n - 1) / p.tile_n), stages = Vc / 64;
    int64_t splits = tiles > 0 ? 512 / tiles : 1;
    if (splits > stages / 8) splits = stages / 8;
    if (splits < 1) splits = 1;
    p.splits = (int32_t)splits;
    size_t at = 0;
    int i = 0;
    auto take = [&](size_t bytes) { p.off[i++] = at; at = (at + bytes + 255) & ~(size_t)255; };
    take((size_t)p.Tp * p.Dp * 2);                          // H
    take(256);                                              // count
    take((size_t)p.Tp * 4); take((size_t)p.Tp * 4); take((size_t)p.Tp * 4);               // token, target, place
    take((size_t)p.Tp * 4); take((size_t)p.Tp * 4); take((size_t)p.Tp * 4); take((size_t)p.Tp * 4);   // weight, lse, nll, hit
    take((size_t)p.parts * p.Tp * 8);                       // part
    // a piece's delta and, where W has to be packed, shorter pieces with the packed rows behind it: room for at least 64 MB of both
    size_t piece = gradient ? (size_t)p.Tp * Vc * 2 : 0, both = (size_t)(p.Tp + p.Dp) * 2 * p.Vp;
    if (both > ((size_t)64 << 20)) both = (size_t)64 << 20;
    if (both < (size_t)(p.Tp + p.Dp) * 2 * 256) both = (size_t)(p.Tp + p.Dp) * 2 * 256;
    take(piece > both ? piece : both);
    take(gradient ? (size_t)p.splits * p.Tp * p.Dp * 4 : 0);
    p.total = at;
    return p;
}

template <class Epilogue, int AK, int BK>
static qless_status loss_product(const LossPlan &p, const ProductArgs &a, const typename Epilogue::Args &e, hipStream_t st) {
    return p.tile_n == 32 ? launch_product<LossFew, AK, BK, Epilogue>(a, e, st) : launch_product<LossWide, AK, BK, Epilogue>(a, e, st);
}

}  // namespace qless

extern "C" size_t qless_token_loss_workspace(int64_t T, int32_t D, int32_t V, int gradient) {
    using namespace qless;
    if (T < 0 || D < 1 || V < 1) return 0;
    return loss_plan(T, D, V, gradient != 0).total;
}

extern "C" qless_status qless_token_loss(const void *H, int64_t ldH, const void *W, int64_t ldW, qless_dtype dt, int64_t T, int32_t D, int32_t V,
                                         const int64_t *target, const float *weight, float *nll, float *lse, void *dH, int64_t ldDH,
                                         void *dW, int64_t ldDW, void *ws, size_t ws_bytes, void *stream) {
    using namespace qless;
    if (T < 0 || D < 1 || V < 1 || (T > 1 && (ldH < D || (dH && ldDH < D))) || (V > 1 && (ldW < D || (dW && ldDW < D)))) return QLESS_ERR_INVALID_ARG;
    if (dt != QLESS_BF16 || D > 65536 || T > 0x3FFFFFFF) return QLESS_ERR_UNSUPPORTED;
    if (T == 0 && !dW) return QLESS_OK;
    if (!W || (T > 0 && (!H || !target || !nll))) return QLESS_ERR_INVALID_ARG;
    const bool gradient = dH || dW;
    LossPlan p = loss_plan(T, D, V, gradient);
    if (!ws || ws_bytes < p.total || ((uintptr_t)ws & 15) != 0) return QLESS_ERR_WORKSPACE;
    const qless_status ready = device_ready();
    if (ready != QLESS_OK) return ready;
    const hipStream_t st = (hipStream_t)stream;
    unsigned char *base = (unsigned char *)ws;
    LossTokens w{};
    w.H = (uint16_t *)(base + p.off[0]); w.count = (int32_t *)(base + p.off[1]);
    w.token = (int32_t *)(base + p.off[2]); w.target = (int32_t *)(base + p.off[3]); w.place = (int32_t *)(base + p.off[4]);
    w.weight = (float *)(base + p.off[5]); w.lse = (float *)(base + p.off[6]); w.nll = (float *)(base + p.off[7]); w.hit = (float *)(base + p.off[8]);
    w.part = (float2 *)(base + p.off[9]); w.delta = (uint16_t *)(base + p.off[10]); w.planes = (float *)(base + p.off[11]);

    hipLaunchKernelGGL(loss_live_kernel, dim3(1), dim3(kLossThreads), 0, st, target, weight, T, V, w, nll, lse);
    hipLaunchKernelGGL(loss_rows_kernel, dim3((unsigned)p.Tp), dim3(256), 0, st, (const uint16_t *)H, ldH, D, w.token, w.count, p.Tp, w.H, p.Dp);

    // W is read where it lies if its rows are whole 16-byte chunks; else a piece at a time is packed into the workspace
    p.packed = ((uintptr_t)W & 15) != 0 || (ldW % 8 != 0 && V > 1) || D % 8 != 0 || ldW * 2 >= ((int64_t)1 << 23);
    int64_t piece = p.Vc;
    if (p.packed) {
        piece = (int64_t)((p.off[11] - p.off[10]) / ((size_t)(p.Tp + p.Dp) * 2)) / 256 * 256;
        if (piece > p.Vc) piece = p.Vc;
        w.pack = w.delta + p.Tp * piece;
    }
    const ProductOperand tokens{w.H, p.Dp * 2, p.Tp, p.Dp * 2};
    auto head = [&](int64_t v0, int64_t n) {               // n entries from v0 on, by rows of D
        if (!p.packed) return ProductOperand{(const uint16_t *)W + v0 * ldW, ldW * 2, n, (int64_t)D * 2};
        hipLaunchKernelGGL(loss_rows_kernel, dim3((unsigned)up_to(n, 256)), dim3(256), 0, st, (const uint16_t *)W + v0 * ldW, ldW, D, nullptr, nullptr, n, w.pack, p.Dp);
        return ProductOperand{w.pack, p.Dp * 2, n, p.Dp * 2};
    };
    qless_status rc = QLESS_OK;
    if (T > 0) {
        for (int64_t v0 = 0; v0 < V && rc == QLESS_OK; v0 += p.packed ? piece : p.Vp) {
            const int64_t n = p.packed && V - v0 > piece ? piece : V - v0;
            ProductArgs a{head(v0, n), tokens, T, p.Dp, w.count, nullptr, (int32_t)((n + 255) / 256), 1};
            rc = loss_product<LossStats, ALONG, ALONG>(p, a, LossStats::Args{w.target, w.hit, w.part, p.Tp, v0, V}, st);
        }
        if (rc != QLESS_OK) return rc;
        if (T <= 64) hipLaunchKernelGGL(loss_join_kernel<1>, dim3((unsigned)T), dim3(256), 0, st, w, p.Tp, p.parts, nll, lse);
        else hipLaunchKernelGGL(loss_join_kernel<16>, dim3((unsigned)((T + 15) / 16)), dim3(256), 0, st, w, p.Tp, p.parts, nll, lse);
    }
    for (int64_t v0 = 0; gradient && v0 < V && rc == QLESS_OK; v0 += piece) {
        const int64_t n = V - v0 < piece ? V - v0 : piece, np = up_to(n, 256);
        const ProductOperand rows = head(v0, n);
        ProductArgs a{rows, tokens, T, p.Dp, w.count, nullptr, (int32_t)(np / 256), 1};
        rc = loss_product<LossDelta, ALONG, ALONG>(p, a, LossDelta::Args{w.target, w.lse, w.nll, w.weight, w.delta, p.Tp, piece, v0, V}, st);
        if (rc == QLESS_OK && dH) {
            ProductArgs b{ProductOperand{rows.base, rows.ld, rows.depth, n}, ProductOperand{w.delta, piece * 2, p.Tp, np * 2}, T, n, w.count, nullptr,
                          (D + 255) / 256, p.splits};
            rc = loss_product<LossPlane, ACROSS, ALONG>(p, b, LossPlane::Args{w.planes, p.Tp, p.Dp, v0 > 0}, st);
        }
        if (rc == QLESS_OK && dW) {
            ProductArgs b{ProductOperand{w.H, p.Dp * 2, p.Dp * 2, p.Tp}, ProductOperand{w.delta, piece * 2, np * 2, up_to(T > 0 ? T : 1, p.tile_n)}, n, p.Tp, nullptr, w.count,
                          (D + 255) / 256, 1};
            rc = launch_product<LossWide, ACROSS, ACROSS, LossHead>(b, LossHead::Args{(uint16_t *)dW, ldDW, v0, V, D}, st);
        }
    }
    if (rc != QLESS_OK) return rc;
    if (dH && T > 0)
        hipLaunchKernelGGL(loss_hidden_kernel, dim3((unsigned)T), dim3(256), 0, st, w, p.Tp, p.Dp, D, p.splits, (uint16_t *)dH, ldDH);
    return launch_status();
}
