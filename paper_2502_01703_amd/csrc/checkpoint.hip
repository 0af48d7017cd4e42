// qless_checkpoint8, qless_checkpoint8_read, qless_checkpoint8_grad: activations kept in 8 bits between the forward and the
// backward pass, and the per-example weight gradients that are taken from them.
//
// A group is 128 columns of a row (the last one of a row may be shorter).  Its step s is the least number of eight significant
// bits, at least 2^-126, of which 127 reach the group's largest absolute value; a code is the nearest whole number of steps, ties
// to even, so that |code| <= 127.  Eight bits of step cost at most 1/128 of resolution, and buy products: a code (7 bits) is a
// bfloat16, and a bfloat16 gradient times a step (16 bits) is the sum of two, so that the backward pass is exact up to its
// fp32 sums with two matrix products instead of three.  A group with an infinity or a NaN gets the step NaN and codes 0.
#include "product.h"
#include "score.h"
#include <cmath>
#include <type_traits>

namespace qless {

constexpr int kGroup = QLESS_CHECKPOINT_GROUP;
constexpr int64_t kMostThreads = ((int64_t)1 << 32) - 256; // of a launch, in whole workgroups of 256

__device__ inline float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ inline uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// Eight elements from p on, whatever its alignment; those past `left` are 0 (left <= 0: none is read).
template <class T> struct Eight;
template <> struct Eight<float> {
    static __device__ inline void load(const float *p, int64_t left, float (&x)[8]) {
        if (left >= 8) __builtin_memcpy(x, p, 32);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = i < left ? p[i] : 0.0f;
    }
    static __device__ inline void store(float *p, int64_t left, const float (&x)[8]) {
        if (left >= 8) __builtin_memcpy(p, x, 32);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i < left) p[i] = x[i];
    }
};
template <> struct Eight<uint16_t> {                      // bfloat16
    static __device__ inline void load(const uint16_t *p, int64_t left, float (&x)[8]) {
        uint16_t b[8];
        if (left >= 8) __builtin_memcpy(b, p, 16);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = i < left ? p[i] : (uint16_t)0;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = bf16_value(b[i]);
    }
    // activations: codes times steps.  127 steps may lie less than one past the largest bfloat16, and stand for it, not for infinity
    static __device__ inline void store(uint16_t *p, int64_t left, const float (&x)[8]) {
        uint16_t b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            b[i] = bf16_bits(x[i]);
            b[i] -= (b[i] & 0x7FFF) == 0x7F80 ? 1 : 0;
        }
        if (left >= 8) __builtin_memcpy(p, b, 16);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i < left) p[i] = b[i];
    }
};

// Maximum over the 16 lanes of a DPP row, in all of them.
template <int CTRL> __device__ inline uint32_t row_rotate(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
__device__ inline uint32_t row_max(uint32_t x) {
    x = max(x, row_rotate<0x128>(x)); x = max(x, row_rotate<0x124>(x));
    x = max(x, row_rotate<0x122>(x)); x = max(x, row_rotate<0x121>(x));
    return x;
}

// The step of a group whose largest absolute value has the bits `top` (order of non-negative floats; above: infinity, NaN).
__device__ inline float group_step(uint32_t top) {
    if (top == 0) return 0.0f;
    if (top >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    const float a = __uint_as_float(top);
    const float s = __uint_as_float((__float_as_uint(__fdiv_rn(a, 127.0f)) + 0xFFFFu) & 0xFFFF0000u);
    // 127 s is exact (15 bits); the quotient may have been rounded down onto a number of eight bits
    const float t = __fmul_rn(s, 127.0f) < a ? __uint_as_float(__float_as_uint(s) + 0x10000u) : s;
    return fmaxf(t, 1.17549435e-38f);
}
// The nearest whole number of steps: the product with the rounded reciprocal is off by less than 2^-16, the remainder
// x - q s is exact (q s has 15 bits, and no bit of x lies below 2^-25 s unless q is 0) and says on which side of the half x lies.
__device__ inline int nearest_code(float x, float s, float inv) {
    float q = rintf(__fmul_rn(x, inv));
    const float r = __builtin_fmaf(-q, s, x), twice = fabsf(r + r);
    const bool odd = ((int)q & 1) != 0;
    if (twice > s || (twice == s && odd)) q += r < 0.0f ? -1.0f : 1.0f;
    return (int)q;
}

// A workgroup takes kItems consecutive groups, 16 lanes a group and eight columns a lane, kPer of them on their way together.  One division
// per workgroup finds its first row; the lanes' own are of 32 bits (one of 64 bits per group took as long as the memory).
// Bound: memory, read once and written once.
constexpr int kPer = 2, kItems = 16 * kPer;
struct GroupPlace { int64_t t; int g; };
__device__ inline GroupPlace group_place(int64_t first, int local, int32_t groups) {       // first: uniform
    const int64_t t0 = first / groups;
    const unsigned at = (unsigned)(first - t0 * groups) + (unsigned)local, up = at / (unsigned)groups;
    return GroupPlace{t0 + up, (int)(at - up * (unsigned)groups)};
}

template <class T>
__global__ void __launch_bounds__(256)
checkpoint_write_kernel(const T *X, int64_t rows, int32_t D, int64_t ldX, int32_t groups, int8_t *codes, int64_t ldC, float *step, int64_t ldS) {
    const int64_t total = rows * groups, first = (int64_t)blockIdx.x * kItems;
    const int col = (threadIdx.x & 15) * 8;
    float x[kPer][8];
    GroupPlace at[kPer];
    int left[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int local = u * 16 + (threadIdx.x >> 4);
        at[u] = group_place(first, local, groups);
        const int c = at[u].g * kGroup + col;
        left[u] = first + local < total ? D - c : 0;
        Eight<T>::load(X + at[u].t * ldX + c, left[u], x[u]);
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[u][j]) & 0x7FFFFFFFu);
        top = row_max(top);
        const float s = group_step(top);
        const bool plain = top != 0 && top < 0x7F800000u;
        const float inv = plain ? __fdiv_rn(1.0f, s) : 0.0f;
        int8_t q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = plain ? (int8_t)nearest_code(x[u][j], s, inv) : (int8_t)0;
        int8_t *out = codes + at[u].t * ldC + at[u].g * kGroup + col;
        if (left[u] >= 8) __builtin_memcpy(out, q, 8);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) if (j < left[u]) out[j] = q[j];
        if (col == 0 && left[u] > 0) step[at[u].t * ldS + at[u].g] = s;
    }
}

template <class T>
__global__ void __launch_bounds__(256)
checkpoint_read_kernel(const int8_t *codes, int64_t ldC, const float *step, int64_t ldS, int64_t rows, int32_t D, int32_t groups, T *X, int64_t ldX) {
    const int64_t total = rows * groups, first = (int64_t)blockIdx.x * kItems;
    const int col = (threadIdx.x & 15) * 8;
    int8_t q[kPer][8];
    float s[kPer];
    GroupPlace at[kPer];
    int left[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int local = u * 16 + (threadIdx.x >> 4);
        at[u] = group_place(first, local, groups);
        const int c = at[u].g * kGroup + col;
        left[u] = first + local < total ? D - c : 0;
        const int8_t *in = codes + at[u].t * ldC + c;
        if (left[u] >= 8) __builtin_memcpy(q[u], in, 8);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) q[u][j] = j < left[u] ? in[j] : (int8_t)0;
        s[u] = left[u] > 0 ? step[at[u].t * ldS + at[u].g] : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __fmul_rn((float)q[u][j], s[u]);
        Eight<T>::store(X + at[u].t * ldX + at[u].g * kGroup + col, left[u], x);
    }
}

// ---------------------------------------------------------------------------------------------------------------------------
// Weight gradients per example: G_e[r][d] = sum over the tokens t of example e of dY[t][r] code[t][d] step[t][d / 128].
//
// An example longer than `chunk` tokens is cut into segments of that many.  With phi(e) = e + floor(offset[e] / chunk), the numbers
// phi(e) .. phi(e + 1) - 1 suffice for those of example e (one may be left over), so that any workgroup finds its segment by a search
// over the offsets, with no list of them in memory; an example of one segment is written at once, the others' segments leave fp32
// planes that a second kernel adds in their order.  Up to 256 examples a wavefront knows them all, and the workgroups are numbered from
// the longest segments to the shortest ones: none of the long ones begins last (32 ragged
// examples of 16384 tokens, R = 128, D = 4096: 75 -> 56 us; 64 of 32768, R = 64: 77 -> 61; 128 of them: 86 -> 73).
struct GradArgs {
    const void *dY; int64_t ldY;
    const int8_t *codes; int64_t ldC;
    const float *step; int64_t ldS;
    const int64_t *offsets;
    int64_t n, T, chunk, segments, first;                  // first: segment of a launch
    int32_t R, D, rtiles, dtiles;
    int32_t Rc, Dc;                                        // columns of dY and codes that may be read: R and D, or more where they are packed
    void *G; int64_t ldG;
    float *planes;                                         // [segments][R][D]
};
struct Segment { int64_t e, lo, hi, plane; bool whole; };     // plane: phi(e) and on

__device__ inline int64_t offset_at(const GradArgs &a, int64_t e) {      // never outside the tokens, whatever the caller wrote there
    const int64_t o = a.offsets[e];
    return o < 0 ? 0 : (o > a.T ? a.T : o);
}
__device__ inline int64_t readlane64(int64_t x, int lane) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)x >> 32), lane);
    return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ inline int64_t phi(const GradArgs &a, int64_t e, int64_t chunk) { return e + offset_at(a, e) / chunk; }
// The example with phi(example) <= j < phi(example + 1), or -1; the whole wavefront asks, 64 examples at a time (a search by halves is a
// chain of loads as long as a few stages of the work itself).
__device__ inline int64_t find_example(const GradArgs &a, int64_t j, int64_t chunk, int64_t &o0, int64_t &o1) {
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = a.n;                              // phi(lo) <= j < phi(hi), once both are known
    bool inside = j < phi(a, a.n, chunk);
    for (;;) {
        const int64_t step = (hi - lo + 63) / 64, e = lo + lane * step < hi ? lo + lane * step : hi - 1;
        const int64_t first = offset_at(a, e), second = offset_at(a, e + 1);
        const uint64_t below = __ballot(lo + lane * step < hi && e + first / chunk <= j);
        if (below == 0) inside = false;                    // j < phi(0)
        if (!inside) return -1;
        const int at = 63 - __clzll((long long)below);
        lo += at * step;
        if (step == 1) {
            o0 = readlane64(first, at);
            o1 = readlane64(second, at);
            break;
        }
        hi = lo + step < hi ? lo + step : hi;
    }
    return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)lo);
}
// Up to 64 K examples, number 64 k + lane in `[k]` of a lane: `full` segments of a.chunk tokens each, and one of `rest` tokens, of which
// the one with r longer ones (or as long and before it) is found by the bits of its length.
template <int K> __device__ inline bool ranked_segment(const GradArgs &a, int64_t j, Segment &s) {
    const int lane = threadIdx.x & 63, n = (int)a.n;
    int64_t o0[K], o1[K], full[K], upto[K], fulls = 0;
    int rest[K];                                           // -1: none
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = 64 * k + lane;
        o0[k] = offset_at(a, e < n ? e : n);
        o1[k] = offset_at(a, e < n ? e + 1 : n);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int64_t len = o1[k] > o0[k] ? o1[k] - o0[k] : 0;
        full[k] = len < a.chunk ? 0 : len / a.chunk;
        upto[k] = full[k];
        if (__any(full[k] > 0))
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int64_t o = __shfl_up(upto[k], d, 64);
                if (lane >= d) upto[k] += o;
            }
        upto[k] += fulls;
        fulls = readlane64(upto[k], 63);
        const int64_t left = len - full[k] * a.chunk;
        rest[k] = 64 * k + lane >= n || (left == 0 && len > 0) ? -1 : left < 0x3FFFFFFF ? (int)left : 0x3FFFFFFF;
    }
    auto count = [&](int least) {
        int c = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) c += __popcll(__ballot(rest[k] >= least));
        return c;
    };
    const bool whole_chunk = j < fulls;
    int64_t r = j - fulls;
    int length = 0;
    if (!whole_chunk) {
        if (r >= count(0)) return false;
        for (int bit = a.chunk < 0x40000000 ? 1 << (31 - __clz((int)a.chunk)) : 0x20000000; bit > 0; bit >>= 1)
            if (count(length | bit) > r) length |= bit;
        r -= count(length + 1);
    }
    bool found = false;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (found) continue;
        const uint64_t at_length = __ballot(rest[k] == length), it = __ballot(whole_chunk ? upto[k] > j : rest[k] == length && __popcll(at_length & (((uint64_t)1 << lane) - 1)) == r);
        if (it == 0) {
            r -= __popcll(at_length);
            continue;
        }
        found = true;
        const int at = __ffsll((unsigned long long)it) - 1;
        const int64_t first = readlane64(o0[k], at), end = readlane64(o1[k], at), len = end > first ? end - first : 0, whole = readlane64(full[k], at);
        const int64_t i = whole_chunk ? j - (readlane64(upto[k], at) - whole) : whole;
        s.e = 64 * k + at;
        s.lo = readlane64(first + i * a.chunk, 0);         // in scalar registers: bases of the copies
        s.hi = readlane64(whole_chunk ? s.lo + a.chunk : first + len, 0);
        s.whole = len <= a.chunk;
        s.plane = s.whole ? 0 : s.e + first / a.chunk + i;
    }
    return found;
}
__device__ inline bool find_segment(const GradArgs &a, int64_t j, Segment &s) {
    if (a.n <= 64) return ranked_segment<1>(a, j, s);
    if (a.n <= 256) return ranked_segment<4>(a, j, s);
    int64_t o0, o1;
    s.e = find_example(a, j, a.chunk, o0, o1);
    if (s.e < 0) return false;
    const int64_t i = j - (s.e + o0 / a.chunk);
    s.lo = o0 + i * a.chunk;
    if (i > 0 && s.lo >= o1) return false;
    s.hi = s.lo + a.chunk < o1 ? s.lo + a.chunk : o1;
    s.whole = o1 - o0 <= a.chunk;
    s.plane = j;
    return true;
}

// What a wavefront writes: its accumulators (a lane holds four columns of one row) through LDS of its own, so that the lanes of a
// store lie along rows of G (64 examples of 32768 tokens, R = 64, D = 4096: 61 -> 56 us; 2 of 11, R = 2409, D = 7603: 123 -> 86).  `row`: the lane's row of 16; first: of the tile.
template <int CM, int CN, class E, bool TAIL>
__device__ inline void put_tile(unsigned char *lds, const f32x4 (&acc)[CM][CN], E *out, int row, int r0, int d0, int32_t R, int32_t D) {
    constexpr int LD = CM * 64 + 16, LANES = CM * 4;       // of a row
    const int lane = threadIdx.x & 63, quad = lane >> 4, at = lane / LANES, c = lane % LANES * 4, left = D - d0 - c;
    out += d0 + c;
#pragma unroll
    for (int n = 0; n < CN; ++n) {
        __builtin_amdgcn_wave_barrier();                   // LDS operations of a wavefront complete in order
#pragma unroll
        for (int m = 0; m < CM; ++m) *(f32x4 *)(lds + row * LD + m * 64 + quad * 16) = acc[m][n];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < CM; ++i) {
            const int k = i * (64 / LANES) + at, r = r0 + n * 16 + k;
            const f32x4 y = *(const f32x4 *)(lds + k * LD + c * 4);
            if (r >= R || left <= 0) continue;
            E x[4], *to = out + (int64_t)r * D;
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = sizeof(E) == 2 ? (E)bf16_bits(y[u]) : (E)y[u];
            if (!TAIL || left >= 4) __builtin_memcpy(to, x, sizeof x);
            else
#pragma unroll
                for (int u = 0; u < 4; ++u) if (u < left) to[u] = x[u];
        }
    }
}
template <class Out, int CM, int CN>
__device__ inline void put_segment(const GradArgs &a, const Segment &s, unsigned char *lds, const f32x4 (&acc)[CM][CN], int row, int r0, int d0) {
    auto put = [&](auto tail) {
        if (s.whole) put_tile<CM, CN, Out, decltype(tail)::value>(lds, acc, (Out *)a.G + s.e * a.ldG, row, r0, d0, a.R, a.D);
        else put_tile<CM, CN, float, decltype(tail)::value>(lds, acc, a.planes + s.plane * a.R * (int64_t)a.D, row, r0, d0, a.R, a.D);
    };
    if (a.D % 4 == 0) put(std::false_type());              // (the code of partial stores is not fetched)
    else put(std::true_type());
}

// Tiles of RT rows of R x 128 columns (one group: a token has one step there), four wavefronts, 64 tokens a stage.  A stage's codes
// become bfloat16, its gradients times their step the sum of TERMS bfloat16; both lie in LDS as rows of a token, and the matrix operands
// (eight tokens of a column in a lane) are formed by the transposing LDS reads.  The order of the tokens inside a product is that of
// those reads, alike on both sides.  32-byte pieces of a row are exchanged by its token's low bits: the eight rows that 32 lanes read
// together lie in different banks.  RT is at most 64: with 128 rows one workgroup fits a compute unit, and waits for its loads alone (2 examples of 11 tokens,
// R = 2409, D = 7603: 86 us, with 64 49; 8 of 4000 tokens, R = 100, D = 1333: 31 and 24).
template <int RT, class Y, int TERMS, class Out>
__global__ void __launch_bounds__(256)
checkpoint_grad_kernel(GradArgs a) {
    constexpr int KT = 64, WY = RT >= 64 ? 2 : 1, WX = 4 / WY, CM = 128 / WX / 16, CN = RT / WY / 16;
    constexpr int YROW = RT * 2, YPLANE = KT * YROW, PIECES = KT * RT / 8, PER = (PIECES + 255) / 256;
    __shared__ __attribute__((aligned(16))) unsigned char s_all[KT * 256 + TERMS * YPLANE];
    unsigned char *s_codes = s_all, *s_y = s_all + KT * 256;
    static_assert(16 * (CM * 64 + 16) * 4 <= KT * 256 + TERMS * YPLANE, "16 rows of each wavefront");
    const int64_t tiles = (int64_t)a.rtiles * a.dtiles, j = blockIdx.x / tiles;
    const int tile = (int)(blockIdx.x - j * tiles), rt = tile / a.dtiles, g = tile - rt * a.dtiles;
    Segment seg;
    if (!find_segment(a, a.first + j, seg)) return;        // the whole workgroup
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wy = wave / WX, wx = wave % WX;
    const int r0 = rt * RT, d0 = g * kGroup, l16 = lane & 15, quad = lane >> 4;
    auto yswizzle = [](int k) { return RT == 64 ? (k >> 1) & 3 : RT == 32 ? (k >> 2) & 1 : 0; };

    f32x4 acc[CM][CN];
#pragma unroll
    for (int m = 0; m < CM; ++m)
#pragma unroll
        for (int n = 0; n < CN; ++n) acc[m][n] = f32x4{0, 0, 0, 0};

    float y[PER][8];
    int8_t q[32];
    auto request = [&](int64_t t0) {
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int piece = tid + 256 * p, k = piece / (RT / 8), r = r0 + piece % (RT / 8) * 8;
            const int64_t t = t0 + k;
            const bool live = piece < PIECES && t < seg.hi;
            Eight<Y>::load((const Y *)a.dY + t * a.ldY + r, live ? a.R - r : 0, y[p]);
            const float s = live ? a.step[t * a.ldS + g] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) y[p][i] = live ? __fmul_rn(y[p][i], s) : 0.0f;
        }
        const int64_t t = t0 + (tid >> 2);
        const int c = d0 + (tid & 3) * 32, left = t < seg.hi ? a.D - c : 0;
        const int8_t *in = a.codes + t * a.ldC + c;
        if (left >= 32) __builtin_memcpy(q, in, 32);
        else
#pragma unroll
            for (int i = 0; i < 32; ++i) q[i] = i < left ? in[i] : (int8_t)0;
    };
    auto store = [&]() {
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int piece = tid + 256 * p, k = piece / (RT / 8), c = piece % (RT / 8);
            if (piece < PIECES) {
#pragma unroll
                for (int term = 0; term < TERMS; ++term) {
                    uint16_t b[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        b[i] = bf16_bits(y[p][i]);
                        y[p][i] = __fsub_rn(y[p][i], bf16_value(b[i]));       // exact
                    }
                    __builtin_memcpy(__builtin_assume_aligned(s_y + term * YPLANE + k * YROW + (((c >> 1) ^ yswizzle(k)) << 5) + ((c & 1) << 4), 16), b, 16);
                }
            }
        }
        const int k = tid >> 2;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            uint16_t b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = (uint16_t)(__float_as_uint((float)q[8 * h + i]) >> 16);
            const int c = (tid & 3) * 4 + h;
            __builtin_memcpy(__builtin_assume_aligned(s_codes + k * 256 + (((c >> 1) ^ (k & 7)) << 5) + ((c & 1) << 4), 16), b, 16);
        }
    };
    typedef __attribute__((address_space(3))) i16x4 lds16x4;
    auto column = [](const unsigned char *lo, const unsigned char *hi) {     // tokens of two times four rows
        const i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16x4 *)lo);
        const i16x4 z = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16x4 *)hi);
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, z, 0, 1, 2, 3, 4, 5, 6, 7));
    };

    if (seg.lo < seg.hi) request(seg.lo);
    for (int64_t t0 = seg.lo; t0 < seg.hi; t0 += KT) {
        __syncthreads();
        store();
        __syncthreads();
        if (t0 + KT < seg.hi) request(t0 + KT);
#pragma unroll
        for (int kk = 0; kk < KT / 32; ++kk) {
            const int k = 32 * kk + 4 * quad + (l16 >> 2), at = (l16 & 3) * 8;
            bf16x8 fm[CM], fn[TERMS][CN];
#pragma unroll
            for (int m = 0; m < CM; ++m) {
                const unsigned char *p = s_codes + k * 256 + (((wx * CM + m) ^ (k & 7)) << 5) + at;
                fm[m] = column(p, p + 16 * 256);
            }
#pragma unroll
            for (int term = 0; term < TERMS; ++term)
#pragma unroll
                for (int n = 0; n < CN; ++n) {
                    const unsigned char *p = s_y + term * YPLANE + k * YROW + (((wy * CN + n) ^ yswizzle(k)) << 5) + at;
                    fn[term][n] = column(p, p + 16 * YROW);
                }
#pragma unroll
            for (int term = TERMS - 1; term >= 0; --term)
#pragma unroll
                for (int m = 0; m < CM; ++m)
#pragma unroll
                    for (int n = 0; n < CN; ++n)
                        acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fm[m], fn[term][n], acc[m][n], 0, 0, 0);
        }
    }
    __syncthreads();                                       // everyone has read the last stage
    put_segment<Out>(a, seg, s_all + wave * 16 * (CM * 64 + 16), acc, l16, r0 + wy * CN * 16, d0 + wx * CM * 16);
}

// The same for operands whose rows are whole 16-byte chunks (or were made so).  A workgroup takes RT rows of R x GROUPS groups, a
// wavefront of it one group (or half of one); stages of 32 tokens' codes, gradients and steps are copied to a ring of NS in LDS
// without passing through registers, the next ones on their way while one is used: codes stay 8 bits wide until the transposing
// reads have brought eight tokens of a column into a lane, and the step is multiplied there, into the gradients or, for bfloat16 ones from 33
// rows on, into the codes (either product has 16 bits: two bfloat16 numbers).  Bound: memory while R is a rank of adapters (codes are read once
// for 128 rows, 64 of fp32); the vector work of a stage is 12 operations for eight numbers of one side and 40 for eight of the other (60 - 80 for
// fp32 gradients).  64 examples of 32768 tokens, 4096 columns: 42 us at R = 16 (codes alone 26); R = 64: 56 us in halves of a group per wavefront
// with the steps in the codes, a quarter more in whole groups with the steps in the gradients (and half the wavefronts' room in registers).
// fp32 gradients are read as rows of twice as many 16-bit columns: a pair of lanes holds the halves of two rows of them (eight apart), and
// exchanges two.  Their products with a step are rounded to fp32 and taken as three bfloat16 terms for fp32 results (all 24 bits), two for bfloat16 ones: R = 16, 64,
// 128 (32 examples of 16384 tokens) 46, 89, 89 us, against 62, 99, 96 without the ring.
// Rows of 128 codes are exchanged by 16-byte chunks, rows of gradients by 32-byte pieces, so that the eight (four) rows of each of two
// lane groups lie in different banks.
template <int RT, class Y> struct GradRing {
    static constexpr bool F32 = sizeof(Y) == 4;
    static constexpr int NW = 4, SPLIT = RT >= 32 ? 2 : 1, GROUPS = NW / SPLIT, KT = 32, NS = 4, CM = 8 / SPLIT, CN = RT / 16;     // SPLIT: wavefronts of a group
    static constexpr int ROW = RT * (int)sizeof(Y), CODES = GROUPS * KT * 128, YS = KT * ROW, STAGE = CODES + YS + NW * 256, LDS = NS * STAGE;
    static constexpr bool SCALE_CODES = RT >= 64 && !F32;          // the side with fewer fragments takes the steps
    static constexpr int UC = 4 / SPLIT, YQ = YS / 1024, UY = (YQ + NW - 1) / NW, U = UC + UY + 1;
    static_assert((NS - 2) * U < 64, "vmcnt is a 6-bit counter");
};
__device__ inline bf16x8 upper_halves(const float (&v)[8]) {
    union { uint32_t u[4]; bf16x8 b; } r;
#pragma unroll
    for (int h = 0; h < 4; ++h) r.u[h] = __builtin_amdgcn_perm(__float_as_uint(v[2 * h + 1]), __float_as_uint(v[2 * h]), 0x07060302u);
    return r.b;
}
// Numbers as sums of bfloat16, of eight significant bits each: two terms hold 16 bits, three all of an fp32 number.
template <int TERMS> __device__ inline void in_terms(float (&v)[8], bf16x8 (&out)[TERMS]) {
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
        out[t] = upper_halves(v);
        if (t + 1 < TERMS)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __fsub_rn(v[i], __uint_as_float(__float_as_uint(v[i]) & 0xFFFF0000u));
    }
}

template <int RT, class Y, class Out>
__global__ void __launch_bounds__(256, 2)
checkpoint_grad_ring_kernel(GradArgs a) {
    typedef GradRing<RT, Y> Sh;
    constexpr int GROUPS = Sh::GROUPS, KT = Sh::KT, NS = Sh::NS, CM = Sh::CM, CN = Sh::CN, ROW = Sh::ROW, YL = ROW / 16, YB = (int)sizeof(Y);      // YL: lanes of a row of gradients
    constexpr int TERMS = Sh::F32 && sizeof(Out) == 4 ? 3 : 2;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int64_t tiles = (int64_t)a.rtiles * a.dtiles, j = blockIdx.x / tiles;
    const int tile = (int)(blockIdx.x - j * tiles), rt = tile / a.dtiles, gt = (tile - rt * a.dtiles) * GROUPS;
    Segment seg;
    if (!find_segment(a, a.first + j, seg)) return;        // the whole workgroup
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, quad = lane >> 4;
    const unsigned lds0 = (unsigned)(uintptr_t)((__attribute__((address_space(3))) unsigned char *)smem);
    const int groups = (a.D + kGroup - 1) / kGroup, r0 = rt * RT;
    const int gl = wave / Sh::SPLIT, c0 = wave % Sh::SPLIT * 64, g = gt + gl < groups ? gt + gl : groups - 1;
    auto yswizzle = [](int k) { return ROW >= 256 ? k & 7 : ROW == 128 ? (k >> 1) & 3 : ROW == 64 ? (k >> 2) & 1 : 0; };
    auto swizzle = [](int k) { return ((k >> 1) & 3) | ((k >> 4) & 1) << 2; };

    // ---- copies: what lane and wavefront take of a stage; rows past the segment repeat its last one, bytes past a row's end its last chunk
    const int len = (int)(seg.hi - seg.lo), stages = (len + KT - 1) / KT;
    unsigned ccol[Sh::UC], ycol[Sh::UY];
    int crow[Sh::UC], yrow[Sh::UY];
#pragma unroll
    for (int u = 0; u < Sh::UC; ++u) {
        const int q = wave * Sh::UC + u;
        crow[u] = 8 * (q & 3) + (lane >> 3);
        const int at = (gt + (q >> 2)) * kGroup + ((lane & 7) ^ swizzle(crow[u])) * 16;
        ccol[u] = (unsigned)(at < a.Dc - 16 ? at : a.Dc - 16);
    }
#pragma unroll
    for (int u = 0; u < Sh::UY; ++u) {
        const int q = wave * Sh::UY + u < Sh::YQ ? wave * Sh::UY + u : Sh::YQ - 1;
        yrow[u] = q * (64 / YL) + lane / YL;
        const int at = r0 * YB + ((lane % YL) ^ (yswizzle(yrow[u]) << 1)) * 16;
        ycol[u] = (unsigned)(at < a.Rc * YB - 16 ? at : a.Rc * YB - 16);
    }
    const unsigned ldC = (unsigned)a.ldC, ldY = (unsigned)a.ldY * YB, ldS = (unsigned)a.ldS * 4;
    auto request = [&](int s, int slot) {
        if (s > stages - 1) s = stages - 1;                // repeated past the end: all stages count alike
        const int64_t t = seg.lo + (int64_t)s * KT;
        const int last = len - s * KT - 1;                 // row
        const unsigned at = lds0 + (unsigned)(slot * Sh::STAGE);
        const unsigned char *c = (const unsigned char *)a.codes + t * a.ldC, *y = (const unsigned char *)a.dY + t * a.ldY * YB;
#pragma unroll
        for (int u = 0; u < Sh::UC; ++u) global_to_lds16(c, (unsigned)(crow[u] < last ? crow[u] : last) * ldC + ccol[u], at + (unsigned)((wave * Sh::UC + u) * 1024));
#pragma unroll
        for (int u = 0; u < Sh::UY; ++u) {
            const int q = wave * Sh::UY + u < Sh::YQ ? wave * Sh::UY + u : Sh::YQ - 1;
            global_to_lds16(y, (unsigned)(yrow[u] < last ? yrow[u] : last) * ldY + ycol[u], at + (unsigned)(Sh::CODES + q * 1024));
        }
        const int row = lane & 31;
        global_to_lds4(a.step + t * a.ldS + g, (unsigned)(row < last ? row : last) * ldS, at + (unsigned)(Sh::CODES + Sh::YS + wave * 256));
    };

    // ---- operands: a lane's eight tokens are 4 quad .. + 3 and 16 + 4 quad .. + 3
    const int krow = (l16 >> 1) < 4 ? 4 * quad + (l16 >> 1) : 12 + 4 * quad + (l16 >> 1);
    const unsigned c_lane = (unsigned)(gl * KT * 128 + krow * 128 + (((swizzle(krow) ^ (c0 >> 4)) << 4) | (l16 & 1) << 3));
    const int yk = 4 * quad + (l16 >> 2);
    const unsigned y_lane = (unsigned)(Sh::CODES + yk * ROW + (yswizzle(yk) << 5) + (l16 & 3) * 8);
    const unsigned s_lane = (unsigned)(Sh::CODES + Sh::YS + wave * 256 + quad * 16);
    typedef __attribute__((address_space(3))) i16x4 lds16x4;
    typedef __attribute__((ext_vector_type(2))) int i32x2;
    typedef __attribute__((address_space(3))) i32x2 lds32x2;

    typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
    const bool odd = lane & 1;

    f32x4 acc[CM][CN];
#pragma unroll
    for (int m = 0; m < CM; ++m)
#pragma unroll
        for (int n = 0; n < CN; ++n) acc[m][n] = f32x4{0, 0, 0, 0};
    if (stages > 0) {
#pragma unroll
        for (int i = 0; i < NS - 1; ++i) request(i, i);
        int slot = 0;
        for (int s = 0; s < stages; ++s) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            wait_vmcnt<(NS - 2) * Sh::U>();                // this wavefront's share of the stage has landed
            __builtin_amdgcn_s_barrier();                  // everyone's; and everyone has read the slot that is requested next
            asm volatile("" ::: "memory");
            request(s + NS - 1, slot == 0 ? NS - 1 : slot - 1);
            const unsigned char *st = smem + slot * Sh::STAGE;
            float w[8];
            const f32x4 w0 = *(const f32x4 *)(st + s_lane), w1 = *(const f32x4 *)(st + s_lane + 64);
            const int left = len - s * KT;
#pragma unroll
            for (int i = 0; i < 4; ++i) { w[i] = w0[i]; w[4 + i] = w1[i]; }
            if (left < KT) {                               // the last stage: tokens past the segment weigh nothing
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = 4 * quad + i < left ? w[i] : 0.0f;
                    w[4 + i] = 16 + 4 * quad + i < left ? w[4 + i] : 0.0f;
                }
            }
            auto column = [&](int piece) {                 // eight tokens of one of 16 columns of 16 bits
                const unsigned char *p = st + (y_lane ^ (unsigned)(piece << 5));
                const i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16x4 *)p);
                const i16x4 z = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16x4 *)(p + 16 * ROW));
                return __builtin_shufflevector(x, z, 0, 1, 2, 3, 4, 5, 6, 7);
            };
            auto codes_of = [&](int m, float (&v)[8]) {
                const i32x2 b = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds32x2 *)(st + (c_lane ^ (unsigned)(m << 4))));
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const int x = b[h >> 1] >> (16 * (h & 1));
                    v[2 * h] = (float)(int8_t)x;
                    v[2 * h + 1] = (float)(int8_t)(x >> 8);
                }
            };
            float v[8];
            if (Sh::SCALE_CODES) {
                bf16x8 fy[CN], fc[2];
#pragma unroll
                for (int n = 0; n < CN; ++n) fy[n] = __builtin_bit_cast(bf16x8, column(n));
#pragma unroll
                for (int m = 0; m < CM; ++m) {
                    codes_of(m, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], w[i]);
                    in_terms(v, fc);
#pragma unroll
                    for (int term = 1; term >= 0; --term)
#pragma unroll
                        for (int n = 0; n < CN; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fc[term], fy[n], acc[m][n], 0, 0, 0);
                }
            } else {
                bf16x8 fc[CM], fy[TERMS];
#pragma unroll
                for (int m = 0; m < CM; ++m) {
                    codes_of(m, v);
                    fc[m] = upper_halves(v);
                }
#pragma unroll
                for (int n = 0; n < CN; ++n) {
                    if (Sh::F32) {
                        const u32x4 x = __builtin_bit_cast(u32x4, column(2 * n)), z = __builtin_bit_cast(u32x4, column(2 * n + 1));
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            const unsigned keep = odd ? z[h] : x[h], give = odd ? x[h] : z[h];
                            const unsigned got = (unsigned)__builtin_amdgcn_update_dpp(0, (int)give, 0xB1, 0xF, 0xF, false);
                            v[2 * h] = __uint_as_float(__builtin_amdgcn_perm(keep, got, odd ? 0x05040100u : 0x01000504u));
                            v[2 * h + 1] = __uint_as_float(__builtin_amdgcn_perm(keep, got, odd ? 0x07060302u : 0x03020706u));
                        }
                    } else {
                        const bf16x8 x = __builtin_bit_cast(bf16x8, column(n));
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], w[i]);
                    in_terms(v, fy);
#pragma unroll
                    for (int term = TERMS - 1; term >= 0; --term)
#pragma unroll
                        for (int m = 0; m < CM; ++m) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fc[m], fy[term], acc[m][n], 0, 0, 0);
                }
            }
            slot = slot + 1 == NS ? 0 : slot + 1;
        }
        wait_vmcnt<0>();                                   // no copy is under way when the workgroup gives its LDS back
    }
    __syncthreads();                                       // everyone has read the last stage
    if (gt + gl >= groups) return;
    put_segment<Out>(a, seg, smem + wave * 16 * (CM * 64 + 16), acc, Sh::F32 ? (l16 >> 1) + 8 * (l16 & 1) : l16, r0, g * kGroup + c0);
}

// Rows of `cols` elements copied to rows of ld (whole 16-byte chunks) with zeros behind them, a chunk a thread.
template <class T>
__global__ void __launch_bounds__(256)
checkpoint_pack_kernel(const T *in, int64_t ld_in, int64_t rows, int32_t cols, T *out, int32_t ld) {
    constexpr int E = 16 / sizeof(T);
    const int chunks = ld / E;
    const int64_t first = (int64_t)blockIdx.x * 256, r0 = first / chunks;
    const unsigned at = (unsigned)(first - r0 * chunks) + threadIdx.x, up = at / (unsigned)chunks;
    const int64_t r = r0 + up;
    const int c = (int)(at - up * (unsigned)chunks) * E;
    if (r >= rows) return;
    T x[E];
    const T *from = in + r * ld_in + c;
    if (c + E <= cols) __builtin_memcpy(x, from, 16);
    else
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = c + i < cols ? from[i] : (T)0;
    __builtin_memcpy(__builtin_assume_aligned(out + r * ld + c, 16), x, 16);
}
template <class T>
static void launch_pack(const T *in, int64_t ld_in, int64_t rows, int32_t cols, T *out, int32_t ld, hipStream_t st) {
    const int64_t chunks = ld / (16 / (int)sizeof(T)), most = kMostThreads / chunks;
    for (int64_t r = 0; r < rows; r += most) {
        const int64_t n = rows - r < most ? rows - r : most;
        hipLaunchKernelGGL(checkpoint_pack_kernel<T>, dim3((unsigned)((n * chunks + 255) / 256)), dim3(256), 0, st, in + r * ld_in, ld_in, n, cols, out + r * ld, ld);
    }
}

// The planes of the examples of more than one segment, added in the order of their tokens.
template <class Out, int W>
__global__ void __launch_bounds__(256)
checkpoint_join_kernel(GradArgs a) {
    const int64_t e = blockIdx.y, size = (int64_t)a.R * a.D, length = offset_at(a, e + 1) - offset_at(a, e);
    if (length <= a.chunk) return;
    const int64_t p0 = phi(a, e, a.chunk);
    int64_t p1 = p0 + (length + a.chunk - 1) / a.chunk;
    if (p1 > a.segments) p1 = a.segments;
    typedef __attribute__((ext_vector_type(W))) float fw;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * W; i < size; i += (int64_t)gridDim.x * 256 * W) {
        fw s = *(const fw *)(a.planes + p0 * size + i);
#pragma unroll 4
        for (int64_t p = p0 + 1; p < p1; ++p) s += *(const fw *)(a.planes + p * size + i);
        Out x[W];
#pragma unroll
        for (int u = 0; u < W; ++u) x[u] = sizeof(Out) == 2 ? (Out)bf16_bits(((const float *)&s)[u]) : (Out)((const float *)&s)[u];
        __builtin_memcpy((Out *)a.G + e * a.ldG + i, x, sizeof x);
    }
}

// ---- Many rows of R (a layer's own weights) with bfloat16 results: the products are the bound, so that the activations are formed once, as
// bfloat16 rows of tokens, rounded once, and the tiles of product.h multiply them with the gradients.  (With fp32 results both terms of an activation would
// enter: 1 x 8192 tokens, R = D = 4096 450 us, the ring 418.  The rounding takes the results' error (2-norm, relative) from 0.0017, what their own
// rounding leaves, to 0.0023; the ring, which does not round, would take 420 us for 240.)
// Workgroups take 64 tokens of an example (the last ones of it with zeros behind them): block e + offset[e] / 64 and on.
__global__ void __launch_bounds__(256)
checkpoint_expand_kernel(GradArgs a, uint16_t *out, int64_t ld) {
    int64_t o0, o1;
    const int64_t j = blockIdx.x, e = find_example(a, j, 64, o0, o1);
    if (e < 0) return;
    const int64_t t0 = o0 + 64 * (j - (e + o0 / 64));
    out += j * 64 * ld;
    for (int64_t i = (int64_t)blockIdx.y * 256 + threadIdx.x; i < 64 * (ld / 8); i += (int64_t)gridDim.y * 256) {
        const int64_t r = i / (ld / 8), c = (i - r * (ld / 8)) * 8, t = t0 + r, left = t < o1 ? a.D - c : 0;
        const int8_t *in = a.codes + t * a.ldC + c;
        int8_t q[8];
        if (left >= 8) __builtin_memcpy(q, in, 8);
        else
#pragma unroll
            for (int u = 0; u < 8; ++u) q[u] = u < left ? in[u] : (int8_t)0;
        const float s = left > 0 ? a.step[t * a.ldS + c / kGroup] : 0.0f;
        float x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = __fmul_rn((float)q[u], s);
        Eight<uint16_t>::store(out + r * ld + c, 8, x);
    }
}
// rows m are columns of G, columns n its rows, the part of K its example
struct GradStore {
    struct Args { uint16_t *G; int64_t ldG; int32_t R, D; };
    template <int FM, int FN>
    static __device__ inline void run(const Args &a, unsigned char *lds, f32x16 (&acc)[FM][FN], int64_t m, int64_t n, int e, int64_t) {
        by_rows<FM, FN>(lds, acc, [&](int r, int c, f32x4 y) {
            const int64_t d = m + c;
            if (n + r >= a.R) return;
            uint16_t x[4], *out = a.G + e * a.ldG + (n + r) * a.D + d;
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = bf16_bits(y[u]);
            if (d + 4 <= a.D) __builtin_memcpy(out, x, sizeof x);
            else
#pragma unroll
                for (int u = 0; u < 4; ++u) if (d + u < a.D) out[u] = x[u];
        });
    }
};
typedef ProductShape<256, 256, 2, 4, 2> GradTile;

static int64_t expand_ld(int32_t D) { return ((int64_t)D + 7) / 8 * 8; }
// Rows of R and examples that fill the chip with tiles (whole examples: with several of different lengths twice as well), of tokens enough that padding them to 64 costs
// little.  16 x 32768 tokens, R = 2048, D = 1024 163 us, by the ring 225; 8 x 65536, R = D = 1024 487 and 252; 64 x 16384, R = 300, D = 2048 99 and 69.
static bool many_rows(int64_t T, int64_t n, int32_t R, int32_t D) {
    return R >= 1024 && T >= 128 * n && n * ((R + 255) / 256) * ((D + 255) / 256) >= (n == 1 ? compute_units() / 2 : compute_units());
}
static bool expand_fits(int64_t T, int64_t n, int32_t D) { return launchable(n + T / 64, 256) && expand_ld(D) < (1 << 22); }      // (the product's rows of it, too)
static size_t expand_bytes(int64_t T, int64_t n, int32_t D) { return (size_t)(n + T / 64) * 64 * (size_t)expand_ld(D) * 2; }

static qless_status launch_many(const GradArgs &a, hipStream_t st) {
    uint16_t *x = (uint16_t *)a.planes;
    const int64_t ld = expand_ld(a.D), blocks = a.n + a.T / 64;
    const ProductArgs p{ProductOperand{x, ld * 2, ld * 2, blocks * 64}, ProductOperand{a.dY, a.ldY * 2, (int64_t)a.Rc * 2, 0},
                        a.R, a.T, nullptr, nullptr, (a.D + 255) / 256, (int32_t)a.n, a.offsets, nullptr, 0, 0};
    hipLaunchKernelGGL(checkpoint_expand_kernel, dim3((unsigned)blocks, (unsigned)((ld + 127) / 128)), dim3(256), 0, st, a, x, ld);
    const qless_status rc = launch_product<GradTile, ACROSS, ACROSS, GradStore, true>(p, GradStore::Args{(uint16_t *)a.G, a.ldG, a.R, a.D}, st);
    return rc == QLESS_OK ? launch_status() : rc;
}

// Tokens of a segment.  32 tokens take a workgroup about half a microsecond, a plane the whole memory 8 R D bytes' time.  Where the
// examples do not fill the two workgroups of each compute unit, they are cut into as many segments as do, or at which one more of
// each would cost by its plane what it saves (1 x 8192 tokens, R = D = 1024 in one piece 262 us, in six 52, in twelve 58; 16 x 512,
// R = 64, D = 4096 in whole examples 35, in four 42); where they do, into what each of those has to do if all were alike: the longest
// example would keep few of them busy for long (rank 16, 64 ragged examples of 32768 tokens 64 us in segments of 2048, 48 of
// 512, 52 of 256), but none so short that its plane costs more than its codes.
static int64_t grad_chunk(int64_t T, int64_t n, int32_t R, int32_t D) {
    const int64_t tiles = ((R + 127) / 128) * ((D + 4 * kGroup - 1) / (4 * kGroup)) * (R > 16 ? 2 : 1), slots = 2 * (int64_t)compute_units();
    const int64_t mean = T / n + 1;
    int64_t chunk;
    if (n * tiles < slots) {
        const double segments = fmin((double)slots / (double)(n * tiles), sqrt((double)mean * 0.8e5 / (8.0 * R * D * (double)n)));
        chunk = segments < 0.5 ? 2 * mean : segments < 1.0 ? mean : (int64_t)((double)mean / segments) + 1;
    } else {
        chunk = T * tiles / slots;
        if (chunk < 8 * (int64_t)R) chunk = 8 * (int64_t)R;
    }
    if (chunk < 128) chunk = 128;
    if (chunk >= T) chunk = T + 1;
    return (chunk + 63) / 64 * 64;
}
static size_t up16(size_t bytes) { return (bytes + 15) & ~(size_t)15; }
// Rows that are no whole chunks may be packed into the workspace: gradients first, then codes.  (By their length alone, as the workspace is asked for without
// the operands: rows of whole chunks that begin elsewhere are read as they lie.  8192 tokens of 4096 x 4096, dY one column into its rows: 1120 us, not 260;
// 32768 of 16 x 4096 68, not 61.)  Both take a launch,
// and codes as long as a product of 64 rows, so that they are packed for more rows only, and where fp32 gradients do not make the vector work the
// bound (R = 100, bfloat16: 64 x 65536 tokens, D = 4095 288 us packed, 394 read as they lie; 32 x 32000, D = 1333 65 and 74; 8 x 4000 33 and 31.  fp32 gradients, 32 x 32000: 91 and
// 76.  R = 16, 64 x 65536, D = 1001: 55 and 44.  Gradients alone, D = 4096: 64 x 65536, R = 100 160 and 326; 16 x 16000, R = 6
// 28 and 31; 16 x 4000 18.5 and 17.5).
static bool worth_packing(int64_t T, int64_t n, int32_t R, int32_t D) { return T >= 20000000 / D || many_rows(T, n, R, D); }
static int32_t packed_R(int32_t R, int bytes) { return (int32_t)up16((size_t)R * bytes) / bytes; }
static int32_t packed_D(int32_t D) { return (D + 15) / 16 * 16; }
static size_t packed_bytes(int64_t T, int64_t n, int32_t R, int32_t D) {
    if (!worth_packing(T, n, R, D)) return 0;
    const size_t y2 = R % 8 ? (size_t)T * packed_R(R, 2) * 2 : 0, y4 = R % 4 ? (size_t)T * packed_R(R, 4) * 4 : 0;
    return (y2 > y4 ? y2 : y4) + (D % 16 && R > 64 ? (size_t)T * packed_D(D) : 0);      // (codes for bfloat16 gradients only)
}
static int64_t grad_segments(int64_t T, int64_t n, int64_t chunk) { return n + T / chunk; }

template <class Out>
static void launch_join(const GradArgs &a, hipStream_t st) {
    if (a.segments <= a.n) return;
    const int64_t size = (int64_t)a.R * a.D;
    int64_t bx = (size + 1023) / 1024;
    const int64_t most = a.n <= 8 ? 1024 : a.n < 64 ? 8192 / a.n : 128;   // few of many examples have parts
    if (bx > most) bx = most;
    if (size % 4 == 0) hipLaunchKernelGGL((checkpoint_join_kernel<Out, 4>), dim3((unsigned)bx, (unsigned)a.n), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((checkpoint_join_kernel<Out, 1>), dim3((unsigned)bx, (unsigned)a.n), dim3(256), 0, st, a);
}
// As many segments at a time as a launch takes.
template <class Out, class Launch>
static qless_status launch_segments(GradArgs &a, hipStream_t st, Launch launch) {
    const int64_t tiles = (int64_t)a.rtiles * a.dtiles, most = kMostThreads / 256 / tiles;
    for (a.first = 0; a.first < a.segments; a.first += most) launch((unsigned)((a.segments - a.first < most ? a.segments - a.first : most) * tiles));
    launch_join<Out>(a, st);
    return launch_status();
}
template <int RT, class Y, int TERMS, class Out>
static qless_status launch_grad(GradArgs a, hipStream_t st) {
    a.rtiles = (a.R + RT - 1) / RT;
    a.dtiles = (a.D + kGroup - 1) / kGroup;
    return launch_segments<Out>(a, st, [&](unsigned grid) { hipLaunchKernelGGL((checkpoint_grad_kernel<RT, Y, TERMS, Out>), dim3(grid), dim3(256), 0, st, a); });
}
template <int RT, class Y, class Out>
static qless_status launch_ring(GradArgs a, hipStream_t st) {
    typedef GradRing<RT, Y> Ring;
    QLESS_LDS_KERNEL((checkpoint_grad_ring_kernel<RT, Y, Out>), Ring::LDS);
    a.rtiles = (a.R + RT - 1) / RT;
    a.dtiles = (a.D + kGroup * Ring::GROUPS - 1) / (kGroup * Ring::GROUPS);
    return launch_segments<Out>(a, st, [&](unsigned grid) { hipLaunchKernelGGL((checkpoint_grad_ring_kernel<RT, Y, Out>), dim3(grid), dim3(64 * Ring::NW), Ring::LDS, st, a); });
}
template <class Y, class Out>
static qless_status launch_ring_rows(const GradArgs &a, hipStream_t st) {
    if (a.R <= 16) return launch_ring<16, Y, Out>(a, st);
    if (a.R <= 32) return launch_ring<32, Y, Out>(a, st);
    if (a.R <= 64) return launch_ring<64, Y, Out>(a, st);
    if constexpr (sizeof(Y) == 4) return launch_ring<64, Y, Out>(a, st);      // (R = 256, D = 2048: 158 us, with 128 rows 166)
    else return launch_ring<128, Y, Out>(a, st);
}
template <class Y, int TERMS, class Out>
static qless_status launch_grad_rows(const GradArgs &a, hipStream_t st) {
    if (a.R <= 16) return launch_grad<16, Y, TERMS, Out>(a, st);
    if (a.R <= 32) return launch_grad<32, Y, TERMS, Out>(a, st);
    return launch_grad<64, Y, TERMS, Out>(a, st);
}

static bool checkpoint_shape_ok(int64_t T, int32_t D, int64_t ldX, int64_t ldC, int64_t ldS) {
    return T >= 0 && D >= 1 && (T <= 1 || (ldX >= D && ldC >= D && ldS >= (D + (int64_t)kGroup - 1) / kGroup));
}
// Rows of a launch, and its workgroups.
static int64_t checkpoint_rows(int64_t T, int32_t groups) {
    const int64_t most = kMostThreads / 256 * kItems / groups;
    return T < most ? T : most;
}
static unsigned checkpoint_grid(int64_t rows, int32_t groups) { return (unsigned)((rows * groups + kItems - 1) / kItems); }
// The sizes of a gradient: rows and columns that 32 bits count, an example's tiles in a launch, tensors of at most 2^40 numbers.
static bool grad_sizes_ok(int64_t T, int32_t R, int32_t D) {
    const int64_t most = (int64_t)1 << 40;
    return R <= 1 << 30 && D <= 1 << 30 && (int64_t)((R + 63) / 64) * ((D + kGroup - 1) / kGroup) <= kMostThreads / 256 && T <= most / R && T <= most / D;
}

}  // namespace qless

extern "C" qless_status qless_checkpoint8(const void *X, qless_dtype dt, int64_t T, int32_t D, int64_t ldX, int8_t *codes, int64_t ldC,
                                          float *step, int64_t ldS, void *stream) {
    using namespace qless;
    if (!checkpoint_shape_ok(T, D, ldX, ldC, ldS)) return QLESS_ERR_INVALID_ARG;
    if (dt != QLESS_F32 && dt != QLESS_BF16) return QLESS_ERR_UNSUPPORTED;
    if (T == 0) return QLESS_OK;
    if (!X || !codes || !step) return QLESS_ERR_INVALID_ARG;
    const int32_t groups = (int32_t)((D + (int64_t)kGroup - 1) / kGroup);
    if (T > ((int64_t)1 << 40) / groups) return QLESS_ERR_UNSUPPORTED;
    const hipStream_t st = (hipStream_t)stream;
    const int64_t rows = checkpoint_rows(T, groups);
    for (int64_t t = 0; t < T; t += rows) {
        const int64_t n = T - t < rows ? T - t : rows;
        auto write = [&](auto kernel, auto *x) {
            hipLaunchKernelGGL(kernel, dim3(checkpoint_grid(n, groups)), dim3(256), 0, st, x + t * ldX, n, D, ldX, groups, codes + t * ldC, ldC, step + t * ldS, ldS);
        };
        if (dt == QLESS_F32) write(checkpoint_write_kernel<float>, (const float *)X);
        else write(checkpoint_write_kernel<uint16_t>, (const uint16_t *)X);
    }
    return launch_status();
}

extern "C" qless_status qless_checkpoint8_read(const int8_t *codes, int64_t ldC, const float *step, int64_t ldS, int64_t T, int32_t D,
                                               void *X, qless_dtype dt, int64_t ldX, void *stream) {
    using namespace qless;
    if (!checkpoint_shape_ok(T, D, ldX, ldC, ldS)) return QLESS_ERR_INVALID_ARG;
    if (dt != QLESS_F32 && dt != QLESS_BF16) return QLESS_ERR_UNSUPPORTED;
    if (T == 0) return QLESS_OK;
    if (!X || !codes || !step) return QLESS_ERR_INVALID_ARG;
    const int32_t groups = (int32_t)((D + (int64_t)kGroup - 1) / kGroup);
    if (T > ((int64_t)1 << 40) / groups) return QLESS_ERR_UNSUPPORTED;
    const hipStream_t st = (hipStream_t)stream;
    const int64_t rows = checkpoint_rows(T, groups);
    for (int64_t t = 0; t < T; t += rows) {
        const int64_t n = T - t < rows ? T - t : rows;
        auto read = [&](auto kernel, auto *x) {
            hipLaunchKernelGGL(kernel, dim3(checkpoint_grid(n, groups)), dim3(256), 0, st, codes + t * ldC, ldC, step + t * ldS, ldS, n, D, groups, x + t * ldX, ldX);
        };
        if (dt == QLESS_F32) read(checkpoint_read_kernel<float>, (float *)X);
        else read(checkpoint_read_kernel<uint16_t>, (uint16_t *)X);
    }
    return launch_status();
}

extern "C" size_t qless_checkpoint8_grad_workspace(int64_t T, int64_t n, int32_t R, int32_t D) {
    using namespace qless;
    if (T < 0 || n < 1 || R < 1 || D < 1 || !grad_sizes_ok(T, R, D)) return 0;
    const int64_t segments = grad_segments(T, n, grad_chunk(T, n, R, D));
    const size_t planes = segments > n ? (size_t)segments * (size_t)R * (size_t)D * 4 : 0, rows = many_rows(T, n, R, D) ? expand_bytes(T, n, D) : 0;
    return up16((planes > rows ? planes : rows)) + packed_bytes(T, n, R, D);
}

extern "C" qless_status qless_checkpoint8_grad(const void *dY, qless_dtype dtY, int64_t ldY, int32_t R, const int8_t *codes, int64_t ldC,
                                               const float *step, int64_t ldS, int32_t D, int64_t T, const int64_t *offsets, int64_t n,
                                               void *G, qless_dtype dtG, int64_t ldG, void *ws, size_t ws_bytes, void *stream) {
    using namespace qless;
    if (R < 1 || n < 0 || !checkpoint_shape_ok(T, D, D, ldC, ldS) || (T > 1 && ldY < R)) return QLESS_ERR_INVALID_ARG;
    if ((dtY != QLESS_F32 && dtY != QLESS_BF16) || (dtG != QLESS_F32 && dtG != QLESS_BF16)) return QLESS_ERR_UNSUPPORTED;
    if (n > 65535 || !grad_sizes_ok(T, R, D)) return QLESS_ERR_UNSUPPORTED;
    if (n > 1 && ldG < (int64_t)R * D) return QLESS_ERR_INVALID_ARG;
    if (n == 0) return QLESS_OK;
    if (!offsets || !G || (T > 0 && (!dY || !codes || !step))) return QLESS_ERR_INVALID_ARG;
    if (T <= 1) { ldY = R; ldC = D; ldS = (D + kGroup - 1) / kGroup; }
    GradArgs a{dY, ldY, codes, ldC, step, ldS, offsets, n, T, grad_chunk(T, n, R, D), 0, 0, R, D, 0, 0, R, D, G, ldG, (float *)ws};
    a.segments = grad_segments(T, n, a.chunk);
    const size_t need = qless_checkpoint8_grad_workspace(T, n, R, D);
    if (need > 0 && (!ws || ws_bytes < need || ((uintptr_t)ws & 15) != 0)) return QLESS_ERR_WORKSPACE;
    const qless_status ready = device_ready();
    if (ready != QLESS_OK) return ready;
    const hipStream_t st = (hipStream_t)stream;
    const int bytes = dtY == QLESS_BF16 ? 2 : 4, rc = packed_R(R, bytes);
    if (T > 0 && T <= 0x3FFFFFFF) {
        unsigned char *pack = (unsigned char *)ws + (need - packed_bytes(T, n, R, D));
        const bool many = dtY == QLESS_BF16 && dtG == QLESS_BF16 && expand_fits(T, n, D) && many_rows(T, n, R, D);
        if (rc != R && worth_packing(T, n, R, D)) {
            if (bytes == 2) launch_pack((const uint16_t *)dY, ldY, T, R, (uint16_t *)pack, rc, st);
            else launch_pack((const float *)dY, ldY, T, R, (float *)pack, rc, st);
            a.dY = pack; a.ldY = a.Rc = rc;
            pack += (size_t)T * rc * bytes;
        }
        if (dtY == QLESS_BF16 && D % 16 != 0 && R > 64 && !many && worth_packing(T, n, R, D)) {
            a.Dc = packed_D(D);
            launch_pack(codes, ldC, T, D, (int8_t *)pack, a.Dc, st);
            a.codes = (const int8_t *)pack; a.ldC = a.Dc;
        }
        // 16-byte copies and 32-bit offsets
        const bool whole_y = a.Rc == rc && (T == 1 || a.ldY * bytes % 16 == 0) && ((uintptr_t)a.dY & 15) == 0 && a.ldY < (1 << 22);
        if (whole_y && many) return launch_many(a, st);
        if (whole_y && a.Dc % 16 == 0 && (T == 1 || a.ldC % 16 == 0) && ((uintptr_t)a.codes & 15) == 0 && a.ldC < (1 << 24) && ldS < (1 << 24)) {
            if (dtY == QLESS_BF16) return dtG == QLESS_BF16 ? launch_ring_rows<uint16_t, uint16_t>(a, st) : launch_ring_rows<uint16_t, float>(a, st);
            return dtG == QLESS_BF16 ? launch_ring_rows<float, uint16_t>(a, st) : launch_ring_rows<float, float>(a, st);
        }
    }
    if (dtY == QLESS_BF16) return dtG == QLESS_BF16 ? launch_grad_rows<uint16_t, 2, uint16_t>(a, st) : launch_grad_rows<uint16_t, 2, float>(a, st);
    return dtG == QLESS_BF16 ? launch_grad_rows<float, 2, uint16_t>(a, st) : launch_grad_rows<float, 3, float>(a, st);
}
