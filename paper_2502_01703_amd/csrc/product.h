// Tiles of matrix products C[m][n] = sum_k A(m, k) B(n, k) of bfloat16 operands with fp32 sums, for the kernels whose epilogues are
// more than a store.  An operand lies in memory by rows of K (ALONG: K contiguous, one row per m or n) or by rows of m or n (ACROSS: one
// row per k); ACROSS operands are transposed by the LDS reads, so that neither form is ever rewritten in memory.
//
// A stage is 64 steps of K.  ALONG tiles lie in LDS as rows of 128 bytes, their eight 16-byte chunks exchanged by the row's bits 1 - 3
// (16 rows read together use all banks); ACROSS tiles as 64 rows of the tile's width, their 64-byte pieces exchanged by the row's
// bits 0 - 1 (the four rows that 32 lanes read together use all banks).  The stages are copied to LDS without passing through registers.
#pragma once
#include "common.h"

namespace qless {

typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

enum { ALONG = 0, ACROSS = 1 };

struct ProductOperand {
    const void *base;          // 16-byte aligned
    int64_t ld;                // bytes from row to row, a multiple of 16, below 2^23
    int64_t extent;            // ALONG: rows that exist; ACROSS: bytes of a row that exist, a multiple of 16
    int64_t depth;             // ALONG: bytes of a row that exist, a multiple of 16; ACROSS: rows that exist (below 2^31)
};
// What is read outside is replaced by what lies next to it inside: m and n past the extents give numbers that the epilogue leaves out;
// where K ends inside a stage, one of the two operands has to hold zeros up to the stage's end.
struct ProductArgs {
    ProductOperand a, b;
    int64_t n;                 // columns of C
    int64_t k;                 // steps of K
    const int32_t *live_n, *live_k;   // device: fewer of them, or null (k rounded up to a stage: the operands are zero there)
    int32_t mtiles, splits;    // splits: K in as many parts of whole stages
    // CUTS: part e of K is the rows [cuts[e], cuts[e + 1]) of b (device; clamped to 0 .. k), its stages in a begin at stage
    // e + cuts[e] / 64, and are zeros behind the part's rows.
    const int64_t *cuts;
    // SHIFT: b holds numbers that are not negative, and b(n, k) is to be multiplied by a power of two for each n and each 64 << shift_stages
    // steps of K: shift[k / (64 << shift_stages)][n] takes it off the exponents of two such numbers at once (bits 7 on of each half), down
    // to 0.  n up to whole tiles is read.
    const uint32_t *shift; int64_t shift_ld; int32_t shift_stages;
};

template <int KIND, int EXT, int NW> struct ProductCopies {
    static constexpr int BYTES = EXT * 128, Q = EXT / 8, U = (Q + NW - 1) / NW;     // copies of 1 KB, per wavefront
    const unsigned char *base;
    int ld, short_stage, left_there;                       // the stage that K ends in, if it is not whole, and what it holds
    unsigned off[U];
    __device__ inline void init(const ProductOperand &op, int first, int lane, int wave) {
        constexpr int WHOLE = KIND == ALONG ? 128 : 64;
        ld = (int)op.ld;
        left_there = (int)op.depth % WHOLE;
        short_stage = left_there ? (int)op.depth / WHOLE : -1;
        // (a tile that lies outside altogether reads the last row, or chunk)
        const int64_t end = KIND == ALONG ? op.extent - 1 : op.extent / 2 - 8, at = first < end ? first : end;
        base = (const unsigned char *)op.base + (KIND == ALONG ? at * ld : at * 2);
        const int64_t there = KIND == ALONG ? end - at : (end - at) * 2;       // of rows, or of a row's bytes
        const int left = there < 65536 ? (int)there : 65536;   // more than a tile
#pragma unroll
        for (int u = 0; u < U; ++u) {
            int row, chunk;
            place(u, lane, wave, row, chunk);
            off[u] = KIND == ALONG ? (unsigned)((row < left ? row : left) * ld) + chunk : (unsigned)(row * ld) + (unsigned)(chunk < left ? chunk : left);
        }
    }
    static __device__ inline void place(int u, int lane, int wave, int &row, int &chunk) {
        int q = wave * U + u;
        if (Q % (NW * U) != 0 && q > Q - 1) q = Q - 1;     // repeats the last copy: all wavefronts count alike
        if (KIND == ALONG) {
            row = 8 * q + (lane >> 3);
            chunk = ((lane & 7) ^ ((row >> 1) & 7)) * 16;
        } else {
            constexpr int LANES = EXT / 8;                 // of a row
            row = q * (64 / LANES) + lane / LANES;
            chunk = ((lane % LANES) ^ ((row & 3) << 2)) * 16;
        }
    }
    // copy u of stage s to its place in the stage at `lds`
    __device__ inline void issue(int u, int s, int lane, int wave, unsigned lds) const {
        int q = wave * U + u;
        if (Q % (NW * U) != 0 && q > Q - 1) q = Q - 1;
        const unsigned char *from = base + (KIND == ALONG ? (int64_t)s * 128 : (int64_t)s * 64 * ld);
        unsigned at = off[u];
        if (s == short_stage) {                            // the same for all lanes
            const int left = left_there;
            int row, chunk;
            place(u, lane, wave, row, chunk);
            if (KIND == ALONG) at -= (unsigned)(chunk < left ? 0 : chunk - (left - 16));
            else at -= (unsigned)((row < left ? 0 : row - (left - 1)) * ld);
        }
        global_to_lds16(from, at, lds + (unsigned)(q * 1024));
    }
};

// A fragment: for 32 rows of the tile from `first` on (a multiple of 32), eight steps of K per lane.
template <int KIND, int EXT>
__device__ inline unsigned fragment_lane(int lane) {
    const int half = lane >> 5, l32 = lane & 31, l16 = lane & 15;
    if (KIND == ALONG) return (unsigned)(l32 * 128 + ((half ^ ((l32 >> 1) & 7)) << 4));
    const int row = 8 * half + (l16 >> 2);
    return (unsigned)(row * EXT * 2 + (l16 >> 2) * 64 + ((lane >> 4) & 1) * 32 + (l16 & 3) * 8);
}
template <int KIND, int EXT>
__device__ inline bf16x8 fragment(const unsigned char *stage, unsigned lane_at, int first, int kk) {
    if (KIND == ALONG) return *(const bf16x8 *)(stage + first * 128 + (lane_at ^ (unsigned)(kk << 5)));
    typedef __attribute__((address_space(3))) i16x4 lds16x4;
    const unsigned char *p = stage + kk * (16 * EXT * 2) + (lane_at ^ (unsigned)(first * 2));
    const i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16x4 *)p);
    const i16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16x4 *)(p + 4 * EXT * 2));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
}

// MT x NT tiles by WY x WX wavefronts with FM x FN accumulators of 32 x 32 each, NS stages in LDS.
template <int MT_, int NT_, int WY_, int WX_, int NS_> struct ProductShape {
    static constexpr int MT = MT_, NT = NT_, WY = WY_, WX = WX_, NS = NS_, NW = WY * WX, FM = MT / WY / 32, FN = NT / WX / 32;
    static constexpr int STAGE = (MT + NT) * 128, LDS = NS * STAGE;
    static_assert(FM * WY * 32 == MT && FN * WX * 32 == NT && NS >= 2 && NW * FM * 4096 <= LDS, "whole fragments, and room for 32 rows of them");
};

// Eight bfloat16 numbers that are not negative, each divided by the same power of two, to 0 if it is too great: a saturating subtraction
// in the exponent field of two at a time.
__device__ inline bf16x8 lower_exponents(bf16x8 x, uint32_t by) {
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    union { bf16x8 v; u16x2 u[4]; } r;
    r.v = x;
    const u16x2 b = __builtin_bit_cast(u16x2, by);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.u[i] = __builtin_elementwise_sub_sat(r.u[i], b);
    return r.v;
}

// A wavefront's accumulators row by row of n: store(r, c, x) is called for every row r < 32 FN with four columns from c = 4 (lane % (8 FM))
// on, so that lanes next to each other hold columns next to each other.  32 rows at a time pass through the wavefront's part of `lds`
// (4 KB per FM), their 16-byte chunks exchanged by the row: the accumulators' own order, 16 to 32 bytes of 32 rows each, took the caches
// two to four times as many requests.
template <int FM, int FN, class Store>
__device__ inline void by_rows(unsigned char *lds, f32x16 (&acc)[FM][FN], Store store) {
    constexpr int CHUNKS = 8 * FM, ROWS = 64 / CHUNKS;
    const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31, wave = threadIdx.x >> 6;
    unsigned char *mine = lds + wave * (FM * 4096);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f32x4 x;
#pragma unroll
                for (int u = 0; u < 4; ++u) x[u] = acc[i][j][4 * q + u];
                *(f32x4 *)(mine + l32 * (CHUNKS * 16) + (((8 * i + 2 * q + half) ^ (l32 & (CHUNKS - 1))) << 4)) = x;
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();                   // LDS operations of a wavefront complete in order
#pragma unroll 8
        for (int r0 = 0; r0 < 32; r0 += ROWS) {
            const int r = r0 + lane / CHUNKS, c = lane % CHUNKS;
            store(32 * j + r, 4 * c, *(const f32x4 *)(mine + r * (CHUNKS * 16) + ((c ^ (r & (CHUNKS - 1))) << 4)));
        }
    }
}

// Epilogue::run(args, lds, acc, m, n, split, live): acc[i][j][v] is C at m + 32 i + 8 (v / 4) + 4 half + v % 4, n + 32 j + lane % 32; lds: the
// workgroup's, free.
template <class Sh, int AK, int BK, class Epilogue, bool CUTS = false, bool SHIFT = false>
__global__ void __launch_bounds__(64 * Sh::NW, Sh::NW / 4)
product_kernel(ProductArgs p, typename Epilogue::Args e) {
    constexpr int FM = Sh::FM, FN = Sh::FN, NS = Sh::NS, NW = Sh::NW;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    // Tiles in an order in which the workgroups of an XCD (ids eight apart) share operands: bands of eight column tiles, row tile by row
    // tile, an eighth of the order each.
    const int64_t n = p.live_n ? *p.live_n : p.n;
    const int64_t k = p.live_k ? *p.live_k : p.k;
    // CUTS: an eighth of every part, whose lengths differ, or a whole one of at most eight tiles, from the longest to the shortest (up to 64).
    const int64_t ntiles = (n + Sh::NT - 1) / Sh::NT, plane = p.mtiles * ntiles, total = plane * p.splits;
    const int64_t xcd = blockIdx.x & 7, q = blockIdx.x >> 3;
    int64_t in;
    int split;
    if (CUTS) {
        const int64_t per = plane <= 8 ? plane : (plane + 7) / 8, at = q / per, part = plane <= 8 ? at * 8 + xcd : at;
        // (an eighth of fewer tiles begins where the part before ended)
        in = plane <= 8 ? q - at * per : ((xcd + at * (8 - (plane + per - 1) / per)) & 7) * per + q - at * per;
        if (part >= p.splits || in >= plane) return;       // the whole workgroup
        split = __builtin_amdgcn_readfirstlane((int)part);
    } else {
        const int64_t per = (total + 7) / 8, idx = xcd * per + q;
        if (q >= per || idx >= total) return;
        split = __builtin_amdgcn_readfirstlane((int)(idx / plane));
        in = idx - split * plane;
    }
    if (CUTS && p.splits > 1 && p.splits <= 64) {
        const int lane = threadIdx.x & 63;
        const int64_t len = lane < p.splits ? p.cuts[lane + 1] - p.cuts[lane] : -1;
        const int key = len < 0 ? -1 : len < 0x7FFFFFFF ? (int)len : 0x7FFFFFFF;
        int longer = 0;
        for (int i = 0; i < p.splits; ++i) {
            const int other = __builtin_amdgcn_readlane(key, i);
            longer += other > key || (other == key && i < lane);
        }
        split = __ffsll((unsigned long long)__ballot(lane < p.splits && longer == split)) - 1;      // (a total order: one lane)
        split = __builtin_amdgcn_readfirstlane(split);
    }
    const int64_t band = in / (8 * p.mtiles), wide = ntiles - band * 8 < 8 ? ntiles - band * 8 : 8, r = in - band * 8 * p.mtiles;
    const int m0 = __builtin_amdgcn_readfirstlane((int)(r / wide * Sh::MT)), n0 = __builtin_amdgcn_readfirstlane((int)((band * 8 + r % wide) * Sh::NT));
    const int64_t stages = (k + 63) / 64;
    int s0 = __builtin_amdgcn_readfirstlane((int)(stages * split / p.splits)), s1 = __builtin_amdgcn_readfirstlane((int)(stages * (split + 1) / p.splits));
    if (CUTS) {
        static_assert(!CUTS || BK == ACROSS, "rows of K");
        int64_t lo = p.cuts[split], hi = p.cuts[split + 1];
        lo = lo < 0 ? 0 : (lo > k ? k : lo);
        hi = hi < lo ? lo : (hi > k ? k : hi);
        const int64_t block = split + lo / 64;
        s0 = __builtin_amdgcn_readfirstlane((int)block);
        s1 = s0 + __builtin_amdgcn_readfirstlane((int)((hi - lo + 63) / 64));
        p.b.base = (const unsigned char *)p.b.base + (lo - 64 * block) * p.b.ld;      // stage s0 begins at row lo
        p.b.depth = 64 * block + hi - lo;
    }

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wy = wave / Sh::WX, wx = wave % Sh::WX;
    const unsigned lds0 = (unsigned)(uintptr_t)((__attribute__((address_space(3))) unsigned char *)smem);
    ProductCopies<AK, Sh::MT, NW> ca;
    ProductCopies<BK, Sh::NT, NW> cb;
    constexpr int UA = ProductCopies<AK, Sh::MT, NW>::U, UB = ProductCopies<BK, Sh::NT, NW>::U;
    ca.init(p.a, m0, lane, wave);
    cb.init(p.b, n0, lane, wave);
    constexpr int U = UA + UB + (SHIFT ? 1 : 0);
    const int ma = wy * FM * 32, nb = wx * FN * 32;
    auto request = [&](int u, int s, int slot) {           // copy u of a stage; past the end the last one again: all stages count alike
        if (s > s1 - 1) s = s1 - 1;
        const unsigned at = lds0 + (unsigned)(slot * Sh::STAGE);
        if (u < UA) ca.issue(u, s, lane, wave, at);
        else if (u < UA + UB) cb.issue(u - UA, s, lane, wave, at + Sh::MT * 128);
        else                                               // this wavefront's columns' shifts
            global_to_lds4(p.shift + (int64_t)(s >> p.shift_stages) * p.shift_ld + n0 + nb, (unsigned)((lane & (32 * FN - 1)) * 4), lds0 + (unsigned)(NS * Sh::STAGE + (slot * NW + wave) * 256));
    };
    f32x16 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
    const unsigned la = fragment_lane<AK, Sh::MT>(lane), lb = fragment_lane<BK, Sh::NT>(lane);
    if (s0 < s1) {
        static_assert(!SHIFT || FN <= 2, "a lane a column");
        bf16x8 fa[2][FM], fb[2][FN];
        uint32_t by[2][FN];                                // shifts of the stage, and of the next
        auto read_shift = [&](int set, int slot) {
#pragma unroll
            for (int j = 0; j < FN; ++j) by[set][j] = *(const uint32_t *)(smem + NS * Sh::STAGE + (slot * NW + wave) * 256 + (32 * j + (lane & 31)) * 4);
        };
        auto read = [&](int set, int f, int slot, int kk) {          // fragment f of a K step of 16: the columns', then the rows'
            const unsigned char *sa = smem + slot * Sh::STAGE;
            if (f < FN) fb[set][f] = fragment<BK, Sh::NT>(sa + Sh::MT * 128, lb, nb + 32 * f, kk);
            else fa[set][f - FN] = fragment<AK, Sh::MT>(sa, la, ma + 32 * (f - FN), kk);
        };
        auto pin = []() { __builtin_amdgcn_sched_barrier(0); };      // keeps the order below
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int u = 0; u < U; ++u) request(u, s0 + i, i);
        wait_vmcnt<(NS - 1) * U>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int f = 0; f < FM + FN; ++f) read(0, f, 0, 0);
        if (SHIFT) read_shift(0, 0);
        int slot = 0;
        // The fragments of a K step are read while the products of the one before run.  The barrier of a stage stands behind the first
        // products of its last K step: by then every fragment of it is in registers, so the slot is free for the stage NS further on, and
        // the next stage, requested NS - 1 stages ago, has landed.
        for (int s = s0; s < s1; ++s) {
            const int next = slot + 1 == NS ? 0 : slot + 1;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                constexpr int I = FM * FN, R = FM + FN, K0 = I > 2 ? 1 : 0;
                const int cur = kk & 1;
                const bool last = kk == 3;
                if (SHIFT)
#pragma unroll
                    for (int j = 0; j < FN; ++j) fb[cur][j] = lower_exponents(fb[cur][j], by[0][j]);
#pragma unroll
                for (int i = 0; i < I; ++i) {
                    pin();
                    acc[i % FM][i / FM] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[cur][i % FM], fb[cur][i / FM], acc[i % FM][i / FM], 0, 0, 0);
                    pin();
                    if (last && i == K0) {
                        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                        wait_vmcnt<(NS - 2) * U>();
                        __builtin_amdgcn_s_barrier();
                        asm volatile("" ::: "memory");
                        pin();
                    }
                    const int first = last ? K0 : 0;       // reads and copies are spread over the products from here on
#pragma unroll
                    for (int f = 0; f < R; ++f)
                        if (f * (I - first) / R + first == i) read(cur ^ 1, f, last ? next : slot, (kk + 1) & 3);
                    if (SHIFT && last && i == I - 1) read_shift(1, next);
                    if (last)
#pragma unroll
                        for (int u = 0; u < U; ++u)
                            if (u * (I - first) / U + first == i) request(u, s + NS, slot);
                }
            }
            if (SHIFT)
#pragma unroll
                for (int j = 0; j < FN; ++j) by[0][j] = by[1][j];
            slot = next;
        }
        wait_vmcnt<0>();                                   // no copy is under way when the workgroup gives its LDS back
    }
    __syncthreads();                                       // everyone has read the last stage
    Epilogue::template run<FM, FN>(e, smem, acc, m0 + ma, n0 + nb, split, n);
}

template <class Sh, int AK, int BK, class Epilogue, bool CUTS = false, bool SHIFT = false>
static qless_status launch_product(const ProductArgs &p, const typename Epilogue::Args &e, hipStream_t st) {
    constexpr int LDS = Sh::LDS + (SHIFT ? Sh::NS * Sh::NW * 256 : 0);
    static_assert(LDS <= 160 * 1024, "the stages fit");
    QLESS_LDS_KERNEL((product_kernel<Sh, AK, BK, Epilogue, CUTS, SHIFT>), LDS);
    const int64_t total = p.mtiles * ((p.n + Sh::NT - 1) / Sh::NT) * p.splits, plane = total / p.splits;
    const int64_t grid = !CUTS ? (total + 7) / 8 * 8 : plane <= 8 ? (p.splits + 7) / 8 * 8 * plane : (plane + 7) / 8 * 8 * p.splits;
    if (!launchable(grid, 64 * Sh::NW)) return QLESS_ERR_UNSUPPORTED;
    if (grid > 0)
        hipLaunchKernelGGL((product_kernel<Sh, AK, BK, Epilogue, CUTS, SHIFT>), dim3((unsigned)grid), dim3(64 * Sh::NW), LDS, st, p, e);
    return QLESS_OK;
}

}  // namespace qless
