// Products with weights in 4-bit codes: out[m][n] = sum over k of A[m][k] W[n][k] on v_mfma_scale_f32_16x16x128_f8f6f4.
//
// The weights are the instruction's first operand and the activations its second, so that a lane ends up with four
// neighbouring columns of one row.  A lane l supplies row l % 16 of an operand and the scale of the 32 values that the
// operand's lane group l / 16 stands for; 4-bit codes sit 32 consecutive k to a lane (group g: k = 32 g ..), 8-bit ones as
// two runs of 16 (k = 16 g .. and 64 + 16 g ..).  A sum over k may go in any order as long as both operands follow it; the
// kernels choose orders in which a lane's scale bytes are neighbours in memory.
#include <type_traits>

#include "layer.hpp"
#include "layer_kernels.hpp"
#include "staging.hpp"

namespace guide {
namespace {

// W times A with scale bytes WSEL of `sw` and ASEL of `sa`.
template <int ABITS, int WSEL, int ASEL>
__device__ __forceinline__ f32x4 mma(i32x4 w, const i32x4 *a, f32x4 c, int sw, int sa) {
    const i32x8 W = {w[0], w[1], w[2], w[3], 0, 0, 0, 0};
    if constexpr (ABITS == 4) {
        const i32x8 A = {a[0][0], a[0][1], a[0][2], a[0][3], 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(W, A, c, 4, 4, WSEL, sw, ASEL, sa);
    } else {
        const i32x8 A = {a[0][0], a[0][1], a[0][2], a[0][3], a[1][0], a[1][1], a[1][2], a[1][3]};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(W, A, c, 4, 0, WSEL, sw, ASEL, sa);
    }
}

// The same on 32 x 32 x 64: lane l supplies row l % 32 and half l / 32 of the 64 (8-bit codes: 16 h .. and 32 + 16 h ..), and
// gets column l % 32 of rows 8 a + 4 (l / 32) .. in its values 4 a ..
template <int ABITS, int SEL>
__device__ __forceinline__ f32x16 mma(i32x4 w, const i32x4 *a, f32x16 c, int sw, int sa) {
    const i32x8 W = {w[0], w[1], w[2], w[3], 0, 0, 0, 0};
    if constexpr (ABITS == 4) {
        const i32x8 A = {a[0][0], a[0][1], a[0][2], a[0][3], 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(W, A, c, 4, 4, SEL, sw, SEL, sa);
    } else {
        const i32x8 A = {a[0][0], a[0][1], a[0][2], a[0][3], a[1][0], a[1][1], a[1][2], a[1][3]};
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(W, A, c, 4, 0, SEL, sw, SEL, sa);
    }
}

template <int T>
__device__ __forceinline__ void store4(typename Elem<T>::type *p, f32x4 v, uint32_t left) {
    typename Elem<T>::type e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = (typename Elem<T>::type)v[i];
    if (left >= 4) {
        __builtin_memcpy(p, e, sizeof e);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((uint32_t)i < left) p[i] = e[i];
    }
}

// ------------------------------------------------------------------------------------------ up to 16 rows: streaming W

// A block takes 16 rows and 16 columns and its waves take turns along k, 512 at a time, straight from memory to registers: every code of
// W is read once, by one wave, in runs of 64 bytes to a lane.  In step s of four, lane group g stands for group 4 g + s of
// the 16, so a lane's four scale bytes are one word.  The waves' sums are joined in LDS, in the waves' order.
// Bound by memory, though not at its full rate: one row against 28672 x 8192 27 us (125 MB, 4.6 TB/s; plain reads of as much 6.6).
template <int T, int ABITS, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void stream_kernel(guide_product_spec s) {
    using E = typename Elem<T>::type;
    constexpr int kA = ABITS / 4;                                   // 16-byte pieces of A to a step
    __shared__ float part[WAVES][16][20];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, row = lane % 16, g = lane / 16;
    const uint32_t n0 = blockIdx.x * 16, m0 = blockIdx.y * 16;
    const uint32_t groups = s.k / 32u;
    const int64_t n = min(n0 + row, s.n - 1), m = min(m0 + row, s.m - 1);
    const uint8_t *w = s.w_codes + n * s.w_codes_stride, *ws = s.w_scales + n * s.w_scales_stride;
    const uint8_t *a = s.a_codes + m * s.a_codes_stride, *as = s.a_scales + m * s.a_scales_stride;
    f32x4 acc = {0, 0, 0, 0};

    // Sixteen groups from g0 on; FULL: all of them exist (past the end codes are zeros, scales finite).
    auto sixteen = [&](auto full, uint32_t g0) __attribute__((always_inline)) {
        constexpr bool FULL = decltype(full)::value;
        i32x4 wv[4], av[4][kA];
        const uint32_t mine = g0 + g * 4u;                          // the lane's four groups
        auto codes = [&](const uint8_t *p, uint32_t group, uint32_t at) __attribute__((always_inline)) {
            return FULL || group < groups ? *(const i32x4 *)(p + at) : i32x4{0, 0, 0, 0};
        };
        auto bytes = [&](const uint8_t *p) __attribute__((always_inline)) {
            int v = 0;
            if constexpr (FULL) {
                __builtin_memcpy(&v, p + mine, 4);
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (mine + q < groups) v |= p[mine + q] << (8 * q);
            }
            return v;
        };
#pragma unroll
        for (int q = 0; q < 4; ++q) wv[q] = codes(w, mine + q, (mine + q) * 16u);
        const int sw = bytes(ws), sa = bytes(as);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (ABITS == 4) {
                av[q][0] = codes(a, mine + q, (mine + q) * 16u);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {                       // half h: 16 of the values of lane groups 2 h + g / 2
                    const uint32_t at = g0 + (2 * h + g / 2) * 4u + q;
                    av[q][h] = codes(a, at, at * 32u + (g % 2) * 16u);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);                          // all loads on their way before the first product waits
        unrolled<4>([&](auto step) __attribute__((always_inline)) {
            constexpr int q = decltype(step)::value;
            acc = mma<ABITS, q, q>(wv[q], av[q], acc, sw, sa);
        });
    };
    uint32_t g0 = wave * 16u;
    for (; g0 + 16 <= groups; g0 += WAVES * 16u) sixteen(std::true_type{}, g0);
    if (g0 < groups) sixteen(std::false_type{}, g0);

    *(f32x4 *)&part[wave][row][g * 4] = acc;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    const int r = threadIdx.x / 4, c = threadIdx.x % 4 * 4;
    if (m0 + r >= s.m || n0 + c >= s.n) return;
    f32x4 sum = *(const f32x4 *)&part[0][r][c];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) sum += *(const f32x4 *)&part[v][r][c];
    store4<T>((E *)s.out + (int64_t)(m0 + r) * s.out_stride + n0 + c, sum, s.n - (n0 + c));
}

// -------------------------------------------------------------------------------------------------- more rows: LDS tiles

// ROWS rows from memory to LDS; what is beyond the operand's last row, and beyond the end of k, becomes zeros (`left` bytes of the row
// are real).
template <int ROWS, int WAVES>
struct Loader : TilePlaces<ROWS, WAVES> {
    using Places = TilePlaces<ROWS, WAVES>;
    __amdgpu_buffer_rsrc_t rsrc;

    __device__ __forceinline__ void init(const uint8_t *base, uint32_t rows, int64_t row_stride, int64_t row_bytes, int wave, int lane) {
        rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)Places::bytes(rows, row_stride, row_bytes), 0x00020000);
        Places::init(row_stride, wave, lane);
    }
    // instruction i of the wave's kLoads
    __device__ __forceinline__ void load(int i, int at, int left, uint8_t *lds, int wave) const {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(lds + (wave * Places::kLoads + i) * 1024), 16,
                                                 (int)Places::of_lane(i, left), (int)Places::of_wave(at, left), 0, 0);
    }
};

// Holds the compiler to the source's order around a row of products: they, whose results nothing needs for long, would
// otherwise all be moved behind the reads and loads that they are there to cover.
template <int N>
__device__ __forceinline__ void pin(f32x16 (&c)[N]) {
    static_assert(N == 1 || N == 2 || N == 4, "columns of tiles of a wave");
    if constexpr (N == 1) asm volatile("" : "+a"(c[0]));
    else if constexpr (N == 2) asm volatile("" : "+a"(c[0]), "+a"(c[1]));
    else asm volatile("" : "+a"(c[0]), "+a"(c[1]), "+a"(c[2]), "+a"(c[3]));
}

// The scale bytes of 16 groups of a row from group `at` on: past the row's end zeros, finite scales for zero codes.  The load
// takes the last 16 bytes before the row's end where fewer are left, real_scales() moves them into place; `back`: there are 16
// (else `other`, any 16 bytes, is loaded for nothing: only a row's first scales exist then, and few_scales() reads them).
struct Scales { uint64_t lo, hi; };
__device__ __forceinline__ Scales load_scales(const uint8_t *row, int at, int groups, bool back, const uint8_t *other) {
    Scales v;
    __builtin_memcpy(&v, back ? row + min(at, groups - 16) : other, 16);
    return v;
}
__device__ __forceinline__ Scales real_scales(Scales v, int left) {
    const int shift = left >= 16 ? 0 : 8 * (16 - max(left, 0));                  // 0 .. 128
    const uint64_t lo = shift >= 128 ? 0 : shift >= 64 ? v.hi >> (shift & 63) : shift ? v.lo >> shift | v.hi << (64 - shift) : v.lo;
    return {lo, shift >= 64 ? 0 : v.hi >> (shift & 63)};
}
__device__ __forceinline__ Scales few_scales(const uint8_t *row, int groups) {
    Scales v = {0, 0};
    for (int i = 0; i < groups; ++i) (i < 8 ? v.lo : v.hi) |= (uint64_t)row[i] << (8 * (i & 7));
    return v;
}

// BM x BN to a block of 2 x 2 waves, each BM / 2 x BN / 2 in tiles of 32 x 32 (16 x 16 x 128 takes 24 to 32 cycles for what
// 32 x 32 x 64 does in 17 to 19 when both sides are 4 bits wide).  A step is 128 of k, two instructions deep; lane half h
// stands for groups 2 h and 2 h + 1 of its four, so that its two scale bytes are neighbours.  Codes come to LDS a pair of steps
// at a time, two pairs being there: in a pair's first step the block multiplies from registers and reads the operands of
// the second, after whose reads the pair's buffer is free; in the second it reads the next pair's first and sends for the
// pair after that one, which has a step to arrive, one load to every few products.  Scale bytes come 16 groups (four
// steps) at a time through registers.
// Where there are too few tiles to fill the chip, k is split over blocks: split p sums split_groups groups (a multiple of
// 16) and writes to row p m of `out`, which is then a plane of 32-bit sums for each split.
// Large products are bound by the card's power as much as by the instructions: 8192 x 28672 x 8192 in 4 bits takes 910 to 960 us (4000
// to 4230 TFLOP/s), 870 on an earlier form with all codes zero where random ones took 1020, and the products alone, without loads and
// reads, 810; 8 bits 1450 to 1520 us, products alone 1135.  Small ones are bound by the codes' way from memory.
template <int T, int ABITS, int BM, int BN>
__global__ __launch_bounds__(256) void tile_kernel(guide_product_spec s, uint32_t m_tiles, uint32_t n_tiles, uint32_t splits, uint32_t split_groups) {
    using E = typename Elem<T>::type;
    constexpr int kA = ABITS / 4;
    constexpr int MT = BM / 64, NT = BN / 64;                                    // 32-row tiles of a wave
    constexpr int kAPart = BM * kRow, kPair = kA * kAPart + BN * kRow;
    // arrays of their own: a read of one does not wait for loads on their way to another
    __shared__ __align__(16) uint8_t buf0[kPair], buf1[kPair], sc0[(BM + BN) * 16], sc1[(BM + BN) * 16];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = lane % 32, half = lane / 32;
    const int wm = wave % 2, wn = wave / 2;

    // Blocks go round the eight XCDs in turn; each XCD gets a run of tiles of its own, walked in strips of 8 rows of tiles,
    // so that the 32 blocks it runs at once share eight rows of A and four of W in its L2.  A block takes the run's tile
    // `local` and then every (blocks of the XCD)-th.
    const uint32_t total = m_tiles * n_tiles * splits, per = (total + 7) / 8;
    uint32_t local = blockIdx.x / 8;
    uint32_t m0, n0, split;
    int first, groups;
    Loader<BM, 4> a_codes;
    Loader<BN, 4> w_codes;
    const uint8_t *a_sc, *w_sc;
    Scales a_first, w_first;
    bool back;

    f32x16 acc[MT][NT];
    i32x4 wv[2][NT][2], av[MT][2][kA];                                           // operands: W's of this step and the next, A's of either
    int sw[2][NT], sa[MT];

    constexpr int kLoadsA = Loader<BM, 4>::kLoads, kSendA = kA * kLoadsA, kSend = kSendA + Loader<BN, 4>::kLoads;
    auto send = [&](int u, int pair, uint8_t *buf) __attribute__((always_inline)) {                             // load u of a pair's kSend
        const int g0 = pair * 8, h = u / kLoadsA;
        if (u < kSendA) a_codes.load(u % kLoadsA, (g0 + h * 4) * (ABITS * 4), (groups - g0 - h * 4) * (ABITS * 4), buf + h * kAPart, wave);
        else w_codes.load(u - kSendA, g0 * 16, (groups - g0) * 16, buf + kA * kAPart, wave);
    };
    // operands of a tile row or column of a step; `at`: the step's number among the four whose scales `sc` holds
    auto read_w = [&](int j, int to, int at, const uint8_t *buf, const uint8_t *sc) __attribute__((always_inline)) {
        const int r = wn * (BN / 2) + row;
#pragma unroll
        for (int q = 0; q < 2; ++q) wv[to][j][q] = *(const i32x4 *)(buf + kA * kAPart + r * kRow + swizzled(row, at % 2 * 4 + 2 * half + q) * 16 + j * 32 * kRow);
        sw[to][j] = *(const uint16_t *)(sc + (BM + r) * 16 + half * 2 + at * 4 + j * 512);
    };
    auto read_a = [&](int i, int at, const uint8_t *buf, const uint8_t *sc) __attribute__((always_inline)) {
        const int r = wm * (BM / 2) + row;
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int h = 0; h < kA; ++h)
                av[i][q][h] = *(const i32x4 *)(buf + at % 2 * (kA - 1) * kAPart + r * kRow + i * 32 * kRow +
                                               swizzled(row, ABITS == 4 ? at % 2 * 4 + 2 * half + q : (2 * h + q) * 2 + half) * 16);
        sa[i] = *(const uint16_t *)(sc + r * 16 + half * 2 + at * 4 + i * 512);
    };
    // A step (W's operands in set z) with the reads for the next (number `at` of its four, from `buf`) and, in a pair's second
    // step, the loads for pair `pair` (to `into`, all read by now) between its products.
    auto turn = [&](auto set, int at, const uint8_t *buf, const uint8_t *sc, int pair, uint8_t *into) __attribute__((always_inline)) {
        constexpr int z = decltype(set)::value, o = 1 - z, kSlots = 2 * MT * NT;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const int y = (2 * i + q) * NT + j;
                    if constexpr (z == 1) {
#pragma unroll
                        for (int u = y * kSend / kSlots; u < (y + 1) * kSend / kSlots; ++u) send(u, pair, into);
                    }
                    if (y % (2 * MT) == 0) read_w(y / (2 * MT), o, at, buf, sc);
                    acc[i][j] = q ? mma<ABITS, 1>(wv[z][j][1], av[i][1], acc[i][j], sw[z][j], sa[i])
                                  : mma<ABITS, 0>(wv[z][j][0], av[i][0], acc[i][j], sw[z][j], sa[i]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                pin<NT>(acc[i]);
            }
            read_a(i, at, buf, sc);                                              // (the products above have taken the last one's)
        }
        __builtin_amdgcn_sched_barrier(0);                                       // (or the last read is merged with another buffer's, and waits for loads)
    };
    // The next pair is in LDS and no wave reads this one's any more.
    auto meet = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0x0070);
        __builtin_amdgcn_s_barrier();
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;

    auto place = [&](uint8_t *sc, Scales a, Scales w) __attribute__((always_inline)) {                          // (threads past a side's rows write what others do)
        *(Scales *)(sc + threadIdx.x % BM * 16) = a;
        *(Scales *)(sc + (BM + threadIdx.x % BN) * 16) = w;
    };
    // Sends for the first two pairs of steps of tile `local`, if there is one.
    auto begin = [&]() __attribute__((always_inline)) {
        const uint32_t turn_of = blockIdx.x % 8 * per + local;
        if (local >= per || turn_of >= total) return false;
        split = turn_of / (m_tiles * n_tiles);
        const uint32_t t = turn_of - split * (m_tiles * n_tiles);
        const uint32_t strip = t / (8 * n_tiles), in = t - strip * 8 * n_tiles, high = min(8u, m_tiles - strip * 8);
        m0 = (strip * 8 + in % high) * BM, n0 = in / high * BN;
        first = (int)(split * split_groups), groups = min((int)split_groups, (int)(s.k / 32u) - first);
        back = first > 0 || groups >= 16;
        a_codes.init(s.a_codes + (int64_t)m0 * s.a_codes_stride + first * (ABITS * 4), s.m - m0, s.a_codes_stride, groups * (ABITS * 4), wave, lane);
        w_codes.init(s.w_codes + (int64_t)n0 * s.w_codes_stride + first * 16, s.n - n0, s.w_codes_stride, groups * 16, wave, lane);
        a_sc = s.a_scales + (int64_t)min(m0 + threadIdx.x % BM, s.m - 1) * s.a_scales_stride + first;
        w_sc = s.w_scales + (int64_t)min(n0 + threadIdx.x % BN, s.n - 1) * s.w_scales_stride + first;
        if (back) {
            a_first = load_scales(a_sc, 0, groups, true, nullptr);
            w_first = load_scales(w_sc, 0, groups, true, nullptr);
        } else {
            a_first = few_scales(a_sc, groups);
            w_first = few_scales(w_sc, groups);
        }
#pragma unroll
        for (int u = 0; u < kSend; ++u) send(u, 0, buf0);
#pragma unroll
        for (int u = 0; u < kSend; ++u) send(u, 1, buf1);
        return true;
    };
    for (bool more = begin(); more;) {
        place(sc0, back ? real_scales(a_first, groups) : a_first, back ? real_scales(w_first, groups) : w_first);
        meet();
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
#pragma unroll
        for (int i = 0; i < MT; ++i) pin<NT>(acc[i]);                                // (no zeros to peel a first step for)
#pragma unroll
        for (int j = 0; j < NT; ++j) read_w(j, 0, 0, buf0, sc0);
#pragma unroll
        for (int i = 0; i < MT; ++i) read_a(i, 0, buf0, sc0);
        for (int step = 0; step * 4 < groups; step += 8) {
            auto four = [&](int step, const uint8_t *sc, uint8_t *next) __attribute__((always_inline)) {
                turn(I0{}, 1, buf0, sc, 0, nullptr);
                meet();
                const Scales a_next = load_scales(a_sc, step * 4 + 16, groups, back, s.w_codes), w_next = load_scales(w_sc, step * 4 + 16, groups, back, s.w_codes);
                turn(I1{}, 2, buf1, sc, step / 2 + 2, buf0);
                turn(I0{}, 3, buf1, sc, 0, nullptr);
                place(next, real_scales(a_next, groups - (step * 4 + 16)), real_scales(w_next, groups - (step * 4 + 16)));
                meet();
                turn(I1{}, 0, buf0, next, step / 2 + 3, buf1);
            };
            four(step, sc0, sc1);
            if (step * 4 + 16 >= groups) break;
            four(step + 4, sc1, sc0);
        }
        // The next tile's loads are on their way while this one's results are written, once no wave reads the buffers any more.
        meet();
        E *const out = (E *)s.out + ((int64_t)split * s.m + m0 + wm * (BM / 2) + row) * s.out_stride;
        const uint32_t m_left = s.m - m0, n_at = n0 + wn * (BN / 2);
        local += gridDim.x / 8;
        more = begin();
        // A lane holds columns 8 a + 4 half .. of row `row`: with 16-bit results, the halves change pieces, so that a lane writes 16
        // bytes and a row's two lanes 32.
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if ((uint32_t)(wm * (BM / 2) + i * 32 + row) >= m_left) continue;
            E *o = out + (int64_t)(i * 32) * s.out_stride;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int a = 0; a < 4; a += 8 / sizeof(E) / 2) {
                    constexpr uint32_t kPer = 16 / sizeof(E);
                    E e[kPer];
                    uint32_t n;
                    if constexpr (sizeof(E) == 4) {
#pragma unroll
                        for (int b = 0; b < 4; ++b) e[b] = acc[i][j][a * 4 + b];
                        n = n_at + j * 32 + a * 8 + half * 4;
                    } else {
                        uint32_t x[2], y[2];                             // pieces a and a + 1
                        E f[8];
#pragma unroll
                        for (int b = 0; b < 8; ++b) f[b] = (E)acc[i][j][a * 4 + b];
                        __builtin_memcpy(x, f, 8);
                        __builtin_memcpy(y, f + 4, 8);
#pragma unroll
                        for (int b = 0; b < 2; ++b) {                    // x: the lower half's piece, y: its next; the upper half's: likewise
                            const auto z = __builtin_amdgcn_permlane32_swap(x[b], y[b], false, false);
                            x[b] = z[0], y[b] = z[1];
                        }
                        __builtin_memcpy(e, x, 8);
                        __builtin_memcpy(e + 4, y, 8);
                        n = n_at + j * 32 + a * 8 + half * 8;
                    }
                    if (n + kPer <= s.n) {
                        __builtin_memcpy(o + n, e, 16);
                    } else {
#pragma unroll
                        for (uint32_t b = 0; b < kPer; ++b)
                            if (n + b < s.n) o[n + b] = e[b];
                    }
                }
        }
    }
}

// out = the sum of the splits' planes, in their order; four columns to a thread.  Bound by its loads' latency: eight planes' are on their
// way at once.
template <int T>
__global__ __launch_bounds__(kBlock) void join_kernel(const float *planes, uint32_t splits, uint32_t m, uint32_t n, uint32_t pitch,
                                                      typename Elem<T>::type *out, int64_t out_stride) {
    const uint32_t c = (blockIdx.x * kBlock + threadIdx.x) * 4, r = blockIdx.y;
    if (c >= n) return;
    const float *p = planes + (size_t)r * pitch + c;
    f32x4 sum = {0, 0, 0, 0};
    for (uint32_t i = 0; i < splits; i += 8) {
        f32x4 v[8];
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) v[u] = *(const f32x4 *)(p + (size_t)min(i + u, splits - 1) * m * pitch);
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u)
            if (i + u < splits) sum += v[u];
    }
    store4<T>(out + (int64_t)r * out_stride + c, sum, n - c);
}

template <int T, int ABITS, int BM, int BN>
hipError_t tile_as(const guide_product_spec &s, uint32_t splits, float *scratch, hipStream_t stream) {
    const uint32_t m_tiles = (s.m + BM - 1) / BM, n_tiles = (s.n + BN - 1) / BN, groups = s.k / 32;
    const uint32_t per = splits > 1 ? (groups + 16 * splits - 1) / (16 * splits) * 16 : groups;
    if (splits > 1) splits = (groups + per - 1) / per;                           // (every split has groups)
    // as many blocks as run at once (by their LDS), or as there are tiles
    constexpr uint32_t kPair = (BM * (ABITS / 4) + BN) * kRow, kAtOnce = kNumCU * (160 * 1024 / (2 * kPair + 2 * (BM + BN) * 16));
    const uint64_t tiles = ((uint64_t)m_tiles * n_tiles * splits + 7) / 8 * 8;
    const uint64_t blocks = tiles < kAtOnce ? tiles : kAtOnce;
    if (splits == 1) {
        tile_kernel<T, ABITS, BM, BN><<<(uint32_t)blocks, 256, 0, stream>>>(s, m_tiles, n_tiles, 1, groups);
        return hipGetLastError();
    }
    const uint32_t pitch = (s.n + 3) / 4 * 4;
    guide_product_spec part = s;
    part.out = scratch;
    part.out_stride = pitch;
    tile_kernel<GUIDE_F32, ABITS, BM, BN><<<(uint32_t)blocks, 256, 0, stream>>>(part, m_tiles, n_tiles, splits, per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    join_kernel<T><<<dim3((s.n + 4 * kBlock - 1) / (4 * kBlock), s.m), kBlock, 0, stream>>>(scratch, splits, s.m, s.n, pitch,
                                                                                          (typename Elem<T>::type *)s.out, s.out_stride);
    return hipGetLastError();
}

// Tiles of a size, and the number of splits of k that brings them near `fill` blocks: at least 1024 of k each, planes within
// the scratch.
uint64_t tiles_of(const guide_product_spec &s, uint32_t bm, uint32_t bn) { return (uint64_t)((s.m + bm - 1) / bm) * ((s.n + bn - 1) / bn); }
uint32_t splits_of(const guide_product_spec &s, uint64_t tiles, uint32_t fill) {
    uint64_t n = fill / tiles;
    n = n < s.k / 1024 ? n : s.k / 1024;
    const uint64_t plane = (uint64_t)s.m * ((s.n + 3) / 4 * 4) * sizeof(float), room = kScratch / plane;
    n = n < room ? n : room;
    return (uint32_t)(n < 1 ? 1 : n > 16 ? 16 : n);
}

// Up to 16 rows: whether W is streamed.  Every 16 columns' block reads all of A, so that with much work tiles are ahead: streamed / in
// tiles, 8 rows of 8 bits 5120 x 13824 16.9 / 13.6 us but 4096 x 8192 7.0 / 8.9, 4 rows 28672 x 8192 30.8 / 27.0 but 8192 x 8192 10.1 / 11.8,
// one row 57344 x 8192 48.6 / 43.8 but 8192 x 28672 23.8 / 26.3, 16 rows of 4 bits 8192 x 16384 20.1 / 16.1 but 5120 x 5120 of 8 bits 9.6 / 9.3.
// And a long k with few columns is worked on by few blocks (one row 512 x 32768 14.3 / 9.1, 256 x 16384 8.0 / 7.2; 1024 x 8192 5.1 / 7.1).
bool streams(const guide_product_spec &s) {
    if (s.k >= 16384 && s.k / 16 >= s.n) return false;
    return (uint64_t)s.m * (uint32_t)s.a_bits * s.n * s.k < 3500000000ull;
}

template <int T, int ABITS>
hipError_t product_as(const guide_product_spec &s, float *scratch, hipStream_t stream) {
    const bool near = s.k > 0 && s.a_codes_stride < (1 << 22) && s.w_codes_stride < (1 << 22);      // a tile's rows within 2^31 bytes
    if (!near || (s.m <= 16 && streams(s))) {
        stream_kernel<T, ABITS, 8><<<dim3((s.n + 15) / 16, (s.m + 15) / 16), 512, 0, stream>>>(s);
        return hipGetLastError();
    }
    // Large tiles reuse more (a compute unit does what one of them holds in 0.7 of the time that it takes in tiles of 128 x 128), but
    // come in rounds of a tile to a compute unit: large / small 2048 x 5120 x 5120 in 4 bits 41.2 / 43.4 us, 4096 x 5120 x 5120
    // 77 / 68, 1024 x 8192 x 8192 55 / 45, 512 x 28672 x 8192 62 / 86, in 8 bits 103 / 131, 1024 x 8192 x 8192 in 8 bits 56 / 74.
    constexpr uint32_t kTall = ABITS == 4 ? 256 : 128, kTimes = kTall * 256 / (128 * 128);
    const uint64_t large = (tiles_of(s, kTall, 256) + kNumCU - 1) / kNumCU, small = (tiles_of(s, 128, 128) + kNumCU - 1) / kNumCU;
    if (s.m > 64 && 5 * kTimes * large <= 7 * small) return tile_as<T, ABITS, kTall, 256>(s, 1, scratch, stream);
    // 96 x 8192 x 8192 takes 18.8 us in tiles of 128 x 128, 21.9 in 64 x 64; 64 x 28672 x 8192 (4 bits) 27.0 and 26.0
    if (s.m > 64) return tile_as<T, ABITS, 128, 128>(s, splits_of(s, tiles_of(s, 128, 128), 256), scratch, stream);
    return tile_as<T, ABITS, 64, 64>(s, splits_of(s, tiles_of(s, 64, 64), 512), scratch, stream);
}

}  // namespace

hipError_t launch_product(const guide_product_spec &s, float *scratch, hipStream_t stream) {
    const int key = (int)s.type * 2 + (s.a_bits == 8);
    switch (key) {
        case 0: return product_as<GUIDE_BF16, 4>(s, scratch, stream);
        case 1: return product_as<GUIDE_BF16, 8>(s, scratch, stream);
        case 2: return product_as<GUIDE_F16, 4>(s, scratch, stream);
        case 3: return product_as<GUIDE_F16, 8>(s, scratch, stream);
        case 4: return product_as<GUIDE_F32, 4>(s, scratch, stream);
        default: return hipErrorInvalidValue;                        // (the C ABI refuses it)
    }
}

}  // namespace guide
