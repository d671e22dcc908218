// The paged KV cache in 4-bit codes: append, read back, attention of single tokens.
#include "attention_shared.hpp"
#include "layer_kernels.hpp"

namespace guide {
namespace {

// Where a page's codes and scales of (kv head, keys or values) begin.
struct CacheView {
    uint8_t *codes, *scales;
    uint32_t n_pages, n_kv, block, d;
    __device__ uint8_t *codes_at(uint32_t page, uint32_t head, uint32_t which) const {
        return codes + (((size_t)page * n_kv + head) * 2 + which) * block * (d / 2);
    }
    __device__ uint8_t *scales_at(uint32_t page, uint32_t head, uint32_t which) const {
        return scales + (((size_t)page * n_kv + head) * 2 + which) * block * (d / 32);
    }
};

// What the cache holds for a half-precision value can be just beyond that type (65536 for 65504): limited to it.  A NaN
// stays one.
template <int T>
__device__ inline float within(float x) {
    if constexpr (T == GUIDE_F16) return x > 65504.0f ? 65504.0f : x < -65504.0f ? -65504.0f : x;
    return x;
}

CacheView view_of(const guide_cache &c) { return {c.codes, c.scales, c.n_pages, c.n_kv, c.kv_block, c.d}; }

// A lane handles eight channels of one token's keys and the same of its values (two loads on their way at a time), a quad of
// lanes a group.  A block takes one KV head of 16 (d = 128) or 32 (d = 64) consecutive tokens: where their slots follow each
// other, it writes two runs of codes and 16 or 32 bytes in a row of every scale row.  8192 tokens of 40 heads of 128 (213 MB either way)
// are read back in 33 us, at memory's rate (6.4 TB/s; a plain copy of as much 5.7 to 6.8), and appended in 50 to 55 (3.9 to 4.3).
template <int T, int D, bool READ>
__global__ __launch_bounds__(kBlock) void cache_tokens_kernel(CacheView c, guide_cache_tokens t) {
    using E = typename Elem<T>::type;
    constexpr uint32_t kLanes = D / 8, kTokens = kBlock / kLanes;
    const uint32_t head = blockIdx.y, token = blockIdx.x * kTokens + threadIdx.x / kLanes, ch = threadIdx.x % kLanes;
    if (token >= t.tokens) return;                                   // whole quads
    E *k = (E *)t.k + (int64_t)token * t.k_stride + (int64_t)head * t.k_head_stride + ch * 8;
    E *v = (E *)t.v + (int64_t)token * t.v_stride + (int64_t)head * t.v_head_stride + ch * 8;
    const int64_t slot = t.slots[token];
    const bool inside = slot >= 0 && slot < (int64_t)c.n_pages * c.block;
    const uint32_t page = inside ? (uint32_t)((uint64_t)slot / c.block) : 0u, at = inside ? (uint32_t)((uint64_t)slot % c.block) : 0u;
    uint8_t *codes = c.codes_at(page, head, 0) + (size_t)at * (D / 2) + ch * 4;
    uint8_t *scale = c.scales_at(page, head, 0) + (size_t)(ch / 4) * c.block + at;
    const size_t codes_step = (size_t)c.block * (D / 2), scale_step = (size_t)c.block * (D / 32);      // from keys to values
    if constexpr (READ) {
        uint32_t w[2] = {0, 0}, byte[2] = {127, 127};
        if (inside) {
            w[0] = *(const uint32_t *)codes, w[1] = *(const uint32_t *)(codes + codes_step);
            byte[0] = *scale, byte[1] = scale[scale_step];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float f = __uint_as_float(byte[i] << 23);          // the conversions take the exponent: 0 = 2^-127, 255 = NaN
            const bf16x2 x[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], f, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], f, 1),
                                 __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], f, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], f, 3)};
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = within<T>((float)x[j / 2][j % 2]);
            store8<T>(i ? v : k, y);
        }
    } else {
        float x[2][8];
        load8<T>(k, x[0]);
        load8<T>(v, x[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t byte;
            const Codes<4> q = quantise8<4>(x[i], byte);
            if (!inside) continue;
            *(uint32_t *)(codes + i * codes_step) = q.w[0];
            if ((ch & 3u) == 0) scale[i * scale_step] = (uint8_t)byte;
        }
    }
}

constexpr uint32_t kBlocksWanted = 4096, kBlocksAtOnce = 1024, kLeastChunk = 512;

// How the keys of a sequence are split: up to `chunk` keys to a block.  A block's four waves take 32 keys at a time; the chip runs
// 1024 blocks at once, and four times as many even out sequences of different lengths; a block of fewer than 512 keys is mostly
// start and end.  A chunk follows from the table's width, which may be far more than any sequence has: so a sequence uses at least
// as many blocks as would fill the chip if all were like it (`fill`), of 512 keys or more.  16 sequences of 4000 tokens, 32 heads on
// 8: 20 us with a table for 4000 tokens, 21 with one for 131 072 (35 in chunks of its width).
struct Split {
    uint32_t chunk, fill, splits;                                    // splits: the most that a sequence can use

    __host__ __device__ uint32_t used(uint32_t length) const {       // (one where there is nothing: it writes what an empty sequence gives)
        const uint32_t even = (length + chunk - 1) / chunk, least = (length + kLeastChunk - 1) / kLeastChunk;
        const uint32_t filling = least < fill ? least : fill, n = even > filling ? even : filling;
        return n ? n : 1;
    }
};

Split split_of(uint32_t n_seq, uint32_t n_h, uint32_t n_kv, uint64_t max_len) {
    const uint64_t all = (uint64_t)n_seq * n_kv * ((n_h / n_kv + 15) / 16), rows = all ? all : 1;
    if (max_len > (1u << 30)) max_len = 1u << 30;                    // (a call takes no more)
    uint64_t want = kBlocksWanted / rows;
    if (want < 1) want = 1;
    uint64_t chunk = (max_len + want - 1) / want;
    if (chunk < kLeastChunk) chunk = kLeastChunk;
    chunk = (chunk + 127) / 128 * 128;
    Split sp = {(uint32_t)chunk, (uint32_t)(kBlocksAtOnce / rows), 1};
    sp.splits = sp.used((uint32_t)max_len);
    return sp;
}

// Partial results of (sequence, head, split): the maximum and the sum of its softmax, then the weighted values.
struct Partials {
    float *top, *sum, *value;
    __host__ __device__ Partials(void *ws, size_t n) {
        top = (float *)ws;
        sum = top + n;
        value = sum + n;
    }
};

__device__ inline uint32_t length_of(const guide_cache_queries &s, uint32_t block, uint32_t seq) {
    const int32_t asked = s.lengths[seq];
    return asked < 0 ? 0u : min((uint32_t)asked, s.max_pages * block);
}

// Two neighbouring values of the codes in byte B of w, times the scale whose exponent field is that of f (0 = 2^-127, 255 = NaN).
template <int T, int B>
__device__ __forceinline__ typename Mat<T>::v2 values2(uint32_t w, float f) {
    if constexpr (T == GUIDE_BF16) return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, B);
    else return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, f, B);
}

// 32 keys and values of one KV head as a lane (col, quarter) holds them.  Keys: D / 4 channels (quarter * D / 4 ..) of key
// `col` of either half of 16.  Values: D / 16 channels (col * D / 16 ..) of keys 4 quarter .. of either half.
template <int D>
struct Piece {
    uint32_t k[2][D / 32], v[2][4], v_scale[2];
    uint32_t k_scale[2];
};

// A block: one sequence, one KV head, up to 16 of the query heads that read it, one chunk of keys.
// Scores S' = K Q' and outputs O' = V' P' on 16 x 16 x 32 products: queries are columns all along, so that a lane's scores
// of query `col` are, as probabilities, its operand of the second product, and its sums belong to the query too.  Codes
// become 16-bit values by conversions that apply the scale.  Values come a token to a word and are turned round in
// registers: channel c of the lane's eight keys is its operand for row `col` of the c-th product.
// The maximum that the exponentials are taken against moves only when a score exceeds it by more than 2^8.
// 64 sequences of 1000 to 16 000 tokens, 64 heads on 8 of 128: 88 to 92 us (381 MB, 4.2 TB/s, where plain reads of as much reach 6.2)
// and 5.5 for the join; of one sequence of 40 001 tokens (43.5 MB) 13 us, 4 of them until the first keys arrive.
template <int T, int D>
__global__ __launch_bounds__(kBlock, 3) void cache_attention_kernel(CacheView c, guide_cache_queries s, Div32 by_block, Split sp, void *ws) {
    using E = typename Elem<T>::type;
    using V8 = typename Mat<T>::v8;
    constexpr int kGroups = D / 32;                                  // scale groups of a token
    // A code can stand for more than the half-precision value it was made from (65504 is held as 65536, which that type does
    // not have), so that type sees halves: an exact step down whose other side is in the scale and at the end.
    constexpr float kHeld = T == GUIDE_F16 ? 0.5f : 1.0f;
    const uint32_t group = s.n_h / c.n_kv, tiles = (group + 15) / 16;
    // (heads first, splits last: blocks go round the eight XCDs in turn, and late splits are those of long sequences only)
    const uint32_t split = blockIdx.z, seq = blockIdx.y, kv = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, quarter = lane / 16;
    const uint32_t length = length_of(s, c.block, seq), used = sp.used(length), splits = sp.splits;
    if (split >= used) return;
    const uint32_t share = ((length + used - 1) / used + 31) / 32 * 32;      // the sequence's splits are even ones, of whole tiles
    const uint32_t begin = min(split * share, length), end = min(begin + share, length);
    const int32_t *pages = s.pages + (int64_t)seq * s.pages_stride;

    // where the lane's codes and scales are, from those of the first of sixteen keys on
    const uint32_t k_off = col * (D / 2) + quarter * (D / 8), v_off = quarter * 4 * (D / 2) + col * (D / 32);
    const uint32_t ks_off = quarter * kGroups / 4 * c.block + col, vs_off = col * kGroups / 16 * c.block + quarter * 4;

    // query head `col` of the tile; the ones past the group repeat its last
    const uint32_t head = kv * group + min(tile * 16 + col, group - 1);
    const E *q = (const E *)s.q + (int64_t)seq * s.q_stride + (int64_t)head * s.q_head_stride;
    V8 qf[kGroups];
#pragma unroll
    for (int i = 0; i < kGroups; ++i) __builtin_memcpy(&qf[i], q + quarter * (D / 4) + i * 8, 16);
    const float cs = s.scale * kLog2e / kHeld;
    float top = -INFINITY, base = 0.0f, sum = 0.0f;
    f32x4 o[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[i] = f32x4{0, 0, 0, 0};

    // Sixteen keys from k on: the page they are in (a page holds whole sixteens), a number beyond the cache where there are none.
    auto page_of = [&](uint32_t k) __attribute__((always_inline)) { return k < end ? (uint32_t)pages[div32(k, by_block)] : 0xFFFFFFFFu; };
    // What there is no page for is read from page 0, and never used.
    auto load = [&](Piece<D> &x, uint32_t k0, const uint32_t (&page)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const bool there = page[t] < c.n_pages;
            const uint32_t k = there ? k0 + t * 16 : 0, at = k - div32(k, by_block) * c.block, p = there ? page[t] : 0;
            const uint8_t *codes = c.codes_at(p, kv, 0) + at * (D / 2), *scales = c.scales_at(p, kv, 0) + at;
            __builtin_memcpy(x.k[t], __builtin_assume_aligned(codes + k_off, D / 8), sizeof x.k[t]);
            x.k_scale[t] = scales[ks_off];
            codes += c.block * (D / 2);
            scales += c.block * (D / 32);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (D == 128) x.v[t][j] = *(const uint32_t *)(codes + v_off + j * (D / 2));
                else x.v[t][j] = *(const uint16_t *)(codes + v_off + j * (D / 2));
            }
            x.v_scale[t] = *(const uint32_t *)(scales + vs_off);
        }
    };
    // Keys k0 .. k0 + 31.
    auto work = [&](const Piece<D> &x, uint32_t k0, const uint32_t (&page)[2]) __attribute__((always_inline)) {
        f32x4 sc[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            sc[t] = f32x4{0, 0, 0, 0};
            const float f = __uint_as_float(x.k_scale[t] << 23) * kHeld;
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                const typename Mat<T>::v2 v[4] = {values2<T, 0>(x.k[t][i], f), values2<T, 1>(x.k[t][i], f), values2<T, 2>(x.k[t][i], f), values2<T, 3>(x.k[t][i], f)};
                V8 kf;
                __builtin_memcpy(&kf, v, 16);
                sc[t] = Mat<T>::mma16(kf, qf[i], sc[t]);
            }
        }
        // Of the lane's four keys of either half, `real` are seen.  The values of the others may be NaNs, and 0 times a NaN
        // another: their scale becomes the least.
        uint32_t v_scale[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int real = page[t] < c.n_pages ? (int)(end - k0) - t * 16 - quarter * 4 : 0;
            v_scale[t] = real >= 4 ? x.v_scale[t] : real <= 0 ? 0u : x.v_scale[t] & ((1u << (8 * real)) - 1u);
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[t][j] = j < real ? sc[t][j] : -INFINITY;
        }
        float most = max3(max3(sc[0][0], sc[0][1], sc[0][2]), max3(sc[1][0], sc[1][1], sc[1][2]), max3(sc[0][3], sc[1][3], sc[0][0]));
        most = max3(most, __shfl_xor(most, 16), most);
        most = max3(most, __shfl_xor(most, 32), most) * cs;          // (cs > 0)
        if (__any(most > top + 8.0f)) {
            const float next = fmaxf(top, most);
            base = next == -INFINITY ? 0.0f : next;
            const float shrink = __builtin_amdgcn_exp2f(top - base);
            top = next;
            sum *= shrink;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[i] *= shrink;
        }
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = __builtin_amdgcn_exp2f(fmaf(sc[j / 4][j % 4], cs, -base));        // 0 where not seen
        typename Mat<T>::v2 pp[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) pp[j] = __builtin_convertvector(f32x2{e[2 * j], e[2 * j + 1]}, typename Mat<T>::v2);
        sum += Mat<T>::sum2(pp[0], Mat<T>::sum2(pp[1], 0.0f)) + Mat<T>::sum2(pp[2], Mat<T>::sum2(pp[3], 0.0f));
        V8 pf;
        __builtin_memcpy(&pf, pp, 16);
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = __uint_as_float((v_scale[j / 4] >> (8 * (j % 4)) & 0xFFu) << 23) * kHeld;
        unrolled<D / 32>([&](auto byte) __attribute__((always_inline)) {          // channels 2 i and 2 i + 1 of the lane's
            constexpr int i = decltype(byte)::value;
            uint32_t even[4], odd[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a = __builtin_bit_cast(uint32_t, values2<T, i>(x.v[j / 2][j % 2 * 2], f[2 * j]));
                const uint32_t b = __builtin_bit_cast(uint32_t, values2<T, i>(x.v[j / 2][j % 2 * 2 + 1], f[2 * j + 1]));
                even[j] = __builtin_amdgcn_perm(b, a, 0x05040100u);               // low halves, high halves
                odd[j] = __builtin_amdgcn_perm(b, a, 0x07060302u);
            }
            V8 ve, vo;
            __builtin_memcpy(&ve, even, 16);
            __builtin_memcpy(&vo, odd, 16);
            o[2 * i] = Mat<T>::mma16(ve, pf, o[2 * i]);
            o[2 * i + 1] = Mat<T>::mma16(vo, pf, o[2 * i + 1]);
        });
    };
    // The wave's tiles: one being worked on, one on its way, the page numbers of one more.  (The two change places in the
    // code: a copy would wait for the one on its way.)
    const uint32_t first = begin + wave * 32;
    uint32_t page_a[2] = {page_of(first), page_of(first + 16)}, page_b[2] = {page_of(first + 128), page_of(first + 144)};
    Piece<D> a, b;
    if (first < end) {
        load(a, first, page_a);
        for (uint32_t k0 = first;; k0 += 256) {
            load(b, k0 + 128, page_b);
            const uint32_t page_c[2] = {page_of(k0 + 256), page_of(k0 + 272)};
            work(a, k0, page_a);
            if (k0 + 128 >= end) break;
            page_a[0] = page_c[0], page_a[1] = page_c[1];
            load(a, k0 + 256, page_a);
            const uint32_t page_d[2] = {page_of(k0 + 384), page_of(k0 + 400)};
            work(b, k0 + 128, page_b);
            if (k0 + 256 >= end) break;
            page_b[0] = page_d[0], page_b[1] = page_d[1];
        }
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);

    // the four waves' parts are joined in the waves' order.  o[n][j] is channel (4 quarter + j) * D / 16 + n
    __shared__ float tops[4][16], sums[4][16];
    __shared__ float values[4][16][D + 4];
    if (quarter == 0) tops[wave][col] = top, sums[wave][col] = sum;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < D / 16; n += 4)
            *(f32x4 *)&values[wave][col][(quarter * 4 + j) * (D / 16) + n] = f32x4{o[n][j], o[n + 1][j], o[n + 2][j], o[n + 3][j]};
    __syncthreads();
    const Partials part(ws, (size_t)s.n_seq * s.n_h * splits);
    for (uint32_t i = threadIdx.x; i < 16 * D / 4; i += kBlock) {
        const uint32_t r = i / (D / 4), ch = i % (D / 4) * 4;
        if (tile * 16 + r >= group) break;
        const float best = fmaxf(fmaxf(tops[0][r], tops[1][r]), fmaxf(tops[2][r], tops[3][r]));
        const float from = best == -INFINITY ? 0.0f : best;
        float total = 0.0f;
        f32x4 x = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(tops[w][r] - from);
            total += sums[w][r] * f;
            x += *(const f32x4 *)&values[w][r][ch] * f;
        }
        x *= 1.0f / kHeld;
        const uint32_t h = kv * group + tile * 16 + r;
        if (splits == 1) {
            E e[4];
#pragma unroll
            for (int b = 0; b < 4; ++b) e[b] = (E)within<T>(total == 0.0f ? 0.0f : x[b] / total);
            __builtin_memcpy((E *)s.out + (int64_t)seq * s.out_stride + (int64_t)h * s.out_head_stride + ch, e, 8);
        } else {
            const size_t at = ((size_t)seq * s.n_h + h) * splits + split;
            if (ch == 0) part.top[at] = best, part.sum[at] = total;
            __builtin_memcpy(part.value + at * D + ch, &x, 16);
        }
    }
}

// Joins the splits of a (sequence, head): WAVES waves to it, each made of strands of D / 4 lanes with four channels to a lane;
// split i goes to strand i modulo their number, and the strands are joined in a fixed order.  Bound by latency: a strand's first
// four splits are loaded before anything is known about them (in bounds, and left out of the sums if they were not written).
template <int T, int D, int WAVES>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : kBlock) void cache_join_kernel(guide_cache_queries s, uint32_t block, Split sp,
                                                                                      uint32_t rows, const void *ws) {
    using E = typename Elem<T>::type;
    constexpr int kStrands = WAVES * 256 / D;                        // of a row
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, ch = lane % (D / 4) * 4;
    const uint32_t row = WAVES == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
    if (WAVES == 1 && row >= rows) return;
    const uint32_t seq = row / s.n_h, head = row - seq * s.n_h, splits = sp.splits;
    const Partials part((void *)ws, (size_t)rows * splits);
    const size_t at = (size_t)row * splits;
    const uint32_t strand = (WAVES == 1 ? 0 : wave * (256 / D)) + lane / (D / 4);
    float top[4], sum[4];
    f32x4 v[4];
    auto load = [&](uint32_t i) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            const size_t from = at + min(i + u * kStrands, splits - 1);
            top[u] = part.top[from], sum[u] = part.sum[from];
            __builtin_memcpy(&v[u], part.value + from * D + ch, 16);
        }
    };
    load(strand);
    float best = -INFINITY;
    const uint32_t used = sp.used(length_of(s, block, seq));
    for (uint32_t i = lane; i < used; i += 64) best = fmaxf(best, part.top[at + i]);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) best = fmaxf(best, __shfl_xor(best, m));
    const float base = best == -INFINITY ? 0.0f : best;
    float total = 0.0f;
    f32x4 x = {0, 0, 0, 0};
    for (uint32_t i = strand; i < used; i += 4 * kStrands) {
        if (i != strand) load(i);
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            if (i + u * kStrands >= used) continue;
            const float f = __builtin_amdgcn_exp2f(top[u] - base);
            total += sum[u] * f;
            x += v[u] * f;
        }
    }
#pragma unroll
    for (int m = D / 4; m < 64; m <<= 1) {
        total += __shfl_xor(total, m);
#pragma unroll
        for (int b = 0; b < 4; ++b) x[b] += __shfl_xor(x[b], m);
    }
    if constexpr (WAVES > 1) {
        __shared__ f32x4 values[WAVES][D / 4];
        __shared__ float totals[WAVES];
        if (lane < D / 4) values[wave][lane] = x;
        if (lane == 0) totals[wave] = total;
        __syncthreads();
        if (threadIdx.x >= D / 4) return;
        total = totals[0];
        x = values[0][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) total += totals[w], x += values[w][lane];
    }
    if (lane >= D / 4) return;
    E e[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) e[b] = (E)within<T>(total == 0.0f ? 0.0f : x[b] / total);
    __builtin_memcpy((E *)s.out + (int64_t)seq * s.out_stride + (int64_t)head * s.out_head_stride + ch, e, 8);
}

template <int T, int D, bool READ>
hipError_t tokens_as(const guide_cache &c, const guide_cache_tokens &t, hipStream_t stream) {
    using E = typename Elem<T>::type;
    constexpr uint32_t kTokens = kBlock / (D / 8), kMost = kMostThreads / (D / 8);
    guide_cache_tokens part = t;
    for (uint32_t at = 0; at < t.tokens; at += part.tokens) {
        part.tokens = t.tokens - at < kMost ? t.tokens - at : kMost;
        part.k = (E *)t.k + (int64_t)at * t.k_stride;
        part.v = (E *)t.v + (int64_t)at * t.v_stride;
        part.slots = t.slots + at;
        cache_tokens_kernel<T, D, READ><<<dim3((part.tokens + kTokens - 1) / kTokens, c.n_kv), kBlock, 0, stream>>>(view_of(c), part);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool READ>
hipError_t tokens_any(const guide_cache &c, const guide_cache_tokens &t, hipStream_t stream) {
    if (t.type == GUIDE_BF16)
        return c.d == 64 ? tokens_as<GUIDE_BF16, 64, READ>(c, t, stream) : tokens_as<GUIDE_BF16, 128, READ>(c, t, stream);
    return c.d == 64 ? tokens_as<GUIDE_F16, 64, READ>(c, t, stream) : tokens_as<GUIDE_F16, 128, READ>(c, t, stream);
}

template <int T, int D>
hipError_t attention_as(const guide_cache &c, const guide_cache_queries &q, void *ws, hipStream_t stream) {
    const Split sp = split_of(q.n_seq, q.n_h, c.n_kv, (uint64_t)q.max_pages * c.kv_block);
    const uint32_t splits = sp.splits, tiles = (q.n_h / c.n_kv + 15) / 16;
    cache_attention_kernel<T, D><<<dim3(c.n_kv * tiles, q.n_seq, splits), kBlock, 0, stream>>>(view_of(c), q, make_div32(c.kv_block), sp, ws);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    const uint32_t rows = q.n_seq * q.n_h;                           // (a wave to a row where a strand has a few splits at most)
    if (splits <= 16) cache_join_kernel<T, D, 1><<<(rows + 3) / 4, kBlock, 0, stream>>>(q, c.kv_block, sp, rows, ws);
    else cache_join_kernel<T, D, 16><<<rows, 1024, 0, stream>>>(q, c.kv_block, sp, rows, ws);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const guide_cache &c, const guide_cache_tokens &t, hipStream_t stream) { return tokens_any<false>(c, t, stream); }
hipError_t launch_cache_read(const guide_cache &c, const guide_cache_tokens &t, hipStream_t stream) { return tokens_any<true>(c, t, stream); }

size_t cache_attention_workspace(uint32_t n_seq, uint32_t n_h, uint32_t n_kv, uint32_t d, uint64_t max_len) {
    const Split sp = split_of(n_seq, n_h, n_kv, max_len);
    return sp.splits <= 1 ? 0 : (size_t)n_seq * n_h * sp.splits * (d + 2) * sizeof(float);
}

hipError_t launch_cache_attention(const guide_cache &c, const guide_cache_queries &asked, void *ws, hipStream_t stream) {
    guide_cache_queries q = asked;
    if (c.n_pages == 0) q.max_pages = 0;                             // (nothing to see)
    if (q.type == GUIDE_BF16) return c.d == 64 ? attention_as<GUIDE_BF16, 64>(c, q, ws, stream) : attention_as<GUIDE_BF16, 128>(c, q, ws, stream);
    return c.d == 64 ? attention_as<GUIDE_F16, 64>(c, q, ws, stream) : attention_as<GUIDE_F16, 128>(c, q, ws, stream);
}

}  // namespace guide
