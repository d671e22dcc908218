// Causal attention over packed sequences.
#include <type_traits>

#include "attention_shared.hpp"
#include "layer_kernels.hpp"
#include "staging.hpp"

namespace guide {
namespace {

constexpr int kRowsPerWave = 32;

// How the keys of a sequence are split over blocks: into as many parts as `size` goes into the number of keys that its queries see on
// average, at most `most` of them, or `many` where it has several tiles of queries.
struct Cut {
    Div32 size;
    uint32_t most, many;
    __device__ uint32_t parts(uint32_t nq, uint32_t nk) const {
        const uint32_t seen = nk > nq / 2 ? nk - nq / 2 : 0;
        return max(1u, min(div32(seen, size), nq > 4 * kRowsPerWave ? many : most));
    }
};

__device__ inline uint32_t clamped(int32_t v, uint32_t total) { return v < 0 ? 0u : (uint32_t)v > total ? total : (uint32_t)v; }

// A lane's sequence.  Units of work: a tile of ceil(n_q / ROWS), or as many as a tile has parts.
template <int ROWS, bool SPLIT>
struct Sequence {
    uint32_t q0 = 0, nq = 0, k0 = 0, nk = 0, parts = 1, units = 0;
    __device__ Sequence(const guide_prompt_spec &s, const Cut &cut, uint32_t i) {
        if (i >= s.n_seq) return;                                    // (all four starts in one trip to memory)
        q0 = clamped(s.q_starts[i], s.total_q);
        k0 = clamped(s.k_starts[i], s.total_k);
        const uint32_t q1 = clamped(s.q_starts[i + 1], s.total_q), k1 = clamped(s.k_starts[i + 1], s.total_k);
        nq = q1 > q0 ? q1 - q0 : 0, nk = k1 > k0 ? k1 - k0 : 0;
        if (SPLIT && nq) parts = cut.parts(nq, nk);
        units = (nq + ROWS - 1) / ROWS * parts;
    }
};

// Units before every 64 sequences, for calls of so many of them that a walk over them in every block takes longer than this kernel does; the
// last entry is the number of all.  Walked / by the table, a query over one key each, 8 heads of 64: 256 sequences 14.1 / 15.7 us, 512
// 27.3 / 24.5, 4096 565 / 148; 2048 over 50 keys each, 32 heads of 128, 1572 / 703.
constexpr uint32_t kMostSequences = 1u << 20, kWalked = 384, kTable = kMostSequences / 64 + 64;
template <int ROWS, bool SPLIT>
__global__ __launch_bounds__(1024) void prompt_table_kernel(guide_prompt_spec s, Cut cut, uint32_t *table) {
    constexpr uint32_t kEach = kMostSequences / 64 / 1024;           // entries of a thread, one after the other
    __shared__ uint32_t units[kMostSequences / 64], sums[16];
    const uint32_t chunks = (s.n_seq + 63) / 64, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    for (uint32_t c = wave; c < chunks; c += 16) {
        uint32_t sum = Sequence<ROWS, SPLIT>(s, cut, c * 64 + lane).units;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
        if (lane == 0) units[c] = sum;
    }
    __syncthreads();
    uint32_t mine[kEach], own = 0;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t c = threadIdx.x * kEach + i;
        mine[i] = own;
        own += c < chunks ? units[c] : 0;
    }
    uint32_t upto = own;                                             // running sums over the threads
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const uint32_t o = __shfl_up(upto, m);
        if (lane >= (uint32_t)m) upto += o;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    uint32_t before = upto - own;
    for (uint32_t w = 0; w < wave; ++w) before += sums[w];
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t c = threadIdx.x * kEach + i;
        if (c < chunks) table[c] = before + mine[i];
    }
    if (threadIdx.x == 1023) table[chunks] = before + own;
}

// The sequence, the tile in it and the part of its keys that unit number `unit` of the packed queries is; false when there are
// fewer units.  Every lane of a wave looks at one sequence at a time.
struct Place { uint32_t q0, nq, k0, nk, tile, part, parts; };

template <int ROWS, bool SPLIT>
__device__ inline bool find_unit(const guide_prompt_spec &s, const Cut &cut, const uint32_t *table, uint32_t unit, Place &p) {
    const uint32_t lane = threadIdx.x % 64;
    uint32_t before = 0, s0 = 0;
    if (table) {                                                     // the last 64 sequences that begin at the unit or before it
        uint32_t end = (s.n_seq + 63) / 64;
        if (unit >= table[end]) return false;
        while (end - s0 > 1) {
            const uint32_t mid = (s0 + end) / 2;
            if (table[mid] <= unit) s0 = mid;
            else end = mid;
        }
        before = table[s0];
        s0 *= 64;
    }
    for (; s0 < s.n_seq; s0 += 64) {
        const Sequence<ROWS, SPLIT> q(s, cut, s0 + lane);
        uint32_t sum = q.units;                                      // running sum over the lanes
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const uint32_t o = __shfl_up(sum, m);
            if ((int)lane >= m) sum += o;
        }
        const uint64_t past = __ballot(before + sum > unit);
        if (past) {
            const int w = __builtin_ctzll(past);
            auto of = [&](uint32_t x) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readlane((int)x, w); };
            p.q0 = of(q.q0), p.nq = of(q.nq), p.k0 = of(q.k0), p.nk = of(q.nk);
            p.tile = unit - (before + of(sum - q.units)), p.part = 0, p.parts = 1;
            if constexpr (SPLIT) {
                p.parts = of(q.parts);
                p.part = p.tile % p.parts, p.tile /= p.parts;
            }
            return true;
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
    }
    return false;
}

// 64 rows of D elements on their way to LDS, in which a row's 16-byte pieces are permuted: an instruction of a wave lays down
// 1024 bytes in the lanes' order, so that the permutation is on the memory's side.
template <int D, bool KEYS, int WAVES>
struct Sender : KeyPlaces<D, KEYS, WAVES> {
    using Places = KeyPlaces<D, KEYS, WAVES>;
    const uint8_t *next;                                             // the tile that is sent next, and the rows from it on
    int64_t stride;                                                  // bytes
    int left;

    __device__ __forceinline__ void init(const void *first, int64_t row_stride, int rows, int wave, int lane) {
        stride = row_stride * 2;
        next = (const uint8_t *)first + (int64_t)(wave * Places::kRows) * stride;
        left = rows - wave * Places::kRows;
        Places::init(stride, wave, lane);
    }
    // The wave's rows of a tile.  The buffer ends with the sequence's last row and answers what lies beyond with zeros.
    __device__ __forceinline__ void send(uint8_t *lds, int wave) {
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)next, 0, (int)Places::bytes(left, stride), 0x00020000);
#pragma unroll
        for (int i = 0; i < Places::kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(lds + (wave * Places::kLoads + i) * 1024), 16,
                                                     (int)Places::of_lane(i, stride), 0, 0, 0);
        next += kTileK * stride;
        left -= kTileK;
    }
};

// A wave's 32 queries of one head.  With the scores transposed, S' = K Q', a lane holds scores of one query (lane % 32) against
// runs of four keys, which is the layout in which O' = V' P' takes its second operand, up to an order of the keys that the
// reads of V follow: the probabilities never leave their registers.
// The maximum that the exponentials are taken against moves only when a score exceeds it by more than 2^kSlack, which saves
// most tiles the rescaling of O; the sums stay exact, as numerator and denominator share it.
constexpr float kSlack = 8.0f;

template <int T, int D>
struct Rows {
    using E = typename Elem<T>::type;
    using V8 = typename Mat<T>::v8;
    static constexpr int kRow = D * 2;                               // bytes of a staged row
    V8 q[D / 16], p[4];
    f32x16 o[D / 32], sc[2];
    float c, top, base, sum;                                         // base: top, or 0 while nothing is seen
    int lane, half, sees;                                            // the row sees keys 0 .. sees - 1 (none when negative)

    __device__ __forceinline__ void init(const E *row_q, float scale, int lane_, int sees_) {
        lane = lane_, half = lane_ / 32, sees = sees_;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) __builtin_memcpy(&q[i], row_q + i * 16 + half * 8, 16);
        c = scale * kLog2e;
        top = -INFINITY, base = 0.0f, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
    }

    // Scores of a tile; score j of half t of it is key 32 t + 8 (j / 4) + 4 half + j % 4.
    __device__ __forceinline__ void scores(const uint8_t *lds_k) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int j = 0; j < 16; ++j) sc[t][j] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int r = t * 32 + lane % 32;
                const V8 kf = *(const V8 *)(lds_k + r * kRow + piece_of<D, true>(r, i * 2 + half) * 16);
                sc[t] = Mat<T>::mma32(kf, q[i], sc[t]);
            }
    }

    // The scores' exponentials, as the second product's operand.  MASKED: not every row of the wave sees all keys k0 ..
    template <bool MASKED>
    __device__ __forceinline__ void exponentials(int k0) {
        if constexpr (MASKED) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (k0 + 32 * t + 8 * (j / 4) + 4 * half + j % 4 >= sees) sc[t][j] = -INFINITY;
        }
        float best[4];                                               // (four chains)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            best[u] = max3(sc[u / 2][u % 2 * 8], sc[u / 2][u % 2 * 8 + 1], sc[u / 2][u % 2 * 8 + 2]);
#pragma unroll
            for (int j = 3; j < 7; j += 2) best[u] = max3(best[u], sc[u / 2][u % 2 * 8 + j], sc[u / 2][u % 2 * 8 + j + 1]);
        }
        float most = max3(max3(best[0], best[1], sc[0][7]), max3(best[2], best[3], sc[0][15]), max3(sc[1][7], sc[1][15], best[0]));
        most = fmaxf(most, __shfl_xor(most, 32)) * c;                // (c > 0)
        if (__any(most > top + kSlack)) {
            const float next = fmaxf(top, most);
            base = next == -INFINITY ? 0.0f : next;
            const float shrink = __builtin_amdgcn_exp2f(top - base);
            top = next;
            sum *= shrink;
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[i][j] *= shrink;
        }
        typename Mat<T>::v2 pp[16];
        float part_sum[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            const float e0 = __builtin_amdgcn_exp2f(fmaf(sc[j / 16][j % 16], c, -base));          // 0 where masked
            const float e1 = __builtin_amdgcn_exp2f(fmaf(sc[j / 16][j % 16 + 1], c, -base));
            pp[j / 2] = __builtin_convertvector(f32x2{e0, e1}, typename Mat<T>::v2);
            part_sum[j / 8] = Mat<T>::sum2(pp[j / 2], part_sum[j / 8]);
        }
        sum += (part_sum[0] + part_sum[1]) + (part_sum[2] + part_sum[3]);
        __builtin_memcpy(p, pp, sizeof p);
    }

    // A value that is no finite number reaches the rows that see its key and no others: 0 times it would be a NaN.  Adds the products
    // with those of keys k0 .. that the row sees; values<true> leaves them out.
    __device__ __forceinline__ void add_odd(int k0, const uint8_t *lds_v) {
        uint32_t pairs[16];
        __builtin_memcpy(pairs, p, sizeof pairs);
        for (int r = 0; r < kTileK; ++r) {
            const int j = r / 8 * 4 + r % 4;                         // the key's probability is number j of half r / 4 % 2
            uint32_t pair = pairs[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) pair = j / 2 == i ? pairs[i] : pair;
            const auto two = __builtin_bit_cast(typename Mat<T>::v2, pair);
            const float weight = __shfl((float)(j % 2 ? two[1] : two[0]), lane % 32 + r / 4 % 2 * 32);
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int a = 0; a < 4; ++a) {                        // channels 32 i + 8 a + 4 half ..
                    E x[4];
                    __builtin_memcpy(x, lds_v + r * kRow + piece_of<D, false>(r, i * 4 + a) * 16 + half * 8, 8);
#pragma unroll
                    for (int b = 0; b < 4; ++b)
                        if (k0 + r < sees && !__builtin_isfinite((float)x[b])) o[i][a * 4 + b] += weight * (float)x[b];
                }
        }
    }

    // O' += V' P'.  V' of channels 32 i .. comes by transposing reads: a group of 16 lanes reads four keys' 16 channels and gets,
    // per lane, one channel of the four keys.
    template <bool MASKED>
    __device__ __forceinline__ void values(const uint8_t *lds_v, bool odd) {
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                i16x4 part[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int r = 16 * w + 8 * u + 4 * half + (lane % 16) / 4;
                    const int at = r * kRow + piece_of<D, false>(r, i * 4 + (lane % 32) / 16 * 2) * 16 + (lane % 4) * 8;
                    part[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(lds_v + at));
                }
                if (MASKED && odd) {
                    uint32_t x[4];
                    __builtin_memcpy(x, part, 16);
#pragma unroll
                    for (int b = 0; b < 4; ++b) x[b] = finite_or_zero<T>(x[b]);
                    __builtin_memcpy(part, x, 16);
                }
                V8 vf;
                __builtin_memcpy(&vf, part, 16);
                o[i] = Mat<T>::mma32(vf, p[w], o[i]);
            }
    }

    // N reads ahead of the products that need them (READS reads to a product), for a stretch of D / 8 products.
    template <int N, int READS>
    static __device__ __forceinline__ void reads_ahead() {
        __builtin_amdgcn_sched_group_barrier(0x100, N * READS, 0);
#pragma unroll
        for (int i = 0; i < D / 8 - N; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, N, 0);
    }

    // The same without the division, for keys that are split over blocks.
    __device__ __forceinline__ void finish_part(float *tops, float *sums, float *values) {
        sum += __shfl_xor(sum, 32);
        if (!tops) return;
        if (half == 0) *tops = top, *sums = sum;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int a = 0; a < 4; ++a) __builtin_memcpy(values + i * 32 + a * 8 + half * 4, (const float *)&o[i] + a * 4, 16);
    }

    __device__ __forceinline__ void finish(E *out) {
        sum += __shfl_xor(sum, 32);
        const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                E e[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) e[b] = (E)(sum != 0.0f ? o[i][a * 4 + b] * inv : 0.0f);
                if (out) __builtin_memcpy(out + i * 32 + a * 8 + half * 4, e, 8);
            }
    }
};

// What a block works on: one head's queries of one tile, and a part of the keys.  Late tiles, which see the most keys, come first.
// Blocks go round the eight XCDs in turn: with a multiple of eight KV heads, the query heads of one KV head stay on one XCD, whose L2
// then holds its keys once.
template <int ROWS, bool SPLIT>
__device__ __forceinline__ bool find_work(const guide_prompt_spec &s, const Cut &cut, const uint32_t *table, uint32_t units, Place &p, uint32_t &head, uint32_t &kv) {
    const uint32_t group = s.n_h / s.n_kv;
    uint32_t unit;
    if (s.n_kv % 8 == 0) {
        const uint32_t per = s.n_h / 8, x = blockIdx.x / 8, h = x % per;
        head = (blockIdx.x % 8 + 8 * (h / group)) * group + h % group;
        unit = x / per;
    } else {
        head = blockIdx.x % s.n_h;
        unit = blockIdx.x / s.n_h;
    }
    kv = head / group;
    return find_unit<ROWS, SPLIT>(s, cut, table, units - 1 - unit, p);
}

// Whether the wave's part of a staged tile of values, which it sent for itself, holds an infinity or a NaN.
template <int T, int LOADS>
__device__ __forceinline__ uint32_t looks_odd(const uint8_t *lds_v, int wave, int lane) {
    uint32_t some = 0;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const uint4 x = *(const uint4 *)(lds_v + (wave * LOADS + i) * 1024 + lane * 16);
        some |= not_finite<T>(x.x) | not_finite<T>(x.y) | not_finite<T>(x.z) | not_finite<T>(x.w);
    }
    return __any(some != 0);
}
template <int WAVES>
__device__ __forceinline__ bool any_of(const uint32_t (&flags)[WAVES]) {
    uint32_t any = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) any |= flags[w];
    return __builtin_amdgcn_readfirstlane(any) != 0;
}

__device__ __forceinline__ void arrived() { __builtin_amdgcn_s_waitcnt(0x0070); }     // the wave's loads and reads are done
__device__ __forceinline__ void meet() { __builtin_amdgcn_s_barrier(); }

// Results of parts of a row's keys: the maximum and the sum of the softmax, then the weighted values.  Row `r` of part `i` is number
// i rows + r, where rows = total_q n_h.
struct Parts {
    float *top, *sum, *value;
    uint64_t rows;
    __host__ __device__ Parts(float *scratch, uint64_t rows_, uint32_t parts) : top(scratch), sum(top + rows_ * parts), value(sum + rows_ * parts), rows(rows_) {}
};

// Four waves take 128 queries of one head, a wave 32 of them; the keys come in tiles of 64 through LDS, the next tile on its
// way while one is worked on.  Two such blocks share a compute unit, so that one's exponentials run beside the other's products
// (48 % of the matrix units' cycles in a pass of six prompts of 300 to 3900 tokens, 64 heads on 8 of 128: 434 us, 890 TFLOP/s of
// visible pairs, and 3 % in vain in tiles that are partly masked; the waves of a block wait for its last one there).
// SPLIT: a sequence of many keys gives every tile so many blocks, each of which takes its part of the keys that any of the queries sees,
// and prompt_join_kernel joins the parts.
template <int T, int D, bool SPLIT>
__global__ __launch_bounds__(256, 2) void prompt_kernel(guide_prompt_spec s, uint32_t units, Cut cut, const uint32_t *table, float *scratch) {
    using E = typename Elem<T>::type;
    constexpr int kRow = D * 2, kTileQ = 4 * kRowsPerWave;
    using SendK = Sender<D, true, 4>;
    using SendV = Sender<D, false, 4>;
    __shared__ __align__(16) uint8_t lds_k0[kTileK * kRow], lds_v0[kTileK * kRow], lds_k1[kTileK * kRow], lds_v1[kTileK * kRow];
    __shared__ uint32_t odd0[4], odd1[4];
    Place p;
    uint32_t head, kv;
    if (!find_work<kTileQ, SPLIT>(s, cut, table, units, p, head, kv)) return;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int first = (int)(p.tile * kTileQ) + wave * kRowsPerWave, row = first + lane % 32;      // queries of the sequence
    const int nq = (int)p.nq, nk = (int)p.nk, shift = nk - nq;
    const int wave_last = first < nq ? min(first + kRowsPerWave, nq) + shift : 0;   // keys that any row of the wave sees
    int last = min((int)p.tile * kTileQ + kTileQ, nq) + shift;                      // ... any row of the block
    int k0 = 0;
    if constexpr (SPLIT) {
        const int part = (max(last, 0) / (int)p.parts + 2 * kTileK) / (2 * kTileK) * (2 * kTileK);      // whole pairs of tiles
        k0 = min((int)p.part * part, (max(last, 0) + 2 * kTileK - 1) / (2 * kTileK) * (2 * kTileK));
        last = min(last, k0 + part);
    }

    SendK send_k;
    SendV send_v;
    send_k.init((const E *)s.k + ((int64_t)p.k0 + k0) * s.k_stride + (int64_t)kv * s.k_head_stride, s.k_stride, nk - k0, wave, lane);
    send_v.init((const E *)s.v + ((int64_t)p.k0 + k0) * s.v_stride + (int64_t)kv * s.v_head_stride, s.v_stride, nk - k0, wave, lane);
    Rows<T, D> rows;

    auto step = [&](const uint8_t *lds_k, const uint8_t *lds_v, uint8_t *next_k, uint8_t *next_v) __attribute__((always_inline)) {
        arrived();
        meet();
        send_k.send(next_k, wave);
        send_v.send(next_v, wave);
        rows.scores(lds_k);
        Rows<T, D>::template reads_ahead<6, 1>();
        __builtin_amdgcn_s_setprio(1);                               // (of two waves on a SIMD, the one that holds up its next products)
        rows.template exponentials<false>(0);
        __builtin_amdgcn_s_setprio(0);
        rows.template values<false>(lds_v, false);
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);           // the first eight reads before the exponentials
        __builtin_amdgcn_sched_group_barrier(0x406, 140, 0);
#pragma unroll
        for (int i = 0; i < D / 8 - 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    };
    auto masked_step = [&](int k0, const uint8_t *lds_k, const uint8_t *lds_v, uint8_t *next_k, uint8_t *next_v, uint32_t (&odd)[4]) __attribute__((always_inline)) {
        arrived();
        odd[wave] = looks_odd<T, SendV::kLoads>(lds_v, wave, lane);
        arrived();
        meet();
        send_k.send(next_k, wave);
        send_v.send(next_v, wave);
        if (k0 >= wave_last) return;
        rows.scores(lds_k);
        Rows<T, D>::template reads_ahead<6, 1>();
        rows.template exponentials<true>(k0);
        const bool bad = any_of(odd);
        if (bad) rows.add_odd(k0, lds_v);
        rows.template values<true>(lds_v, bad);
    };
    send_k.send(lds_k0, wave);
    send_v.send(lds_v0, wave);
    rows.init((const E *)s.q + (int64_t)(p.q0 + min(row, nq - 1)) * s.q_stride + (int64_t)head * s.q_head_stride, s.scale, lane,
              min(row + shift + 1, nk));
    // Tiles that every row of the block sees come two at a time; an odd one among them goes with the masked ones.  (A loop of its
    // own for it gains nothing: the third copy costs the others registers.)
    int full = max(((int)p.tile * kTileQ + shift + 1) / (2 * kTileK) * (2 * kTileK), 0);
    if constexpr (SPLIT) full = min(full, last);                     // (`last` is a whole pair's end, or beyond the full ones)
    for (; k0 < full; k0 += 2 * kTileK) {
        step(lds_k0, lds_v0, lds_k1, lds_v1);
        step(lds_k1, lds_v1, lds_k0, lds_v0);
    }
    for (; k0 < last; k0 += 2 * kTileK) {
        masked_step(k0, lds_k0, lds_v0, lds_k1, lds_v1, odd0);
        if (k0 + kTileK >= last) break;
        masked_step(k0 + kTileK, lds_k1, lds_v1, lds_k0, lds_v0, odd1);
    }
    arrived();                                                       // (no load may be on its way to the LDS of a block that has ended)
    if (SPLIT && p.parts > 1) {
        const Parts parts(scratch, (uint64_t)s.total_q * s.n_h, cut.most);
        const uint64_t at = p.part * parts.rows + (uint64_t)(p.q0 + row) * s.n_h + head;
        const bool real = row < nq;
        rows.finish_part(real ? parts.top + at : nullptr, parts.sum + at, parts.value + at * D);
    } else {
        rows.finish(row < nq ? (E *)s.out + (int64_t)(p.q0 + row) * s.out_stride + (int64_t)head * s.out_head_stride : nullptr);
    }
}

// Eight waves take 256 queries, in two groups of four (one wave of each on every SIMD) that take turns: while one group
// multiplies -- the values of its last tile, the scores of its next --, the other takes exponentials, so that matrix and
// vector units work side by side.  Both groups meet after every turn; group 1 is one turn behind.  Turn 2 t, of which group 0's
// products are of tile t, sends for the keys of tile t + 1 and the values of tile t, which are needed from turn 2 t + 2 on.
// 8192 queries over 32 768 keys, 32 heads on 8: 3150 to 3310 us, 1160 to 1220 TFLOP/s, 65 % of the matrix units' cycles; the
// group at its exponentials has more instructions to issue than the other's products leave room for.
template <int T, int D>
__global__ __launch_bounds__(512, 2) void prompt_pair_kernel(guide_prompt_spec s, uint32_t tiles, const uint32_t *table) {
    using E = typename Elem<T>::type;
    constexpr int kRow = D * 2, kTileQ = 8 * kRowsPerWave;
    using SendK = Sender<D, true, 8>;
    using SendV = Sender<D, false, 8>;
    __shared__ __align__(16) uint8_t lds_k0[kTileK * kRow], lds_v0[kTileK * kRow], lds_k1[kTileK * kRow], lds_v1[kTileK * kRow];
    __shared__ uint32_t odd0[8], odd1[8];
    Place p;
    uint32_t head, kv;
    if (!find_work<kTileQ, false>(s, Cut{}, table, tiles, p, head, kv)) return;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int first = (int)(p.tile * kTileQ) + wave * kRowsPerWave, row = first + lane % 32;
    const int nq = (int)p.nq, nk = (int)p.nk, shift = nk - nq;
    const int wave_last = first < nq ? min(first + kRowsPerWave, nq) + shift : 0;
    const int last = min((int)p.tile * kTileQ + kTileQ, nq) + shift;
    const int full = max(((int)p.tile * kTileQ + shift + 1) / (2 * kTileK) * (2 * kTileK), 0);

    SendK send_k;
    SendV send_v;
    send_k.init((const E *)s.k + (int64_t)p.k0 * s.k_stride + (int64_t)kv * s.k_head_stride, s.k_stride, nk, wave, lane);
    send_v.init((const E *)s.v + (int64_t)p.k0 * s.v_stride + (int64_t)kv * s.v_head_stride, s.v_stride, nk, wave, lane);
    Rows<T, D> rows;
    send_k.send(lds_k0, wave);
    rows.init((const E *)s.q + (int64_t)(p.q0 + min(row, nq - 1)) * s.q_stride + (int64_t)head * s.q_head_stride, s.scale, lane,
              min(row + shift + 1, nk));
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) rows.p[i][j] = (E)0.0f;          // of no tile: the first product with values adds zeros
    for (int i = threadIdx.x; i < kTileK * kRow / 16; i += 512) *(uint4 *)(lds_v1 + i * 16) = make_uint4(0, 0, 0, 0);
    arrived();
    meet();

    auto run = [&](auto group) __attribute__((always_inline)) {
        constexpr int G = decltype(group)::value;
        // Products of tile t (keys lds_k) after those with the values of tile t - 1 (lds_v); LATE: of a tile that is masked.
        auto products = [&](auto late, int k0, const uint8_t *lds_k, const uint8_t *lds_v, uint32_t (&odd)[8]) __attribute__((always_inline)) {
            constexpr bool LATE = decltype(late)::value;
            if constexpr (LATE) {
                const bool bad = k0 > full && any_of(odd);
                if (bad && k0 - kTileK < wave_last) rows.add_odd(k0 - kTileK, lds_v);
                rows.template values<true>(lds_v, bad);
                if (k0 < wave_last) rows.scores(lds_k);
            } else {
                rows.template values<false>(lds_v, false);
                Rows<T, D>::template reads_ahead<4, 2>();
                rows.scores(lds_k);
                Rows<T, D>::template reads_ahead<6, 1>();
            }
        };
        // One tile, two turns.  next_k / next_v: where the loads of this step's even turn go.
        auto step = [&](auto late, int k0, const uint8_t *lds_k, const uint8_t *old_v, uint8_t *next_k, uint8_t *next_v, uint32_t (&old_odd)[8],
                        uint32_t (&odd)[8]) __attribute__((always_inline)) {
            constexpr bool LATE = decltype(late)::value;
            if constexpr (G == 0) {
                send_k.send(next_k, wave);
                send_v.send(next_v, wave);
            }
            products(late, k0, lds_k, old_v, old_odd);
            if constexpr (G == 1) {
                arrived();
                if constexpr (LATE) odd[wave] = looks_odd<T, SendV::kLoads>(next_v, wave, lane);
                arrived();
            }
            meet();
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (G == 1) {                                  // (the next step's loads: its even turn is this one)
                send_k.send((uint8_t *)lds_k, wave);
                send_v.send((uint8_t *)old_v, wave);
            }
            if (!LATE || k0 < wave_last) {
                rows.template exponentials<LATE>(k0);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) rows.p[i][j] = (E)0.0f;
            }
            if constexpr (G == 0) {
                arrived();
                if constexpr (LATE) odd[wave] = looks_odd<T, SendV::kLoads>(next_v, wave, lane);
                arrived();
            }
            meet();
            __builtin_amdgcn_sched_barrier(0);
        };
        if constexpr (G == 1) {                                      // turn 0
            send_k.send(lds_k1, wave);
            send_v.send(lds_v0, wave);
            meet();
        }
        int k0 = 0;
        for (; k0 < full; k0 += 2 * kTileK) {
            step(std::false_type{}, k0, lds_k0, lds_v1, lds_k1, lds_v0, odd1, odd0);
            step(std::false_type{}, k0 + kTileK, lds_k1, lds_v0, lds_k0, lds_v1, odd0, odd1);
        }
        for (; k0 < last; k0 += 2 * kTileK) {
            step(std::true_type{}, k0, lds_k0, lds_v1, lds_k1, lds_v0, odd1, odd0);
            step(std::true_type{}, k0 + kTileK, lds_k1, lds_v0, lds_k0, lds_v1, odd0, odd1);
        }
        // the values of the last tile
        const bool bad = k0 > full && any_of(odd1);
        if (bad && k0 - kTileK < wave_last) rows.add_odd(k0 - kTileK, lds_v1);
        rows.template values<true>(lds_v1, bad);
        if constexpr (G == 0) meet();                                // group 1's last turn
    };
    if (wave < 4) run(std::integral_constant<int, 0>{});
    else run(std::integral_constant<int, 1>{});
    arrived();                                                       // (no load may be on its way to the LDS of a block that has ended)
    rows.finish(row < nq ? (E *)s.out + (int64_t)(p.q0 + row) * s.out_stride + (int64_t)head * s.out_head_stride : nullptr);
}

// Joins the parts of the rows that have several, in their order: a block takes some heads of one query, D / 4 lanes to a head, four
// channels to a lane.  Bound by latency (4 to 5 us) until the parts are many megabytes.
constexpr uint32_t kMostParts = 16, kWorth = 8192;
template <int T, int D>
__global__ __launch_bounds__(256) void prompt_join_kernel(guide_prompt_spec s, Cut cut, const float *scratch) {
    using E = typename Elem<T>::type;
    constexpr uint32_t kHeads = 256 / (D / 4);
    const uint32_t groups = (s.n_h + kHeads - 1) / kHeads, query = blockIdx.x / groups;
    const uint32_t head = blockIdx.x % groups * kHeads + threadIdx.x / (D / 4), ch = threadIdx.x % (D / 4) * 4;
    uint32_t count = 0, s0 = 0;
    for (uint32_t end = (s.n_seq + 63) / 64; s.n_seq > kWalked && end - s0 > 1;) {      // the last 64 sequences that begin at the query or before it
        const uint32_t mid = (s0 + end) / 2;
        if (clamped(s.q_starts[mid * 64], s.total_q) <= query) s0 = mid;
        else end = mid;
    }
    for (s0 *= 64; s0 < s.n_seq && count == 0; s0 += 64) {
        const Sequence<4 * kRowsPerWave, true> q(s, cut, s0 + threadIdx.x % 64);
        const uint64_t here = __ballot(q.q0 <= query && query - q.q0 < q.nq);
        if (here) count = (uint32_t)__builtin_amdgcn_readlane((int)q.parts, __builtin_ctzll(here));
    }
    if (count < 2 || head >= s.n_h) return;
    const Parts parts((float *)scratch, (uint64_t)s.total_q * s.n_h, cut.most);
    const uint64_t at = (uint64_t)query * s.n_h + head;
    float top[kMostParts], sum[kMostParts];
    f32x4 v[kMostParts];
#pragma unroll
    for (uint32_t i = 0; i < kMostParts; ++i) {                      // (all on their way at once)
        const uint64_t from = at + min(i, count - 1) * parts.rows;
        top[i] = parts.top[from], sum[i] = parts.sum[from];
        __builtin_memcpy(&v[i], parts.value + from * D + ch, 16);
    }
    float best = top[0];
#pragma unroll
    for (uint32_t i = 1; i < kMostParts; ++i) best = fmaxf(best, top[i]);
    const float base = best == -INFINITY ? 0.0f : best;
    float total = 0.0f;
    f32x4 x = {0, 0, 0, 0};
#pragma unroll
    for (uint32_t i = 0; i < kMostParts; ++i) {
        if (i >= count) continue;
        const float f = __builtin_amdgcn_exp2f(top[i] - base);
        total += sum[i] * f;
        x += v[i] * f;
    }
    E e[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) e[b] = (E)(total != 0.0f ? x[b] / total : 0.0f);
    __builtin_memcpy((E *)s.out + (int64_t)query * s.out_stride + (int64_t)head * s.out_head_stride + ch, e, 8);
}

// launch(tiles, blocks) for the blocks of all tiles times heads, the last tiles first, as many at a time as a launch holds:
// find_work() counts from the `tiles` that are left.
template <class Launch>
hipError_t over_tiles(uint32_t tiles, uint32_t n_h, Launch launch) {
    const uint32_t most = (uint32_t)(kMostThreads / 512 / n_h);      // (n_h < 2^16)
    for (uint32_t left = tiles; left;) {
        const uint32_t some = left < most ? left : most;
        launch(left, some * n_h);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        left -= some;
    }
    return hipSuccess;
}

// The table for a call of many sequences (at the start of the scratch), or none.
template <int ROWS, bool SPLIT>
const uint32_t *make_table(const guide_prompt_spec &s, const Cut &cut, float *scratch, hipStream_t stream) {
    if (s.n_seq <= kWalked) return nullptr;
    prompt_table_kernel<ROWS, SPLIT><<<1, 1024, 0, stream>>>(s, cut, (uint32_t *)scratch);
    return (const uint32_t *)scratch;
}

template <int T, int D>
hipError_t prompt_as(const guide_prompt_spec &s, float *scratch, hipStream_t stream) {
    // The pairs of groups pay where their turns are many and their tiles of 256 queries fill the chip: 8192 queries over 32 768
    // keys 1182 against 1113 TFLOP/s, 4096 over 8192 1057 against 1004; equal at 2048 keys to a query, behind with fewer, with
    // fewer tiles than compute units (512 queries of 64 heads: 742 against 912) and with 64 channels (945 against 980).
    const uint32_t filled = s.n_seq < s.total_q ? s.n_seq : s.total_q;              // sequences that can have queries
    const uint64_t keys = (2ull * s.total_k > s.total_q ? 2ull * s.total_k - s.total_q : 0) / (2 * s.n_seq);     // that a query sees, about
    if constexpr (D == 128) {
        if (keys >= 4096 && (uint64_t)(s.total_q / 256) * s.n_h >= kNumCU) {
            const uint32_t *table = make_table<256, false>(s, Cut{}, scratch, stream);
            return over_tiles(s.total_q / 256 + filled, s.n_h, [&](uint32_t left, uint32_t blocks) {
                prompt_pair_kernel<T, D><<<blocks, 512, 0, stream>>>(s, left, table);
            });
        }
    }
    const uint32_t tiles = s.total_q / 128 + filled;                // at least as many as there are
    // Too little work to give every compute unit two blocks: keys are split, into parts of what two blocks to a unit would have of all of
    // it.  Whole / split, 32 heads on 8 of 128: 1 query over 8001 keys 135 / 26 us, 256 over 32 256 536 / 155, 512 over 8512 154 / 90.
    // Of the least number of keys to a part, 256 / 512: 1 over 1001 15.4 / 23.5, 64 over 1064 20.2 / 21.4; but with more rows to join,
    // 128 over 2128 of 32 heads 29 / 24, 1500 over 1500 of 12 heads 37.7 / 32.2.
    // Blocks enough, but for what is known here all keys may be one sequence's: sequences of one tile are split where their own keys ask
    // for it.  One query each over 100 keys, 15 times, and 60 000: 990 / 122, with 64 heads 990 / 237; 16 over 100 to 8000 keys 155 /
    // 100.  Where they are equal after all, that is for nothing (16 over 4000 each 125 / 133, 64 over 1000 of 64 heads 232 / 244), so it
    // is done only where a sequence of all keys would take four times as long as equal ones and 0.14 ms more.
    const uint64_t fewest = (uint64_t)((s.total_q + 127) / 128 > filled ? (s.total_q + 127) / 128 : filled) * s.n_h;
    const uint64_t room = (kScratch - kTable * sizeof(float)) / ((uint64_t)s.total_q * s.n_h * (D + 2) * sizeof(float)), least = (uint64_t)s.total_q * s.n_h <= 2048 ? 256 : 512;
    const uint64_t share = (fewest * keys + 2 * kNumCU - 1) / (2 * kNumCU), size = share > least ? share : least, most = room < kMostParts ? room : kMostParts;
    const bool all = keys >= 2 * size, some = s.n_seq > 1 && s.total_k >= 4 * share + kWorth;
    if (most < 2 || !(all || some)) {
        const uint32_t *table = make_table<128, false>(s, Cut{}, scratch, stream);
        return over_tiles(tiles, s.n_h, [&](uint32_t left, uint32_t blocks) {
            prompt_kernel<T, D, false><<<blocks, 256, 0, stream>>>(s, left, Cut{}, table, nullptr);
        });
    }
    const Cut cut = {make_div32((uint32_t)size), (uint32_t)most, all ? (uint32_t)most : 1u};
    // At least as many units as there are: one to a tile, and beyond those as many to a sequence's last tile as size goes into its keys, which
    // is total_k / size for all sequences, and no more to each of the others, which are total_q / 128.
    const uint64_t more = s.total_k / size, units = tiles + more + (all ? s.total_q / 128 * (more < most ? more : most - 1) : 0);
    const uint32_t *table = make_table<128, true>(s, cut, scratch, stream);
    float *const parts = scratch + kTable;
    const hipError_t e = over_tiles((uint32_t)units, s.n_h, [&](uint32_t left, uint32_t blocks) {
        prompt_kernel<T, D, true><<<blocks, 256, 0, stream>>>(s, left, cut, table, parts);
    });
    if (e != hipSuccess) return e;
    prompt_join_kernel<T, D><<<s.total_q * ((s.n_h * (D / 4) + 255) / 256), 256, 0, stream>>>(s, cut, parts);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_prompt_attention(const guide_prompt_spec &s, float *scratch, hipStream_t stream) {
    if (s.type == GUIDE_BF16) return s.d == 64 ? prompt_as<GUIDE_BF16, 64>(s, scratch, stream) : prompt_as<GUIDE_BF16, 128>(s, scratch, stream);
    return s.d == 64 ? prompt_as<GUIDE_F16, 64>(s, scratch, stream) : prompt_as<GUIDE_F16, 128>(s, scratch, stream);
}

}  // namespace guide
