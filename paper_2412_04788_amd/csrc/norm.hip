// Group quantisation, and the root-mean-square norm whose output is quantised.
#include "layer.hpp"
#include "layer_kernels.hpp"

namespace guide {
namespace {

// Codes of a matrix.  A lane takes eight neighbouring elements (16 or 32 bytes in one load), a quad of lanes a group of 32, whose
// maximum goes round the quad.  Bound by memory: 8192 x 8192 of 16 bits to 4-bit codes 33 to 40 us (170 MB, 4.2 to 5.1 TB/s).
template <int T, int BITS>
__global__ __launch_bounds__(kBlock) void quantise_kernel(guide_quantise_spec s, Div32 per_row, uint32_t n) {
    using E = typename Elem<T>::type;
    const uint32_t at = blockIdx.x * kBlock + threadIdx.x;          // n is a multiple of four: quads live and die together
    if (at >= n) return;
    const uint32_t row = div32(at, per_row), c = at - row * per_row.d;
    float x[8];
    load_upto8<T>((const E *)s.x + (int64_t)row * s.x_stride + c * 8u, (int)s.cols - (int)(c * 8u), x);
    uint32_t byte;
    const Codes<BITS> q = quantise8<BITS>(x, byte);
    store_codes<BITS>(s.codes + (int64_t)row * s.codes_stride + (size_t)c * BITS, q);
    if ((c & 3u) == 0) s.scales[(int64_t)row * s.scales_stride + (c >> 2)] = (uint8_t)byte;
}

// One row per group of LANES lanes, its t held in registers between the sum of its squares and its codes (CHUNKS times eight
// elements a lane), so that everything is read once.  Bound by memory: 8192 rows of 8192 in 16 bits with residual to 8-bit codes
// 89 to 94 us (472 MB, 5.0 to 5.3 TB/s); seven rows of 4096 take 4 us, a launch and two trips to memory.
template <int T, int BITS, int LANES, int CHUNKS>
__global__ __launch_bounds__(LANES < kBlock ? kBlock : LANES) void norm_kernel(guide_norm_spec s) {
    using E = typename Elem<T>::type;
    constexpr int kThreads = LANES < kBlock ? kBlock : LANES;
    constexpr int kRows = kThreads / LANES;
    const uint32_t lane = threadIdx.x % LANES;
    const uint32_t row = blockIdx.x * kRows + threadIdx.x / LANES;
    if (kRows > 1 && row >= s.rows) return;                          // whole waves
    const E *x = (const E *)s.x + (int64_t)row * s.x_stride;
    const E *r = (const E *)s.residual + (int64_t)row * s.residual_stride;
    float t[CHUNKS][8];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        const int at = (int)(lane + i * LANES) * 8, left = (int)s.d - at;
        load_upto8<T>(x + at, left, t[i]);
        if (s.residual) {
            float u[8];
            load_upto8<T>(r + at, left, u);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[i][j] += u[j];
        }
    }
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        const int at = (int)(lane + i * LANES) * 8, left = (int)s.d - at;
        if (s.total && left > 0) store_upto8<T>((E *)s.total + (int64_t)row * s.total_stride + at, left, t[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(t[i][j], t[i][j], sum);
    }
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) sum += __shfl_xor(sum, m);
    if constexpr (LANES > kWave) {
        __shared__ float part[LANES / kWave];
        if (lane % kWave == 0) part[lane / kWave] = sum;
        __syncthreads();
        sum = 0.0f;
#pragma unroll
        for (int w = 0; w < LANES / kWave; ++w) sum += part[w];
    }
    const float inv = 1.0f / sqrtf(sum / (float)s.d + s.eps);
    const int padded = (int)((s.d + 31u) / 32u * 32u);
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        const int at = (int)(lane + i * LANES) * 8;
        if (at >= padded) break;                                     // whole quads
        float w[8];
        load_upto8<T>((const E *)s.weight + at, (int)s.d - at, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = at + j < (int)s.d ? t[i][j] * inv * w[j] : 0.0f;   // (0 * inf is no zero)
        uint32_t byte;
        const Codes<BITS> q = quantise8<BITS>(w, byte);
        store_codes<BITS>(s.codes + (int64_t)row * s.codes_stride + (size_t)at * BITS / 8, q);
        if ((lane & 3u) == 0) s.scales[(int64_t)row * s.scales_stride + at / 32] = (uint8_t)byte;
    }
}

template <int T, int BITS>
hipError_t quantise_as(const guide_quantise_spec &s, hipStream_t stream) {
    const uint32_t per_row = (s.cols + 31u) / 32u * 4u, most = (uint32_t)(kMostThreads / per_row);        // (per_row <= 2^28)
    guide_quantise_spec part = s;
    for (uint32_t at = 0; at < s.rows; at += part.rows) {
        part.rows = s.rows - at < most ? s.rows - at : most;
        part.x = (const typename Elem<T>::type *)s.x + (int64_t)at * s.x_stride;
        part.codes = s.codes + (int64_t)at * s.codes_stride;
        part.scales = s.scales + (int64_t)at * s.scales_stride;
        const uint32_t n = per_row * part.rows;
        quantise_kernel<T, BITS><<<(n + kBlock - 1) / kBlock, kBlock, 0, stream>>>(part, make_div32(per_row), n);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int T, int BITS, int LANES, int CHUNKS>
hipError_t norm_with(const guide_norm_spec &s, hipStream_t stream) {
    using E = typename Elem<T>::type;
    constexpr uint32_t kThreads = LANES < kBlock ? kBlock : LANES, kRows = kThreads / LANES, kMost = kMostThreads / LANES;
    guide_norm_spec part = s;
    for (uint32_t at = 0; at < s.rows; at += part.rows) {
        part.rows = s.rows - at < kMost ? s.rows - at : kMost;
        part.x = (const E *)s.x + (int64_t)at * s.x_stride;
        if (s.residual) part.residual = (const E *)s.residual + (int64_t)at * s.residual_stride;
        if (s.total) part.total = (E *)s.total + (int64_t)at * s.total_stride;
        part.codes = s.codes + (int64_t)at * s.codes_stride;
        part.scales = s.scales + (int64_t)at * s.scales_stride;
        norm_kernel<T, BITS, LANES, CHUNKS><<<(part.rows + kRows - 1) / kRows, kThreads, 0, stream>>>(part);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int T, int BITS>
hipError_t norm_as(const guide_norm_spec &s, hipStream_t stream) {
    const uint32_t chunks = (s.d + 7u) / 8u;
    // a wave per row up to 1024 elements, a block beyond: 32 elements a lane at most
    if (chunks <= 64) return norm_with<T, BITS, 64, 1>(s, stream);
    if (chunks <= 128) return norm_with<T, BITS, 64, 2>(s, stream);
    if (chunks <= 256) return norm_with<T, BITS, 256, 1>(s, stream);
    if (chunks <= 512) return norm_with<T, BITS, 256, 2>(s, stream);
    if (chunks <= 1024) return norm_with<T, BITS, 256, 4>(s, stream);
    if (chunks <= 2048) return norm_with<T, BITS, 1024, 2>(s, stream);
    return norm_with<T, BITS, 1024, 4>(s, stream);
}

}  // namespace

hipError_t launch_quantise(const guide_quantise_spec &s, hipStream_t stream) {
    const int key = (int)s.type * 2 + (s.bits == 8);
    switch (key) {
        case 0: return quantise_as<GUIDE_BF16, 4>(s, stream);
        case 1: return quantise_as<GUIDE_BF16, 8>(s, stream);
        case 2: return quantise_as<GUIDE_F16, 4>(s, stream);
        case 3: return quantise_as<GUIDE_F16, 8>(s, stream);
        case 4: return quantise_as<GUIDE_F32, 4>(s, stream);
        default: return quantise_as<GUIDE_F32, 8>(s, stream);
    }
}

hipError_t launch_norm(const guide_norm_spec &s, hipStream_t stream) {
    const int key = (int)s.type * 2 + (s.bits == 8);
    switch (key) {
        case 0: return norm_as<GUIDE_BF16, 4>(s, stream);
        case 1: return norm_as<GUIDE_BF16, 8>(s, stream);
        case 2: return norm_as<GUIDE_F16, 4>(s, stream);
        case 3: return norm_as<GUIDE_F16, 8>(s, stream);
        case 4: return norm_as<GUIDE_F32, 4>(s, stream);
        default: return norm_as<GUIDE_F32, 8>(s, stream);
    }
}

}  // namespace guide
