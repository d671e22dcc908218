// Launchers of the layer operators, called by the C ABI after it has checked the specs.
#pragma once

#include "guide_layer.h"
#include <hip/hip_runtime.h>

namespace guide {

// Threads of a launch: HIP takes fewer than 2^32 along a dimension, and what needs more goes in several launches.
constexpr uint64_t kMostThreads = 1ull << 31;

hipError_t launch_quantise(const guide_quantise_spec &s, hipStream_t stream);
hipError_t launch_norm(const guide_norm_spec &s, hipStream_t stream);
// scratch: kScratch bytes that work split over blocks (a product's k, a prompt's keys) keeps its parts in.
constexpr size_t kScratch = 64u << 20;
hipError_t launch_product(const guide_product_spec &s, float *scratch, hipStream_t stream);
hipError_t launch_prompt_attention(const guide_prompt_spec &s, float *scratch, hipStream_t stream);
hipError_t launch_cache_append(const guide_cache &c, const guide_cache_tokens &t, hipStream_t stream);
hipError_t launch_cache_read(const guide_cache &c, const guide_cache_tokens &t, hipStream_t stream);
hipError_t launch_cache_attention(const guide_cache &c, const guide_cache_queries &q, void *ws, hipStream_t stream);
size_t cache_attention_workspace(uint32_t n_seq, uint32_t n_h, uint32_t n_kv, uint32_t d, uint64_t max_len);

}  // namespace guide
