// Device-side helpers and host-side launchers of the 8-bit paged key/value cache (internal to the library).
#pragma once
#include "razer_kernels.hpp"
#include "../../include/razer_cache.h"

namespace razer {

// A cache as the kernels take it: validated on the host, the page size as its logarithm.
struct CacheView {
    uint8_t* k_codes;
    uint8_t* v_codes;
    uint8_t* k_scales;
    uint8_t* v_scales;
    int64_t pages;
    int heads, dim, lp;          // lp = log2(tokens per page)
};

// 2^(b-127) of an exponent byte in [1, 254]
__device__ __forceinline__ float exponent_value(int b) { return __uint_as_float((uint32_t)b << 23); }

razer_status check_cache(const razer_cache* c, CacheView& out);

hipError_t launch_cache_plan(const int32_t* lens, const int32_t* fresh, int requests, int32_t* table, int width, int64_t ld_table,
                             const int32_t* free_pages, int free_count, int lp, int64_t tokens, int32_t* cu, int32_t* total,
                             int64_t* slots, int32_t* positions, int32_t* request_of, int32_t* used, hipStream_t st);
hipError_t launch_cache_append(const CacheView& c, const void* k, int64_t ld_k, const void* v, int64_t ld_v, int bf16,
                               int64_t tokens, const int64_t* slots, hipStream_t st);

struct AttentionArgs {
    const uint16_t* q;
    uint16_t* out;
    int64_t ld_q, ld_out;
    int tokens, requests, q_heads, group;      // group = query heads per key/value head
    const int32_t* cu;
    const int32_t* total;
    const int32_t* table;
    int64_t ld_table;
    int width;
    float scale, cap;
    int window;
    const float* slopes;
    const int32_t* prefix;
};
size_t attention_workspace_bytes(const CacheView& c, const AttentionArgs& a, int64_t max_new, int64_t max_len);   // what a caller is told
size_t attention_workspace_used(const CacheView& c, const AttentionArgs& a, int64_t max_new, int64_t max_len);    // what the call takes of it
hipError_t launch_attention(const CacheView& c, const AttentionArgs& a, int64_t max_new, int64_t max_len, float* ws, hipStream_t st);

}  // namespace razer
