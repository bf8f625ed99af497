// Internal declarations of the paged-cache operators (include/jupiter_paged.h): arguments as the kernels take them.
#pragma once

#include "bf16_common.h"
#include "jupiter_paged.h"

namespace jup {

constexpr int kMaxPageSize = 65536;

// A workspace: arrival counters, zero between launches, then what the workgroups of a launch leave for each other.
constexpr size_t kCountBytes = (size_t)JUP_PAGED_MAX_SEQS * 4;
constexpr int kVerifySlices = 64;  // of the vocabulary
constexpr size_t kVerifyBytes = (size_t)JUP_PAGED_MAX_SEQS * kVerifySlices * 8;

// page_size is a power of two
inline int log2_of(int page_size) { return __builtin_ctz((unsigned)page_size); }

// A launch of 2^32 threads or more along one axis runs some of its workgroups only, and reports no error: many workgroups lie in lines of 2^20.
// There may be more of them than asked for.
constexpr int kLineBits = 20;
inline dim3 grid_of(long long blocks) {
    const long long line = 1ll << kLineBits;
    return blocks <= line ? dim3((unsigned)blocks) : dim3((unsigned)line, (unsigned)((blocks + line - 1) / line));
}
__device__ __forceinline__ unsigned block_number() { return blockIdx.y << kLineBits | blockIdx.x; }

// ---- tables and append (paged_tables.hip) -------------------------------------------------------------------------
hipError_t launch_paged_extend(const jup_paged_extend_t& a, hipStream_t s);
hipError_t launch_paged_append(const jup_paged_pool_t& pool, const jup_paged_append_t& a, hipStream_t s);

// ---- attention (paged_attention.hip) --------------------------------------------------------------------------------
// tiled (JUP_BF16 only): 0, or out is [n_rows, n_heads * 128] in the layout of a projection's operand (tiled_offset), this many stages
hipError_t launch_paged_attention(const jup_paged_pool_t& pool, const jup_paged_attention_t& a, hipStream_t s, int tiled = 0);

// ---- verification (paged_verify.hip) --------------------------------------------------------------------------------
hipError_t launch_verify_drafts(const jup_verify_drafts_t& a, hipStream_t s);

// ---- a stage over pages (bf16_forward.hip, kernels_f32.hip) -----------------------------------------------------------
// What a forward over a ragged batch needs in place of a cache.  attention: the call of one layer, but for q, out and their
// strides.
struct PagedStep {
    jup_paged_pool_t pool;   // the first layer's
    int64_t layer_stride;    // elements
    const int32_t *positions, *slots;
    jup_paged_attention_t attention;
    jup_paged_pool_t layer(int l) const {
        jup_paged_pool_t p = pool;
        const size_t at = (size_t)l * layer_stride * (pool.dtype == JUP_F32 ? 4 : 2);
        p.k = (char*)pool.k + at;
        p.v = (char*)pool.v + at;
        return p;
    }
};

}  // namespace jup
