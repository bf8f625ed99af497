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

// ---- pools in 8 bits (paged_codes.hip, paged_attention8.hip) ----------------------------------------------------------
hipError_t launch_paged_append8(const jup_paged_pool_t& pool, const jup_paged_scales_t& scales, const jup_paged_append_t& a, hipStream_t s);
hipError_t launch_paged_read(const jup_paged_pool_t& pool, const jup_paged_scales_t* scales, const jup_paged_read_t& a, hipStream_t s);  // (of any pool)
hipError_t launch_paged_attention8(const jup_paged_pool_t& pool, const jup_paged_scales_t& scales, const jup_paged_attention_t& a, hipStream_t s, int tiled = 0);

// ---- beams (paged_beams.hip, paged_reorder.hip) --------------------------------------------------------------------------
hipError_t launch_beam_select(const jup_beam_select_t& a, hipStream_t s);
hipError_t launch_paged_reorder(const jup_paged_reorder_t& a, hipStream_t s);
hipError_t launch_paged_copy(const jup_paged_pool_t& pool, const jup_paged_scales_t* scales, const jup_paged_copy_t& a, hipStream_t s);

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
    jup_paged_scales_t scales;  // the first layer's; k null: a pool of values
    const int32_t *positions, *slots;
    jup_paged_attention_t attention;
    jup_paged_pool_t layer(int l) const {
        jup_paged_pool_t p = pool;
        const size_t at = (size_t)l * layer_stride * (pool.dtype == JUP_F32 ? 4 : scales.k ? 1 : 2);
        p.k = (char*)pool.k + at;
        p.v = (char*)pool.v + at;
        return p;
    }
    jup_paged_scales_t layer_scales(int l) const {
        jup_paged_scales_t x = scales;
        x.k += (size_t)l * scales.layer_stride;
        x.v += (size_t)l * scales.layer_stride;
        return x;
    }
};

}  // namespace jup
