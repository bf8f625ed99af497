// Attention of the new tokens of a ragged batch over a paged cache (include/jupiter_paged.h).
#include "paged.h"

namespace jup {
namespace {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(u16 x) { return bf2f(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(u16* p, float x) { *p = f2bf(x); }

// One wave per (row, query head): 64 keys at a time, a lane has a key's score, then D / 64 columns of the output (rounded up).
template <class T>
__global__ __launch_bounds__(64) void attention_rows(const jup_paged_pool_t pool, const jup_paged_attention_t a, int shift) {
    __shared__ float q[256];
    const int lane = threadIdx.x, row = blockIdx.x / a.n_heads, head = blockIdx.x - row * a.n_heads;
    const int D = pool.head_dim, kv_head = head / (a.n_heads / pool.n_kv_heads);
    int lo = 0, hi = a.n_seqs;  // the request: the last one that begins at or before the row
    if (row < a.row_start[0]) return;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.row_start[mid] <= row) lo = mid;
        else hi = mid;
    }
    const int end = a.row_start[lo + 1];
    if (row >= end) return;
    const long long last = min((long long)a.lengths[lo] - (end - row), ((long long)a.table_width << shift) - 1);
    const int* table = a.table + lo * a.table_stride;
    for (int i = lane; i < D; i += 64) q[i] = to_f32(((const T*)a.q)[row * a.q_row_stride + head * a.q_head_stride + i]);
    __syncthreads();
    float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (long long first = 0; first <= last; first += 64) {
        const long long key = first + lane;
        long long at = -1;
        float s = -INFINITY;
        if (key <= last) {
            const int block = table[key >> shift];
            if (block >= 0 && block < pool.n_blocks) {
                at = block * pool.block_stride + kv_head * pool.head_stride + (key & ((1 << shift) - 1)) * pool.slot_stride;
                const T* k = (const T*)pool.k + at;
                float sum = 0.f;
                for (int i = 0; i < D; ++i) sum = __builtin_fmaf(q[i], to_f32(k[i]), sum);
                s = sum * a.scale;
            }
        }
        float top = s;
        bool nan = s != s;
        for (int by = 32; by > 0; by >>= 1) top = fmaxf(top, __shfl_xor(top, by, 64));
        const float m_new = fmaxf(m, top);
        if (m_new == -INFINITY && !__any(nan)) continue;
        const float back = m == -INFINITY ? 0.f : expf(m - m_new);
        const float p = at < 0 ? 0.f : expf(s - m_new);
        float sum = p;
        for (int by = 32; by > 0; by >>= 1) sum += __shfl_xor(sum, by, 64);
        l = l * back + sum;
        m = m_new;
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] *= back;
        for (int j = 0; j < 64; ++j) {
            const long long from = __shfl(at, j, 64);
            const float w = __shfl(p, j, 64);
            if (from < 0) continue;
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (lane + 64 * c < D) acc[c] = __builtin_fmaf(w, to_f32(((const T*)pool.v)[from + lane + 64 * c]), acc[c]);
        }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (lane + 64 * c < D) put((T*)a.out + row * a.out_row_stride + head * a.out_head_stride + lane + 64 * c, l == 0.f ? 0.f : acc[c] / l);
}

}  // namespace

hipError_t launch_paged_attention(const jup_paged_pool_t& pool, const jup_paged_attention_t& a, hipStream_t s) {
    const int shift = log2_of(pool.page_size);
    const dim3 grid((unsigned)a.n_rows * (unsigned)a.n_heads);
    if (pool.dtype == JUP_BF16)
        hipLaunchKernelGGL(attention_rows<u16>, grid, dim3(64), 0, s, pool, a, shift);
    else
        hipLaunchKernelGGL(attention_rows<float>, grid, dim3(64), 0, s, pool, a, shift);
    return hipGetLastError();
}

}  // namespace jup

extern "C" size_t jup_paged_workspace_bytes(void) { return 256; }
