// Attention of the new tokens of a ragged batch over a pool in 8 bits (include/jupiter_paged.h).
#include "codes.h"

namespace jup {
namespace {

// One wave per (row, query head): 64 keys at a time, a lane has a key's score, then two columns of the output.
template <int CODE>
__global__ __launch_bounds__(64) void attention_plain(const jup_paged_pool_t pool, const jup_paged_scales_t scales, const jup_paged_attention_t a, int shift, int tiled) {
    __shared__ float q[128];
    const int lane = threadIdx.x, row = (int)(block_number() / (unsigned)a.n_heads), head = (int)block_number() - row * a.n_heads;
    if (row >= a.n_rows) return;
    const int kv_head = head / (a.n_heads / pool.n_kv_heads);
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
    for (int i = lane; i < 128; i += 64) q[i] = bf2f(((const u16*)a.q)[row * a.q_row_stride + head * a.q_head_stride + i]);
    __syncthreads();
    float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f};
    for (long long first = 0; first <= last; first += 64) {
        const long long key = first + lane;
        long long at = -1;
        float s = -INFINITY, v_scale = 0.f;
        if (key <= last) {
            const int block = table[key >> shift];
            if (block >= 0 && block < pool.n_blocks) {
                const long long in = key & ((1 << shift) - 1), scale_at = block * scales.block_stride + kv_head * scales.head_stride + in;
                at = block * pool.block_stride + kv_head * pool.head_stride + in * pool.slot_stride;
                const u8* k = (const u8*)pool.k + at;
                float sum = 0.f;
                for (int i = 0; i < 128; i += 4) {
                    float x[4];
                    numbers_of<CODE>(*(const unsigned*)(k + i), x);
                    for (int e = 0; e < 4; ++e) sum = __builtin_fmaf(q[i + e], x[e], sum);
                }
                s = sum * scales.k[scale_at] * a.scale;
                v_scale = scales.v[scale_at];
            }
        }
        float top = s;
        const bool nan = s != s;
        for (int by = 32; by > 0; by >>= 1) top = fmaxf(top, __shfl_xor(top, by, 64));
        const float m_new = fmaxf(m, top);
        if (m_new == -INFINITY && !__any(nan)) continue;
        const float back = m == -INFINITY ? 0.f : expf(m - m_new);
        const float p = at < 0 ? 0.f : expf(s - m_new);
        float sum = p;
        for (int by = 32; by > 0; by >>= 1) sum += __shfl_xor(sum, by, 64);
        l = l * back + sum;
        m = m_new;
        acc[0] *= back;
        acc[1] *= back;
        const float pv = at < 0 ? 0.f : p * v_scale;
        for (int j = 0; j < 64; ++j) {
            const long long from = __shfl(at, j, 64);
            const float w = __shfl(pv, j, 64);
            if (from < 0) continue;
            float x[4];
            numbers_of<CODE>(((const u8*)pool.v)[from + lane] | ((const u8*)pool.v)[from + 64 + lane] << 8, x);
            acc[0] = __builtin_fmaf(w, x[0], acc[0]);
            acc[1] = __builtin_fmaf(w, x[1], acc[1]);
        }
    }
    for (int x = 0; x < 2; ++x) {
        const int i = lane + 64 * x;
        u16* out = (u16*)a.out + (tiled ? (long long)tiled_offset(row, head * 16 + (i >> 3), tiled) + (i & 7) : row * a.out_row_stride + head * a.out_head_stride + i);
        *out = f2bf(l == 0.f ? 0.f : acc[x] / l);
    }
}

}  // namespace

hipError_t launch_paged_attention8(const jup_paged_pool_t& pool, const jup_paged_scales_t& scales, const jup_paged_attention_t& a, hipStream_t s, int tiled) {
    const int shift = log2_of(pool.page_size);
    const dim3 grid = grid_of((long long)a.n_rows * a.n_heads);
    if (pool.dtype == JUP_I8) hipLaunchKernelGGL(attention_plain<JUP_I8>, grid, dim3(64), 0, s, pool, scales, a, shift, tiled);
    else hipLaunchKernelGGL(attention_plain<JUP_E4M3>, grid, dim3(64), 0, s, pool, scales, a, shift, tiled);
    return hipGetLastError();
}

}  // namespace jup
