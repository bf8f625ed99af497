// Rows into the slots of a pool in 8 bits, and rows out of the slots of any pool (include/jupiter_paged.h).
//
// A head's 128 values x_i become codes and a scale: m = max(2^-100, max |x_i|), scale = m / T, code_i = round(x_i (T / m)).  Two divisions per head,
// a product per value; keys are rotated first and stay in fp32 up to their code.
#include "codes.h"
#include "paged_rows.h"

namespace jup {
namespace {

// Eight neighbouring lanes have a head: its largest magnitude as bits (as integers magnitudes are in order, with infinities and then NaN on top).
__device__ __forceinline__ unsigned largest(const float* x, const float* y) {
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, max(__float_as_uint(x[e]) & 0x7FFFFFFFu, __float_as_uint(y[e]) & 0x7FFFFFFFu));
    top = max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, true));   // one lane further
    top = max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, true));   // two
    return max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0x141, 0xf, 0xf, true)); // the other four of eight (row_half_mirror)
}

__device__ __forceinline__ void widen8(const u32x4 v, float* x) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = bf2f((u16)(v[e / 2] >> (16 * (e & 1))));
}

// One workgroup per row, as append_bf16: 64 threads make the row's turns, then eight threads have a head of q, k or v each.  Bound by memory: 5940 rows
// of 40 heads, 306 MB in and out, take 57 µs, 5.4 TB/s; with rows that are read through the caches, where nothing looks for them again, 71.  (A scale is
// 4 bytes in a line of its own head: 10 MB more are written than there are.)  80 rows of 32 heads take 4.9 µs: slots, rows, stores behind one another.
template <int CODE>
__global__ __launch_bounds__(256) void append_codes(const jup_paged_pool_t pool, const jup_paged_scales_t scales, const jup_paged_append_t a, int shift,
                                                    const Turns turns) {
    __shared__ float2 cs[64];
    const int row = (int)block_number(), tid = threadIdx.x;
    if (row >= a.n_rows) return;
    const bool rotates = a.rope_theta > 0.0f;
    if (rotates && tid < 64) cs[tid] = turn(a.positions[row], turns.per_position[tid]);
    __syncthreads();
    const int slot = a.slots[row];
    const bool stored = slot >= 0 && (slot >> shift) < pool.n_blocks;
    const long long block = slot >> shift, at = slot & ((1 << shift) - 1);
    const long long place = block * pool.block_stride + at * pool.slot_stride, scale_place = block * scales.block_stride + at;
    const int heads = a.q ? a.n_heads : 0, all = heads + (stored ? 2 * pool.n_kv_heads : 0);
    for (int w = tid; w < all * 8; w += 256) {
        const int piece = (w & 7) * 8;
        int h = w >> 3;
        if (h < heads) {
            const u16* from = (const u16*)a.q + row * a.q_row_stride + h * a.q_head_stride;
            u16* to = (u16*)a.q_out + row * a.q_out_row_stride + h * a.q_out_head_stride;
            u32x4 lo = __builtin_nontemporal_load((const u32x4*)(from + piece)), hi = __builtin_nontemporal_load((const u32x4*)(from + piece + 64));
            rotate8(lo, hi, cs + piece, lo, hi);
            *(u32x4*)(to + piece) = lo;
            *(u32x4*)(to + piece + 64) = hi;
            continue;
        }
        h -= heads;
        const bool keys = h < pool.n_kv_heads;
        if (!keys) h -= pool.n_kv_heads;
        const u16* from = keys ? (const u16*)a.k + row * a.k_row_stride + h * a.k_head_stride : (const u16*)a.v + row * a.v_row_stride + h * a.v_head_stride;
        u8* to = (u8*)(keys ? pool.k : pool.v) + place + h * pool.head_stride;
        const u32x4 lo = __builtin_nontemporal_load((const u32x4*)(from + piece)), hi = __builtin_nontemporal_load((const u32x4*)(from + piece + 64));
        float x[8], y[8];
        if (keys && rotates) {
            rotate8(lo, hi, cs + piece, x, y);
        } else {
            widen8(lo, x);
            widen8(hi, y);
        }
        const unsigned top = largest(x, y);
        const bool number = top < 0x7F800000u;
        const float m = fmaxf(__uint_as_float(top), kLeastMaximum), by = kTopCode<CODE> / m;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = number ? x[e] * by : 0.f;
            y[e] = number ? y[e] * by : 0.f;
        }
        *(u32x2*)(to + piece) = (u32x2){codes_of<CODE>(x), codes_of<CODE>(x + 4)};
        *(u32x2*)(to + piece + 64) = (u32x2){codes_of<CODE>(y), codes_of<CODE>(y + 4)};
        if (piece == 0) (keys ? scales.k : scales.v)[scale_place + h * scales.head_stride] = number ? m / kTopCode<CODE> : __uint_as_float(0x7FC00000u);
    }
}

// One workgroup per row.  Pools in 8 bits: eight threads have a head, 16 codes each.  Bound by memory: 342 MB in and out take 77 µs, 4.4 TB/s; 82 with
// results that stay in the caches, where they push out codes that are read yet.
template <int CODE>
__global__ __launch_bounds__(256) void read_codes(const jup_paged_pool_t pool, const jup_paged_scales_t scales, const jup_paged_read_t a, int shift) {
    const int row = (int)block_number();
    if (row >= a.n_rows) return;
    const int slot = a.slots[row];
    const bool there = slot >= 0 && (slot >> shift) < pool.n_blocks;
    const long long block = there ? slot >> shift : 0, at = there ? slot & ((1 << shift) - 1) : 0;
    const long long place = block * pool.block_stride + at * pool.slot_stride, scale_place = block * scales.block_stride + at;
    for (int w = threadIdx.x; w < pool.n_kv_heads * 16; w += 256) {
        const int piece = (w & 7) * 16;
        int h = w >> 3;
        const bool keys = h < pool.n_kv_heads;
        if (!keys) h -= pool.n_kv_heads;
        u16* to = keys ? (u16*)a.k : (u16*)a.v;
        if (!to) continue;
        to += keys ? row * a.k_row_stride + h * a.k_head_stride : row * a.v_row_stride + h * a.v_head_stride;
        const u32x4 codes = *(const u32x4*)((const u8*)(keys ? pool.k : pool.v) + place + h * pool.head_stride + piece);
        const float scale = (keys ? scales.k : scales.v)[scale_place + h * scales.head_stride];
        u32x4 out[2];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x[4];
            numbers_of<CODE>(codes[e], x);
            out[e >> 1][(e & 1) * 2] = there ? pack_bf16x2(x[0] * scale, x[1] * scale) : 0u;
            out[e >> 1][(e & 1) * 2 + 1] = there ? pack_bf16x2(x[2] * scale, x[3] * scale) : 0u;
        }
        __builtin_nontemporal_store(out[0], (u32x4*)(to + piece));
        __builtin_nontemporal_store(out[1], (u32x4*)(to + piece + 8));
    }
}

// The other pools, as they are.  T: what a thread moves (16 bytes of bf16, a float of a head of any size).
template <class T>
__global__ __launch_bounds__(256) void read_rows(const jup_paged_pool_t pool, const jup_paged_read_t a, int shift, int per_head) {
    const int row = (int)block_number();
    if (row >= a.n_rows) return;
    const int slot = a.slots[row], size = pool.dtype == JUP_F32 ? 4 : 2;
    const bool there = slot >= 0 && (slot >> shift) < pool.n_blocks;
    const long long place = there ? (slot >> shift) * pool.block_stride + (slot & ((1 << shift) - 1)) * pool.slot_stride : 0;
    const int half = pool.n_kv_heads * per_head;
    for (int w = threadIdx.x; w < 2 * half; w += 256) {
        const bool keys = w < half;
        char* to = (char*)(keys ? a.k : a.v);
        if (!to) continue;
        const int x = keys ? w : w - half, h = x / per_head, i = x - h * per_head;
        const T value = ((const T*)((const char*)(keys ? pool.k : pool.v) + (place + h * pool.head_stride) * size))[i];
        ((T*)(to + (keys ? row * a.k_row_stride + h * a.k_head_stride : row * a.v_row_stride + h * a.v_head_stride) * size))[i] = there ? value : T{};
    }
}

}  // namespace

hipError_t launch_paged_append8(const jup_paged_pool_t& pool, const jup_paged_scales_t& scales, const jup_paged_append_t& a, hipStream_t s) {
    const Turns turns = turns_of(a.rope_theta, pool.head_dim);
    const int shift = log2_of(pool.page_size);
    if (pool.dtype == JUP_I8) hipLaunchKernelGGL(append_codes<JUP_I8>, grid_of(a.n_rows), dim3(256), 0, s, pool, scales, a, shift, turns);
    else hipLaunchKernelGGL(append_codes<JUP_E4M3>, grid_of(a.n_rows), dim3(256), 0, s, pool, scales, a, shift, turns);
    return hipGetLastError();
}

hipError_t launch_paged_read(const jup_paged_pool_t& pool, const jup_paged_scales_t* scales, const jup_paged_read_t& a, hipStream_t s) {
    const int shift = log2_of(pool.page_size);
    const dim3 grid = grid_of(a.n_rows), block(256);
    if (pool.dtype == JUP_I8) hipLaunchKernelGGL(read_codes<JUP_I8>, grid, block, 0, s, pool, *scales, a, shift);
    else if (pool.dtype == JUP_E4M3) hipLaunchKernelGGL(read_codes<JUP_E4M3>, grid, block, 0, s, pool, *scales, a, shift);
    else if (pool.dtype == JUP_BF16) hipLaunchKernelGGL(read_rows<u32x4>, grid, block, 0, s, pool, a, shift, pool.head_dim / 8);
    else hipLaunchKernelGGL(read_rows<float>, grid, block, 0, s, pool, a, shift, pool.head_dim);
    return hipGetLastError();
}

}  // namespace jup
