// Tables of requests that go on from others, and copies of their pages (include/jupiter_paged.h).
//
// Three launches: who takes what (one workgroup, while others clear two bit maps of the blocks); table rows, the old tables' blocks marked in
// one map and the new ones' in the other; blocks that are in the first alone go back on the stack, in the order of their numbers.
#include "paged.h"

namespace jup {
namespace {

constexpr int kPart = 1024;

// In the workspace, behind the arrival counters.
struct Scratch {
    int* first;               // [n_in]: the lowest request that goes on from it
    unsigned *before, *after; // bit maps of the blocks
};
__host__ __device__ inline int words_of(int n_free) { return (n_free + 31) / 32; }

__device__ __forceinline__ int owned_of(const jup_paged_reorder_t& a, int i) { return min(max(a.owned[i], 0), a.table_width); }

// Sums of the threads before this one, and of all.
__device__ int scan_part(int mine, int& all, int* lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int run = mine;
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        const int left = __shfl_up(run, by, 64);
        if (lane >= by) run += left;
    }
    __syncthreads();  // (lds is free again)
    if (lane == 63) lds[wave] = run;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kPart / 64; ++w) {
        if (w < wave) before += lds[w];
        all += lds[w];
    }
    return before + run - mine;
}

__global__ __launch_bounds__(kPart) void reorder_plan(const jup_paged_reorder_t a, int shift, Scratch x) {
    const int tid = threadIdx.x;
    if (blockIdx.x > 0) {
        const int words = words_of(a.n_free);
        for (int w = (blockIdx.x - 1) * kPart + tid; w < words; w += (gridDim.x - 1) * kPart) x.before[w] = x.after[w] = 0;
        return;
    }
    __shared__ int lds[kPart / 64], worst;
    if (tid == 0) worst = 5;
    for (int i = tid; i < a.n_in; i += kPart) __hip_atomic_store(x.first + i, INT32_MAX, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    wait_stores_performed();
    __syncthreads();
    const int F = *a.free_count, P = 1 << shift;
    int why = F < 0 || F > a.n_free ? 1 : 5;
    for (int i = tid; i < a.n_out; i += kPart) {
        const int p = a.parents[i];
        if (p == -1) continue;
        if (p < 0 || p >= a.n_in) {
            why = 1;
            continue;
        }
        const int length = a.lengths[p], owned = a.owned[p];
        const int need = (int)(((long long)length + P - 1) >> shift);
        if (length < 0 || owned < 0 || owned > a.table_width || need > owned) why = 1;
        else if (need > a.new_table_width) why = min(why, 2);
        atomicMin(x.first + p, i);
    }
    wait_stores_performed();  // (atomics that return nothing count as stores)
    if (why < 5) atomicMin(&worst, why);
    __syncthreads();
    // copies: of a page that is partly filled, for all but the first
    auto copied = [&](int i, int& p, int& length) {
        p = i < a.n_out ? a.parents[i] : -1;
        if (p < 0 || p >= a.n_in) {
            p = -1;
            length = 0;
            return 0;
        }
        length = a.lengths[p];
        return (length & (P - 1)) != 0 && __hip_atomic_load(x.first + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != i ? 1 : 0;
    };
    int copies = 0;
    for (int part = 0; part < a.n_out; part += kPart) {
        int p, length, all;
        const int mine = copied(part + tid, p, length);
        scan_part(mine, all, lds);
        copies += all;
    }
    if (tid == 0 && worst == 5 && copies > F) worst = 4;
    __syncthreads();
    const int status = worst == 5 ? 0 : worst;
    int done = 0;
    for (int part = 0; part < a.n_out; part += kPart) {
        const int i = part + tid;
        int p, length, all;
        const int mine = copied(i, p, length), at = done + scan_part(mine, all, lds);
        done += all;
        if (i >= a.n_out) continue;
        const bool goes = status == 0 && p >= 0;
        a.new_lengths[i] = goes ? length : 0;
        a.new_owned[i] = goes ? (int)(((long long)length + P - 1) >> shift) : 0;
        a.copy_from[i] = goes && mine ? a.table[(long long)p * a.table_stride + (length >> shift)] : -1;
        a.copy_to[i] = goes && mine ? a.free_blocks[F - 1 - at] : -1;
    }
    __syncthreads();  // (free_count may be new_free_count)
    if (tid == 0) {
        *a.status = status;
        *a.new_free_count = status == 0 ? F - copies : F;
    }
}

__device__ __forceinline__ void mark(unsigned* map, int block, int n_free) {
    if ((unsigned)block < (unsigned)n_free) atomicOr(map + (block >> 5), 1u << (block & 31));
}

// A workgroup per old and per new table row, and some for the stack.
__global__ __launch_bounds__(256) void reorder_rows(const jup_paged_reorder_t a, int shift, Scratch x) {
    const int tid = threadIdx.x, status = *a.status;
    int i = (int)blockIdx.x;
    if (i < a.n_in) {
        if (status != 0) return;
        const int* row = a.table + (long long)i * a.table_stride;
        const int n = owned_of(a, i);
        for (int j = tid; j < n; j += 256) mark(x.before, row[j], a.n_free);
        return;
    }
    i -= a.n_in;
    if (i < a.n_out) {
        int* to = a.new_table + (long long)i * a.new_table_stride;
        const int n = a.new_owned[i];  // (0 where nothing goes on)
        const int* row = a.table + (n > 0 ? (long long)a.parents[i] * a.table_stride : 0);
        const int length = a.new_lengths[i], page = a.copy_from[i] >= 0 || a.copy_to[i] >= 0 ? length >> shift : -1, copy = a.copy_to[i];
        for (int j = tid; j < a.new_table_width; j += 256) {
            const int block = j >= n ? -1 : j == page ? copy : row[j];
            to[j] = block;
            mark(x.after, block, a.n_free);
        }
        return;
    }
    i -= a.n_out;
    for (int j = i * 256 + tid; j < a.n_free; j += ((int)gridDim.x - a.n_in - a.n_out) * 256) a.new_free_blocks[j] = a.free_blocks[j];
}

__global__ __launch_bounds__(kPart) void reorder_release(const jup_paged_reorder_t a, Scratch x) {
    __shared__ int lds[kPart / 64];
    if (*a.status != 0) return;
    const int words = words_of(a.n_free), F = *a.new_free_count;
    int done = F;
    for (int part = 0; part < words; part += kPart) {
        const int w = part + (int)threadIdx.x;
        unsigned gone = w < words ? x.before[w] & ~x.after[w] : 0u;
        if (a.held)
            for (unsigned left = gone; left; left &= left - 1) {
                const int bit = __builtin_ctz(left);
                if (a.held[w * 32 + bit]) gone &= ~(1u << bit);
            }
        int all;
        int at = done + scan_part(__popc(gone), all, lds);
        done += all;
        for (; gone; gone &= gone - 1, ++at)
            if (at < a.n_free) a.new_free_blocks[at] = w * 32 + __builtin_ctz(gone);
    }
    __syncthreads();  // (everybody has read the count)
    if (threadIdx.x == 0) *a.new_free_count = min(done, a.n_free);
}

// A workgroup per (copy, layer, k or v, `heads` heads), pieces of T.
template <class T>
__global__ __launch_bounds__(256) void copy_pages(const jup_paged_pool_t pool, const jup_paged_scales_t scales, const jup_paged_copy_t a, int shift,
                                                  int heads, int groups, int size) {
    long long n = block_number();
    const int group = (int)(n % groups);
    n /= groups;
    const bool values = n & 1;
    n >>= 1;
    const int layer = (int)(n % a.n_layers), i = (int)(n / a.n_layers);
    if (i >= a.n_copies) return;
    const int from = a.copy_from[i], to = a.copy_to[i], P = 1 << shift;
    if ((unsigned)from >= (unsigned)pool.n_blocks || (unsigned)to >= (unsigned)pool.n_blocks) return;
    const int slots = a.lengths ? a.lengths[i] & (P - 1) : P;
    const int head0 = group * heads, count = min(heads, pool.n_kv_heads - head0);
    const int pieces = (int)(pool.head_dim * size / sizeof(T));
    char* base = (char*)(values ? pool.v : pool.k) + ((long long)layer * a.layer_stride + head0 * pool.head_stride) * size;
    const long long source = from * pool.block_stride * size, target = to * pool.block_stride * size;
    const long long all = (long long)count * slots * pieces;
    for (long long w = threadIdx.x; w < all; w += 256) {
        const int slot_of_head = (int)(w / pieces), piece = (int)(w - (long long)slot_of_head * pieces);
        const int h = slot_of_head / slots, slot = slot_of_head - h * slots;
        char* at = base + (h * pool.head_stride + slot * pool.slot_stride) * size + piece * sizeof(T);
        *(T*)(at + target) = *(const T*)(at + source);
    }
    if (!scales.k) return;
    float* scale = (values ? scales.v : scales.k) + (long long)layer * scales.layer_stride + head0 * scales.head_stride;
    for (int w = threadIdx.x; w < count * slots; w += 256) {
        float* at = scale + w / slots * scales.head_stride + w % slots;
        at[to * scales.block_stride] = at[from * scales.block_stride];
    }
}

}  // namespace

hipError_t launch_paged_reorder(const jup_paged_reorder_t& a, hipStream_t s) {
    const int shift = log2_of(a.page_size), words = words_of(a.n_free);
    char* at = (char*)a.workspace + kCountBytes;
    const Scratch x{(int*)at, (unsigned*)(at + JUP_PAGED_MAX_SEQS * 4), (unsigned*)(at + JUP_PAGED_MAX_SEQS * 4) + words};
    const int clear = (words + kPart - 1) / kPart;
    hipLaunchKernelGGL(reorder_plan, dim3(1 + (clear > 255 ? 255 : clear)), dim3(kPart), 0, s, a, shift, x);
    const int stack = a.new_free_blocks == a.free_blocks ? 0 : (a.n_free + 1023) / 1024;
    const int rows = a.n_in + a.n_out + (stack > 1024 ? 1024 : stack);
    if (rows > 0) hipLaunchKernelGGL(reorder_rows, dim3((unsigned)rows), dim3(256), 0, s, a, shift, x);
    hipLaunchKernelGGL(reorder_release, dim3(1), dim3(kPart), 0, s, a, x);
    return hipGetLastError();
}

hipError_t launch_paged_copy(const jup_paged_pool_t& pool, const jup_paged_scales_t* scales, const jup_paged_copy_t& a, hipStream_t s) {
    const int shift = log2_of(pool.page_size);
    const int size = pool.dtype == JUP_F32 ? 4 : pool.dtype == JUP_BF16 ? 2 : 1;
    // heads of a workgroup: about 1024 pieces
    const int pieces = pool.head_dim * size / (pool.dtype == JUP_F32 ? 4 : 16);
    const long long per_head = (long long)pieces << shift;
    int heads = per_head >= 1024 ? 1 : (int)(1024 / per_head);
    if (heads > pool.n_kv_heads) heads = pool.n_kv_heads;
    const int groups = (pool.n_kv_heads + heads - 1) / heads;
    const long long grid = (long long)a.n_copies * a.n_layers * 2 * groups;
    if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
    const jup_paged_scales_t none{};
    if (pool.dtype == JUP_F32) hipLaunchKernelGGL(copy_pages<float>, grid_of(grid), dim3(256), 0, s, pool, none, a, shift, heads, groups, size);
    else hipLaunchKernelGGL(copy_pages<u32x4>, grid_of(grid), dim3(256), 0, s, pool, scales ? *scales : none, a, shift, heads, groups, size);
    return hipGetLastError();
}

}  // namespace jup
