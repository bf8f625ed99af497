// Tables of requests that go on from others, and copies of their pages (include/jupiter_paged.h).
//
// Who takes what is one workgroup's work; then table rows are written, with the blocks of the old tables marked in one map and those of the new ones in
// another; then blocks that are in the first alone go back on the stack, in the order of their numbers.  Three launches, or one workgroup for it all
// where there is little of it.
#include "paged.h"

namespace jup {
namespace {

constexpr int kPart = 1024;

// The workgroup's scratch.  first: the lowest request that goes on from each, in the workspace where there are more of them (the plan of 512 beams took
// 6.0 µs with it there, and what a thread knows of its request read again; 5.0 so).
constexpr int kNear = 2048;
struct Plan {
    int sums[kPart / 64], worst, first[kNear];
};

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

// Lengths, pages and copies of the new requests, the status, and what is left of the stack (new_free_count).  One workgroup of kPart threads; what it
// writes is there for all of them behind it.  Returns the status.
__device__ int make_plan(const jup_paged_reorder_t& a, int shift, int* first, Plan& s) {
    const int tid = threadIdx.x;
    const bool near = a.n_in <= kNear;
    if (tid == 0) s.worst = 5;
    if (near)
        for (int i = tid; i < a.n_in; i += kPart) s.first[i] = INT32_MAX;
    else
        for (int i = tid; i < a.n_in; i += kPart) __hip_atomic_store(first + i, INT32_MAX, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    wait_stores_performed();
    __syncthreads();
    const int F = *a.free_count, P = 1 << shift;
    int why = F < 0 || F > a.n_free ? 1 : 5;
    int my_parent = -1, my_length = 0;  // of request tid
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
        if (near) atomicMin(s.first + p, i);
        else atomicMin(first + p, i);
        if (i == tid) {
            my_parent = p;
            my_length = length;
        }
    }
    wait_stores_performed();  // (atomics that return nothing count as stores)
    if (why < 5) atomicMin(&s.worst, why);
    __syncthreads();
    // copies: of a page that is partly filled, for all but the first
    auto copied = [&](int i, int& p, int& length) {
        p = my_parent;
        length = my_length;
        if (i >= kPart) {
            p = i < a.n_out ? a.parents[i] : -1;
            if (p < 0 || p >= a.n_in) p = -1;
            length = p < 0 ? 0 : a.lengths[p];
        }
        if (p < 0 || (length & (P - 1)) == 0) return 0;
        return (near ? s.first[p] : __hip_atomic_load(first + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) != i ? 1 : 0;
    };
    int copies = 0;
    for (int part = 0; part < a.n_out; part += kPart) {
        int p, length, all;
        const int mine = copied(part + tid, p, length);
        scan_part(mine, all, s.sums);
        copies += all;
    }
    if (tid == 0 && s.worst == 5 && copies > F) s.worst = 4;
    __syncthreads();
    const int status = s.worst == 5 ? 0 : s.worst;
    int done = 0;
    for (int part = 0; part < a.n_out; part += kPart) {
        const int i = part + tid;
        int p, length, all;
        const int mine = copied(i, p, length), at = done + scan_part(mine, all, s.sums);
        done += all;
        if (i >= a.n_out) continue;
        const bool goes = status == 0 && p >= 0;
        a.new_lengths[i] = goes ? length : 0;
        a.new_owned[i] = goes ? (int)(((long long)length + P - 1) >> shift) : 0;
        a.copy_from[i] = goes && mine ? a.table[(long long)p * a.table_stride + (length >> shift)] : -1;
        a.copy_to[i] = goes && mine ? a.free_blocks[F - 1 - at] : -1;
    }
    wait_stores_performed();
    __syncthreads();  // (free_count may be new_free_count)
    if (tid == 0) {
        *a.status = status;
        *a.new_free_count = status == 0 ? F - copies : F;
    }
    return status;
}

// Old request i's blocks, new request i's row: `threads` threads, each `mark`s blocks of the pool.
template <class M>
__device__ __forceinline__ void old_row(const jup_paged_reorder_t& a, int i, int tid, int threads, M mark) {
    const int* row = a.table + (long long)i * a.table_stride;
    const int n = min(max(a.owned[i], 0), a.table_width);
    for (int j = tid; j < n; j += threads) {
        const int block = row[j];
        if ((unsigned)block < (unsigned)a.n_free) mark(block);
    }
}
template <class M>
__device__ __forceinline__ void new_row(const jup_paged_reorder_t& a, int shift, int i, int tid, int threads, M mark) {
    int* to = a.new_table + (long long)i * a.new_table_stride;
    const int n = a.new_owned[i];  // (0 where nothing goes on)
    const int* row = a.table + (n > 0 ? (long long)a.parents[i] * a.table_stride : 0);
    const int copy = a.copy_to[i], page = a.copy_from[i] >= 0 || copy >= 0 ? a.new_lengths[i] >> shift : -1;
    for (int j = tid; j < a.new_table_width; j += threads) {
        const int block = j >= n ? -1 : j == page ? copy : row[j];
        to[j] = block;
        if ((unsigned)block < (unsigned)a.n_free) mark(block);
    }
}

// Blocks that go back: gone(x) has a bit for each of the blocks 32 x .. 32 x + 31 that was in a table and is not any more.  One workgroup.
template <class G>
__device__ void release(const jup_paged_reorder_t& a, int left, int* sums, G gone_of) {
    const int words = (a.n_free + 31) / 32;
    int done = left;
    for (int part = 0; part < words; part += kPart) {
        const int w = part + (int)threadIdx.x;
        unsigned gone = w < words ? gone_of(w) : 0u;
        if (a.held)
            for (unsigned bits = gone; bits; bits &= bits - 1) {
                const int bit = __builtin_ctz(bits);
                if (a.held[w * 32 + bit]) gone &= ~(1u << bit);
            }
        int all;
        int at = done + scan_part(__popc(gone), all, sums);
        done += all;
        for (; gone; gone &= gone - 1, ++at)
            if (at < a.n_free) a.new_free_blocks[at] = w * 32 + __builtin_ctz(gone);
    }
    if (threadIdx.x == 0) *a.new_free_count = min(done, a.n_free);
}

// All of it.  Up to 2^15 blocks, whose maps are bits in LDS; a wave has a table row.
constexpr int kSmallWords = 1024, kSmallEntries = 16384, kSmallRows = 64;
__global__ __launch_bounds__(kPart) void reorder_small(const jup_paged_reorder_t a, int shift, int* first) {
    __shared__ Plan s;
    __shared__ unsigned before[kSmallWords], after[kSmallWords];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    before[tid] = after[tid] = 0;  // (behind the barriers of the plan)
    if (a.new_free_blocks != a.free_blocks)
        for (int i = tid; i < a.n_free; i += kPart) a.new_free_blocks[i] = a.free_blocks[i];
    const int status = make_plan(a, shift, first, s);
    if (status == 0)
        for (int i = wave; i < a.n_in; i += kPart / 64) old_row(a, i, lane, 64, [&](int block) { atomicOr(before + (block >> 5), 1u << (block & 31)); });
    for (int i = wave; i < a.n_out; i += kPart / 64) new_row(a, shift, i, lane, 64, [&](int block) { atomicOr(after + (block >> 5), 1u << (block & 31)); });
    wait_stores_performed();  // (the stack's copy too: what goes back is written over it)
    __syncthreads();
    const int left = *a.new_free_count;
    __syncthreads();
    if (status == 0) release(a, left, s.sums, [&](int w) { return before[w] & ~after[w]; });
}

// Three launches: maps of a byte per block in the workspace, so that marking one needs no atomic (maps of bits with atomics: 15.7 µs for the rows of 512
// beams, 3.1 so).  512 beams of 64 requests in a pool of 3387 blocks: 5.0 + 3.3 + 3.2 µs, trips to memory behind one another.  The maps are cleared by
// many workgroups and gone through by one, 64 KB of them at a time, so that large pools take their own time, whatever the tables: all three launches, in
// place / with a new stack, take 8.7 / 10.2 µs in a pool of 3900 blocks, 9.1 / 10.5 of 32768, 19 / 21 of 2^18, 54 / 56 of 2^20, 197 / 206 of 2^22.
struct Maps {
    int* first;
    unsigned char *before, *after;
};
__host__ __device__ inline long long map_bytes(int n_free) { return ((long long)n_free + 31) / 32 * 32; }

__global__ __launch_bounds__(kPart) void reorder_plan(const jup_paged_reorder_t a, int shift, Maps x) {
    if (blockIdx.x > 0) {  // these clear the maps (one lies behind the other)
        const long long pieces = 2 * map_bytes(a.n_free) / 16;
        for (long long i = (long long)(blockIdx.x - 1) * kPart + threadIdx.x; i < pieces; i += (long long)(gridDim.x - 1) * kPart)
            ((u32x4*)x.before)[i] = (u32x4){0, 0, 0, 0};
        return;
    }
    __shared__ Plan s;
    make_plan(a, shift, x.first, s);
}

// A workgroup per old and per new table row, and some for the stack.
__global__ __launch_bounds__(128) void reorder_rows(const jup_paged_reorder_t a, int shift, Maps x) {
    const int tid = threadIdx.x;
    int i = (int)blockIdx.x;
    if (i < a.n_in) {
        if (*a.status == 0) old_row(a, i, tid, 128, [&](int block) { x.before[block] = 1; });
        return;
    }
    i -= a.n_in;
    if (i < a.n_out) {
        new_row(a, shift, i, tid, 128, [&](int block) { x.after[block] = 1; });
        return;
    }
    i -= a.n_out;
    for (int j = i * 128 + tid; j < a.n_free; j += ((int)gridDim.x - a.n_in - a.n_out) * 128) a.new_free_blocks[j] = a.free_blocks[j];
}

__global__ __launch_bounds__(kPart) void reorder_release(const jup_paged_reorder_t a, Maps x) {
    __shared__ int sums[kPart / 64];
    if (*a.status != 0) return;
    const int left = *a.new_free_count;
    __syncthreads();  // (everybody has read it)
    release(a, left, sums, [&](int w) {
        unsigned gone = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // 16 bytes, each 0 or 1
            const u32x4 b = *(const u32x4*)(x.before + w * 32ll + 16 * h), c = *(const u32x4*)(x.after + w * 32ll + 16 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned d = b[e] & ~c[e];  // bits 0, 8, 16 and 24
                gone |= ((d * 0x10204080u) >> 28) << (16 * h + 4 * e);
            }
        }
        return gone;
    });
}

// A workgroup per (copy, layer, k or v, `heads` heads), pieces of T.  256 copies of up to 15 slots in four layers of 8 heads, 62 MB in and out: 13.6 µs,
// 4.6 TB/s.
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
    const int shift = log2_of(a.page_size);
    char* at = (char*)a.workspace + kCountBytes;
    int* first = (int*)at;
    // One workgroup for it all, a wave per row: up to 64 rows, 16384 table entries and 2^15 blocks.  Four beams of one request take 6.1 µs; with another
    // plan, which took them 6.7, 10.7 in three launches (and the host two launches more).  In place they take 5.2 µs in any such pool, 8.4 in one of 32769
    // blocks; a new stack is copied by the same workgroup, 4 bytes per thread at a time: 6.5 µs with 200 blocks, 7.6 with 8192, 10.7 with 32768 (lost
    // by the rule: 9.8 with 32769).
    if (a.n_in + a.n_out <= kSmallRows && (long long)a.n_in * a.table_width + (long long)a.n_out * a.new_table_width <= kSmallEntries && a.n_free <= kSmallWords * 32) {
        hipLaunchKernelGGL(reorder_small, dim3(1), dim3(kPart), 0, s, a, shift, first);
        return hipGetLastError();
    }
    unsigned char* maps = (unsigned char*)at + JUP_PAGED_MAX_SEQS * 4;
    const Maps x{first, maps, maps + map_bytes(a.n_free)};
    const long long clear = (2 * map_bytes(a.n_free) / 16 + kPart - 1) / kPart;
    hipLaunchKernelGGL(reorder_plan, dim3(1 + (unsigned)(clear > 1023 ? 1023 : clear)), dim3(kPart), 0, s, a, shift, x);
    const int stack = a.new_free_blocks == a.free_blocks ? 0 : (a.n_free + 1023) / 1024;
    const int rows = a.n_in + a.n_out + (stack > 1024 ? 1024 : stack);
    if (rows > 0) hipLaunchKernelGGL(reorder_rows, dim3((unsigned)rows), dim3(128), 0, s, a, shift, x);
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
