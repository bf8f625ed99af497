// Tables of a step over a paged cache, and its rows into their slots (include/jupiter_paged.h).
//
// Tables.  Request i of n needs fresh_i = max(0, ceil((L_i + m_i) / P) - owned_i) pages; prefix sums over the requests of m and
// of fresh give every request its rows and its place in the stack of free blocks.  One workgroup goes through the requests
// 1024 at a time, twice: the sums alone (does the step fit?), then with the sums of the parts before it the writes.
// Sums saturate: what the arrays hold is the caller's, and a sum that wraps would pass the checks.
// Bound by latencies (loads, prefix sum, search, loads, stores): pages and rows are looked up four at a time.  Eight requests of five
// tokens take 4.4 µs, 1024 requests of one to 230 9.5 in two launches.
#include "paged.h"

namespace jup {
namespace {

constexpr int kPart = 1024;  // requests (and threads) of one part

struct Pair {
    unsigned rows, fresh;
};
__device__ __forceinline__ unsigned sum(unsigned a, unsigned b) { return __builtin_elementwise_add_sat(a, b); }
__device__ __forceinline__ Pair operator+(Pair a, Pair b) { return {sum(a.rows, b.rows), sum(a.fresh, b.fresh)}; }

// Sums of the threads before this one, and of all; lds: one entry per wave.  (What is before a thread is of use where nothing is saturated.)
__device__ Pair scan_part(Pair mine, Pair& all, Pair* lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Pair run = mine;
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        const Pair left{__shfl_up(run.rows, by, 64), __shfl_up(run.fresh, by, 64)};
        if (lane >= by) run = run + left;
    }
    __syncthreads();  // (lds is free again)
    if (lane == 63) lds[wave] = run;
    __syncthreads();
    Pair before{0, 0};
    all = Pair{0, 0};
#pragma unroll
    for (int w = 0; w < kPart / 64; ++w) {
        if (w < wave) before = before + lds[w];
        all = all + lds[w];
    }
    return {before.rows + run.rows - mine.rows, before.fresh + run.fresh - mine.fresh};
}

struct Request {
    int length, rows, owned, fresh, why;  // why: status 1 or 2, or 0
};
__device__ __forceinline__ Request request_of(const jup_paged_extend_t& a, int shift, int i) {
    Request r{0, 0, 0, 0, 0};
    if (i >= a.n_seqs) return r;
    r.length = a.lengths[i];
    r.rows = a.n_new[i];
    r.owned = a.owned[i];
    if (r.length < 0 || r.rows < 0 || r.owned < 0 || r.owned > a.table_width) {
        r.why = 1;
        return r;
    }
    const long long need = ((long long)r.length + r.rows + (1 << shift) - 1) >> shift;
    if (need > a.table_width) {
        r.why = 2;
        return r;
    }
    r.fresh = need > r.owned ? (int)need - r.owned : 0;
    return r;
}

// Last i of at[0 .. n) with at[i] <= x; at[0] <= x.
__device__ __forceinline__ int last_not_above(const int* at, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The same for four numbers at once, neighbours in the part by 1024, those below `end`; at[0] = 0.
__device__ __forceinline__ void find4(const int* at, int n, int first, int end, int* found) {
    int lo[4] = {0, 0, 0, 0}, size = n;
    while (size > 1) {  // the same size for all: the last not above lies in [lo, lo + size)
        const int half = size >> 1;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (at[lo[k] + half] <= min(first + k * kPart, end - 1)) lo[k] += half;
        size -= half;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) found[k] = lo[k];
}

// Slot of a position in a request's table row; -1 where there is none (a block number that no pool has).
__device__ __forceinline__ int slot_of(const int* table_row, int shift, int width, int position) {
    const int page = position >> shift;
    if (page >= width) return -1;
    const int block = table_row[page];
    const long long slot = ((long long)block << shift) + (position & ((1 << shift) - 1));
    return block < 0 || slot > INT32_MAX ? -1 : (int)slot;
}

// ROWS: positions and slots too (a launch of their own writes them where they are many).
template <bool ROWS>
__global__ __launch_bounds__(kPart) void extend_tables(const jup_paged_extend_t a, int shift) {
    __shared__ Pair sums[kPart / 64];
    __shared__ int row_at[kPart], fresh_at[kPart], length_at[kPart], owned_at[kPart];
    __shared__ int worst;
    const int tid = threadIdx.x;
    if (tid == 0) worst = 5;
    const int F = *a.free_count;
    Pair total{0, 0}, first_at{0, 0};
    Request first{0, 0, 0, 0, 0};
    int why = 5;
    if (F < 0 || F > a.n_free) why = 1;
    for (int part = 0; part < a.n_seqs; part += kPart) {
        const Request r = request_of(a, shift, part + tid);
        if (r.why) why = min(why, r.why);
        Pair all;
        const Pair at = scan_part({(unsigned)max(r.rows, 0), (unsigned)r.fresh}, all, sums);
        total = total + all;
        if (part == 0) {
            first = r;
            first_at = at;
        }
    }
    if (total.rows > (unsigned)a.max_rows) why = min(why, 3);
    if (F >= 0 && total.fresh > (unsigned)F) why = min(why, 4);
    __syncthreads();
    if (why < 5) atomicMin(&worst, why);
    __syncthreads();
    const bool fits = worst == 5;
    if (tid == 0) {
        *a.status = fits ? 0 : worst;
        *a.new_free_count = fits ? F - (int)total.fresh : F;
        a.row_start[a.n_seqs] = fits ? (int)total.rows : 0;
    }
    Pair done{0, 0};
    for (int part = 0; part < a.n_seqs; part += kPart) {
        const int i = part + tid, here = min(kPart, a.n_seqs - part);
        Request r = first;
        Pair all = total, at = first_at;
        if (!fits) {  // nothing happens to any
            if (part > 0) r = request_of(a, shift, i);
            r.rows = r.fresh = 0;
            all = at = {0, 0};
        } else if (a.n_seqs > kPart) {
            if (part > 0) r = request_of(a, shift, i);
            at = scan_part({(unsigned)r.rows, (unsigned)r.fresh}, all, sums);
        }
        if (i < a.n_seqs) {
            a.row_start[i] = (int)(done.rows + at.rows);
            a.new_lengths[i] = r.length + r.rows;
            a.new_owned[i] = r.owned + r.fresh;
        }
        row_at[tid] = (int)at.rows;
        fresh_at[tid] = (int)at.fresh;
        length_at[tid] = r.length;
        owned_at[tid] = r.owned;
        __syncthreads();
        // the part's pages, dealt to the threads one by one (a prompt needs hundreds where a decoding request needs none)
        for (int p = tid; p < (int)all.fresh; p += 4 * kPart) {
            int q[4], block[4];
            find4(fresh_at, here, p, (int)all.fresh, q);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (p + k * kPart < (int)all.fresh) block[k] = a.free_blocks[F - 1 - (int)done.fresh - p - k * kPart];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (p + k * kPart < (int)all.fresh)
                    a.table[(long long)(part + q[k]) * a.table_stride + owned_at[q[k]] + p + k * kPart - fresh_at[q[k]]] = block[k];
        }
        if (ROWS) {
            __syncthreads();  // the entries are there
            for (int row = tid; row < (int)all.rows; row += 4 * kPart) {
                int q[4];
                find4(row_at, here, row, (int)all.rows, q);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (row + k * kPart >= (int)all.rows) continue;
                    const int position = length_at[q[k]] + row + k * kPart - row_at[q[k]];
                    const int to = (int)done.rows + row + k * kPart;
                    a.positions[to] = position;
                    a.slots[to] = slot_of(a.table + (long long)(part + q[k]) * a.table_stride, shift, a.table_width, position);
                }
            }
        }
        __syncthreads();  // (the part's arrays are free again)
        done = done + all;
    }
    if (ROWS) {
        for (int row = (int)done.rows + tid; row < a.max_rows; row += kPart) {
            a.positions[row] = 0;
            a.slots[row] = -1;
        }
    }
}

// Positions and slots of steps with many rows, from what extend_tables left.  A wave has 64 neighbouring rows: it finds the request of the
// first of them 64 probes at a time, and the others' among the 64 requests from there on.
__global__ __launch_bounds__(256) void extend_rows(const jup_paged_extend_t a, int shift) {
    const int lane = threadIdx.x & 63, row = blockIdx.x * 256 + threadIdx.x;
    const int total = a.n_seqs > 0 ? a.row_start[a.n_seqs] : 0;
    const int row0 = row - lane;
    int position = 0, slot = -1;
    if (row0 < total) {
        int first = 0, size = a.n_seqs;
        while (size > 1) {
            const int step = (size + 63) / 64, at = first + lane * step;
            const bool below = lane * step < size && a.row_start[min(at, a.n_seqs)] <= row0;
            const int n = __popcll(__ballot(below));  // (row_start does not fall: the lanes below are the first n, and n > 0)
            first += (n - 1) * step;
            size = min(step, size - (n - 1) * step);
        }
        const int mine = min(first + lane, a.n_seqs);
        const int start = a.row_start[mine];
        int lo = 0;  // the last of the 64 that begins at or before the row
#pragma unroll
        for (int half = 32; half > 0; half >>= 1)
            if (__shfl(start, lo + half, 64) <= row) lo += half;
        int i = min(first + lo, a.n_seqs - 1);
        if (row < total) {
            if (lo == 63) i = first + 63 + last_not_above(a.row_start + first + 63, a.n_seqs - first - 63, row);  // (idle requests lie between)
            position = a.new_lengths[i] - (a.row_start[i + 1] - row);
            slot = slot_of(a.table + (long long)i * a.table_stride, shift, a.table_width, position);
        }
    }
    if (row < a.max_rows) {
        a.positions[row] = position;
        a.slots[row] = slot;
    }
}

// ---- rows into their slots -----------------------------------------------------------------------------------------------
// The rotation turns the pair (x_i, x_(i + D/2)) by position * theta^(-2i/D).  The host hands over the turns per position,
// theta^(-2i/D) / 2 pi in 64 bits (one pow() and products), and a thread takes the fraction of a turn that is left in 64
// bits too: at position 10^6 the angle has lost 10^-10 of a turn.  Sine and cosine are fp32, as is the rotation; one rounding
// at the end.
struct Turns {
    double per_position[128];
};
__device__ __forceinline__ float2 turn(int position, double per_position) {
    const double t = (double)position * per_position;
    float s, c;
    sincospif(2.0f * (float)(t - rint(t)), &s, &c);
    return make_float2(c, s);
}

__device__ __forceinline__ void rotate8(const u32x4 lo, const u32x4 hi, const float2* cs, u32x4& out_lo, u32x4& out_hi) {
    float x[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float a = bf2f((u16)(lo[e / 2] >> (16 * (e & 1)))), b = bf2f((u16)(hi[e / 2] >> (16 * (e & 1))));
        x[e] = a * cs[e].x - b * cs[e].y;
        y[e] = b * cs[e].x + a * cs[e].y;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        out_lo[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
        out_hi[e] = pack_bf16x2(y[2 * e], y[2 * e + 1]);
    }
}

// One workgroup per row: 64 threads make the row's turns, then eight threads have a head of q, k or v each (two pieces of 16 bytes,
// 64 elements apart).  Bound by memory: prompts of 365 MB in and out take 69 µs, 5.3 TB/s (a large copy: 4.9 to 5.2).
__global__ __launch_bounds__(256) void append_bf16(const jup_paged_pool_t pool, const jup_paged_append_t a, int shift, const Turns turns) {
    __shared__ float2 cs[64];
    const int row = (int)block_number(), tid = threadIdx.x;
    if (row >= a.n_rows) return;
    const bool rotates = a.rope_theta > 0.0f;
    if (rotates && tid < 64) cs[tid] = turn(a.positions[row], turns.per_position[tid]);
    __syncthreads();
    const int slot = a.slots[row];
    const bool stored = slot >= 0 && (slot >> shift) < pool.n_blocks;
    const long long place = (long long)(slot >> shift) * pool.block_stride + (long long)(slot & ((1 << shift) - 1)) * pool.slot_stride;
    const int heads = a.q ? a.n_heads : 0, all = heads + (stored ? 2 * pool.n_kv_heads : 0);
    for (int w = tid; w < all * 8; w += 256) {
        const int piece = (w & 7) * 8;
        int h = w >> 3;
        const u16* from;
        u16* to;
        bool turned = rotates;
        if (h < heads) {
            from = (const u16*)a.q + row * a.q_row_stride + h * a.q_head_stride;
            to = (u16*)a.q_out + row * a.q_out_row_stride + h * a.q_out_head_stride;
        } else if ((h -= heads) < pool.n_kv_heads) {
            from = (const u16*)a.k + row * a.k_row_stride + h * a.k_head_stride;
            to = (u16*)pool.k + place + h * pool.head_stride;
        } else {
            h -= pool.n_kv_heads;
            from = (const u16*)a.v + row * a.v_row_stride + h * a.v_head_stride;
            to = (u16*)pool.v + place + h * pool.head_stride;
            turned = false;
        }
        u32x4 lo = *(const u32x4*)(from + piece), hi = *(const u32x4*)(from + piece + 64);
        if (turned) rotate8(lo, hi, cs + piece, lo, hi);
        *(u32x4*)(to + piece) = lo;
        *(u32x4*)(to + piece + 64) = hi;
    }
}

// Check mode: a thread per pair.
__global__ __launch_bounds__(256) void append_f32(const jup_paged_pool_t pool, const jup_paged_append_t a, int shift, const Turns turns) {
    const int row = (int)block_number(), half = pool.head_dim / 2;
    if (row >= a.n_rows) return;
    const bool rotates = a.rope_theta > 0.0f;
    const int position = rotates ? a.positions[row] : 0;
    const int slot = a.slots[row];
    const bool stored = slot >= 0 && (slot >> shift) < pool.n_blocks;
    const long long place = (long long)(slot >> shift) * pool.block_stride + (long long)(slot & ((1 << shift) - 1)) * pool.slot_stride;
    const int heads = a.q ? a.n_heads : 0, all = heads + (stored ? 2 * pool.n_kv_heads : 0);
    for (int w = threadIdx.x; w < all * half; w += 256) {
        int h = w / half;
        const int i = w - h * half;
        const float* from;
        float* to;
        bool turned = rotates;
        if (h < heads) {
            from = (const float*)a.q + row * a.q_row_stride + h * a.q_head_stride;
            to = (float*)a.q_out + row * a.q_out_row_stride + h * a.q_out_head_stride;
        } else if ((h -= heads) < pool.n_kv_heads) {
            from = (const float*)a.k + row * a.k_row_stride + h * a.k_head_stride;
            to = (float*)pool.k + place + h * pool.head_stride;
        } else {
            h -= pool.n_kv_heads;
            from = (const float*)a.v + row * a.v_row_stride + h * a.v_head_stride;
            to = (float*)pool.v + place + h * pool.head_stride;
            turned = false;
        }
        float x = from[i], y = from[i + half];
        if (turned) {
            const float2 cs = turn(position, turns.per_position[i]);
            const float z = x * cs.x - y * cs.y;
            y = y * cs.x + x * cs.y;
            x = z;
        }
        to[i] = x;
        to[i + half] = y;
    }
}

}  // namespace

hipError_t launch_paged_extend(const jup_paged_extend_t& a, hipStream_t s) {
    const int shift = log2_of(a.page_size);
    // One workgroup for the rows as well, or a launch of their own: 4096 rows of 64 requests 6.4 and 7.5 µs, 8192 rows 8.2 and 7.6, 16384
    // rows of 16 requests 11.0 and 7.4.
    if (a.max_rows <= 4096) {
        hipLaunchKernelGGL(extend_tables<true>, dim3(1), dim3(kPart), 0, s, a, shift);
    } else {
        hipLaunchKernelGGL(extend_tables<false>, dim3(1), dim3(kPart), 0, s, a, shift);
        hipLaunchKernelGGL(extend_rows, dim3((unsigned)(((long long)a.max_rows + 255) / 256)), dim3(256), 0, s, a, shift);
    }
    return hipGetLastError();
}

hipError_t launch_paged_append(const jup_paged_pool_t& pool, const jup_paged_append_t& a, hipStream_t s) {
    Turns turns;
    const int half = pool.head_dim / 2;
    if (a.rope_theta > 0.0f) {
        const double step = pow((double)a.rope_theta, -1.0 / half);
        double t = 0.15915494309189533577;  // 1 / 2 pi
        for (int i = 0; i < half; ++i, t *= step) turns.per_position[i] = t;
    }
    const int shift = log2_of(pool.page_size);
    if (pool.dtype == JUP_BF16)
        hipLaunchKernelGGL(append_bf16, grid_of(a.n_rows), dim3(256), 0, s, pool, a, shift, turns);
    else
        hipLaunchKernelGGL(append_f32, grid_of(a.n_rows), dim3(256), 0, s, pool, a, shift, turns);
    return hipGetLastError();
}

}  // namespace jup
