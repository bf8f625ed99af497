// Attention over a paged cache, what its kernels share: a call as they take it, who does what, pages, pieces put together, launches.
//
// Rows.  A key/value head serves G = n_heads / n_kv_heads query heads, so the rows that read the same keys are (token, query
// head of the group): row r of a request is token r / G, head r % G.  A workgroup has a TILE of such rows of one request and one
// key/value head and a range of its keys.
//
// Who does what is found on the GPU: lengths are known nowhere else.  Every wave reads the lengths of all requests (64 lanes, a
// prefix sum), so a launch needs no table of work and no launch before it: the host's grid is an upper bound, and the
// workgroups past the last piece of work leave.  Of more than 64 requests plan_work() makes a table first.  See find_work().
#pragma once

#include "codes.h"

namespace jup {
namespace {

__device__ inline f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

constexpr int kKT = 32;  // keys per tile

// A call, as the kernels take it.
struct Attention {
    const u16 *q, *k, *v;
    u16* out;
    long long q_row, q_head, out_row, out_head;   // strides
    int tiled;                                    // not 0: out is [rows, heads x 128] in the layout of a projection's operand, so many stages
    long long block, head, slot;
    const int *row_start, *lengths, *table;
    long long table_row;
    int n_seqs, n_rows, n_kv_heads, n_blocks, shift, positions;  // positions: of a table row, table_width pages
    Quotient group;                               // G
    float scale_log2e;
    const int2* plan;                             // of more than 64 requests: see plan_work()
    int* count;                                   // arrival counters of rows whose keys are divided, zero between launches
    float* partial;                               // [slot][kv head][row of the tile][kPartRow]
    float chunk_factor;                           // 1 / pieces of work per key/value head that fill the chip (find_work); large: keys are not divided
    int most_items, most_places;                  // pieces of the grid and places of the scratch, per key/value head
    int least_rows, most_rows;                    // requests with so many rows (tokens x G) are this launch's
};
// Of a pool in 8 bits.  k, v, block, head and slot count bytes there.
struct Attention8 : Attention {
    const float *k_scale, *v_scale;
    long long scale_block, scale_head;
};
template <int CODE>
struct Args {
    typedef Attention8 type;
};
template <>
struct Args<JUP_BF16> {
    typedef Attention type;
};
template <int CODE>
using ArgsOf = typename Args<CODE>::type;
template <int CODE>
__device__ __forceinline__ auto pool_of(const u16* p) {
    if constexpr (CODE == JUP_BF16) return p;
    else return (const u8*)p;
}
// The arguments, read from memory where they are used: behind a main loop that needs the scalar registers itself.
template <class A = Attention>
__device__ __forceinline__ A args_again() {
    typedef const __attribute__((address_space(4))) char* kernarg;
    kernarg p = (kernarg)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const A*)p;
}
constexpr int kPartRow = 132;  // 128 un-normalised outputs, maximum, sum, two unused

// Where 16-byte piece `ch` of a row's head goes.
__device__ __forceinline__ u16* out_piece(const Attention& a, int row, int head, int ch) {
    if (a.tiled) return a.out + tiled_offset(row, head * 16 + ch, a.tiled);
    return a.out + row * a.out_row + head * a.out_head + ch * 8;
}

// ---- who does what -------------------------------------------------------------------------------------------------------
// A request of m new tokens has ceil(m G / R) tiles of R rows; a tile whose last row sees n keys has ceil(n / 32) key tiles,
// and these are divided into pieces of at most `chunk`.  chunk = all key tiles of all rows / pieces wanted: about `pieces`
// pieces per key/value head then fill the chip, however uneven the requests are, and no piece is longer than the others
// by more than rounding.  Row tiles are numbered from the end: the longest first.
struct Work {
    int begin, tokens;    // rows of q of this request
    int before;           // position of its first new token (negative: lengths shorter than the new tokens)
    int seq, tile;        // request, tile of rows
    int keys;             // that the last row of the tile sees
    int tile_lo, tile_hi; // key tiles of this piece
    int piece, pieces;    // of this tile of rows
    int slot;             // of piece 0 in the scratch (pieces > 1)
    // (every lane has the same; the compiler is told so)
    __device__ __forceinline__ void make_uniform() {
        for (int* x : {&begin, &tokens, &before, &seq, &tile, &keys, &tile_lo, &tile_hi, &piece, &pieces, &slot}) *x = __builtin_amdgcn_readfirstlane(*x);
    }
};

__device__ __forceinline__ int pieces_of(int key_tiles, int chunk) { return max(1, (int)(((unsigned)key_tiles + (unsigned)chunk - 1) / (unsigned)chunk)); }

template <int R>
struct Request {
    int begin, tokens, before, tiles, key_tiles;  // key_tiles: of the last tile
    Request() = default;
    // (no branches: the loads of several requests are in flight together)
    __device__ __forceinline__ Request(const Attention& a, int i, int last) {
        const int at = min(i, last - 1);
        const int start = a.row_start[at], end = a.row_start[at + 1], length = a.lengths[at];
        const int n = (int)((unsigned)min(end, a.n_rows) - (unsigned)start);  // (start >= 0 where it counts)
        const long long rows = (long long)n * a.group.d;
        const bool counts = i < last && start >= 0 && end > start && n > 0 && rows >= a.least_rows && rows <= a.most_rows;
        begin = counts ? start : 0;
        tokens = counts ? n : 0;
        before = (int)max((long long)length - ((long long)end - start), -(long long)INT32_MAX);
        tiles = counts ? (int)((rows + R - 1) / R) : 0;
        key_tiles = counts ? (keys_of(a, tokens - 1) + kKT - 1) / kKT : 0;
    }
    // keys that token t sees
    __device__ __forceinline__ int keys_of(const Attention& a, int t) const {
        return (int)min(max((long long)before + t + 1, 0ll), (long long)a.positions);
    }
    __device__ __forceinline__ float cost(const Attention& a) const {
        if (R > 32 && tiles > 1)  // (half as much for a prompt from its first token on; at least half of tiles x key_tiles)
            return (float)tiles * 0.5f * (float)(key_tiles + (keys_of(a, a.group.of(R - 1)) + kKT - 1) / kKT);
        return (float)tiles * (float)key_tiles;
    }
    __device__ __forceinline__ int pieces(int chunk) const { return tiles == 0 ? 0 : pieces_of(key_tiles, chunk); }
    __device__ __forceinline__ int items(int chunk) const { return tiles * pieces(chunk); }
    __device__ __forceinline__ int slots(int chunk) const { return pieces(chunk) > 1 ? items(chunk) : 0; }
};

// The longest piece: all requests' costs over the pieces wanted.  (Rounded up by more than the sums are off: at most as many pieces
// more than tiles as are wanted.)  least: the shortest piece worth a workgroup, in key tiles.
__device__ __forceinline__ int chunk_of(const Attention& a, float cost, int least) {
    return __builtin_amdgcn_readfirstlane((int)fminf(fmaxf(cost * a.chunk_factor + 1.0f, (float)least), 1e9f));
}
__device__ __forceinline__ void prefix_sums(int& x, int& y, int lane) {  // inclusive, over a wave
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        const int x2 = __shfl_up(x, by, 64), y2 = __shfl_up(y, by, 64);
        if (lane >= by) {
            x += x2;
            y += y2;
        }
    }
}

// More than 64 requests, whose prefix sums every wave of every workgroup would otherwise make again (256 requests of one token behind
// 100 to 900: 259 µs, and 226 with the plan; 1024 with grouped heads 482 and 242; 4096 5090 and 478): entry i of the plan is the pieces and
// the places of the scratch before request i, the one behind the last request all pieces and the longest piece.  One workgroup, a few
// neighbouring requests per thread.
template <int R>
__global__ __launch_bounds__(1024) void plan_work(const Attention a, int least, int2* plan) {
    __shared__ float costs[16];
    __shared__ int2 sums[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (a.n_seqs + 1023) / 1024, from = tid * each, to = min(a.n_seqs, from + each);
    float cost = 0.f;
    for (int i = from; i < to; ++i) cost += Request<R>(a, i, to).cost(a);
    cost = wave_sum(cost);
    if (lane == 0) costs[wave] = cost;
    __syncthreads();
    cost = 0.f;
    for (int x = 0; x < 16; ++x) cost += costs[x];
    const int chunk = chunk_of(a, cost, least);
    int items = 0, slots = 0;
    for (int i = from; i < to; ++i) {
        const Request<R> r(a, i, to);
        items += r.items(chunk);
        slots += r.slots(chunk);
    }
    int items_to = items, slots_to = slots;
    prefix_sums(items_to, slots_to, lane);
    if (lane == 63) sums[wave] = make_int2(items_to, slots_to);
    __syncthreads();
    for (int x = 0; x < wave; ++x) {
        items_to += sums[x].x;
        slots_to += sums[x].y;
    }
    if (tid == 1023) plan[a.n_seqs] = make_int2(items_to, chunk);
    items_to -= items;
    slots_to -= slots;
    for (int i = from; i < to; ++i) {
        const Request<R> r(a, i, to);
        plan[i] = make_int2(items_to, slots_to);
        items_to += r.items(chunk);
        slots_to += r.slots(chunk);
    }
}

// Piece number `item` of a key/value head; false: there are fewer.  All lanes of a wave call it and get the same.  R: rows of a tile.
constexpr int kOrdered = 16;  // requests that are put in order of their lengths

template <int R>
__device__ bool find_work(const Attention& a, int item, int least, Work& w) {
    const int lane = threadIdx.x & 63;
    const int at_item = item;
    int seq, chunk, slots_before;
    Request<R> r;
    if (!a.plan) {  // a lane per request
        const int n = a.n_seqs;
        r = Request<R>(a, lane, n);
        chunk = chunk_of(a, wave_sum(r.cost(a)), least);
        const int items = r.items(chunk), slots = r.slots(chunk);
        int items_to = items, slots_to = slots;
        if (R > 32 && n <= kOrdered) {
            // whole prompts: the requests with the most keys first, so that what is left for the end is short (four chunks of 1 to 1000
            // tokens behind 100 to 8000: 164 -> 139 µs; others the same)
            for (int j = 0; j < n; ++j) {
                const int keys = __builtin_amdgcn_readlane(r.key_tiles, j);
                const bool before = keys > r.key_tiles || (keys == r.key_tiles && j < lane);
                items_to += before ? __builtin_amdgcn_readlane(items, j) : 0;
                slots_to += before ? __builtin_amdgcn_readlane(slots, j) : 0;
            }
        } else {
            prefix_sums(items_to, slots_to, lane);
        }
        const unsigned long long there = __ballot(item < items_to && item >= items_to - items);
        if (!there) return false;
        seq = __builtin_ctzll(there);
        item -= __builtin_amdgcn_readlane(items_to - items, seq);
        slots_before = __builtin_amdgcn_readlane(slots_to - slots, seq);
        for (int* x : {&r.begin, &r.tokens, &r.before, &r.tiles, &r.key_tiles}) *x = __builtin_amdgcn_readlane(*x, seq);
    } else {  // the last request with no more than `item` pieces before it: of 64 runs of neighbours, then of 64 of the run's, ...
        const int2 all = a.plan[a.n_seqs];
        if (item >= all.x) return false;
        chunk = all.y;
        seq = 0;
        for (int last = a.n_seqs, each = (last + 63) / 64;; each = (each + 63) / 64) {
            const int i = seq + lane * each;
            const int2 before = a.plan[min(i, last - 1)];
            const unsigned long long there = __ballot(i < last && before.x <= item);
            if (!there) return false;
            const int at = 63 - __builtin_clzll(there);
            seq += at * each;
            if (each == 1) {
                item -= __builtin_amdgcn_readlane(before.x, at);
                slots_before = __builtin_amdgcn_readlane(before.y, at);
                break;
            }
            last = min(last, seq + each);
        }
        r = Request<R>(a, seq, a.n_seqs);
    }
    const int most = r.pieces(chunk);
    const int nth = (unsigned)item / (unsigned)max(most, 1);
    // (requests that overlap in a row_start that makes no sense: sums can wrap, and a tile whose pieces are not all in the grid is left
    // out, so that its counter stays 0)
    if (item < 0 || nth >= r.tiles || slots_before < 0 || (most > 1 && slots_before + nth * most > a.most_places - most)) return false;
    w.seq = seq;
    w.begin = r.begin;
    w.tokens = r.tokens;
    w.before = r.before;
    w.tile = r.tiles - 1 - nth;
    w.piece = item - nth * most;
    w.slot = slots_before + nth * most;
    const int last_token = min(a.group.of(w.tile * R + min(R, r.tokens * (int)a.group.d - w.tile * R) - 1), r.tokens - 1);
    w.keys = r.keys_of(a, last_token);
    const int key_tiles = (w.keys + kKT - 1) / kKT;
    w.pieces = pieces_of(key_tiles, chunk);
    if (w.piece >= w.pieces || at_item - w.piece + w.pieces > a.most_items) return false;  // (an earlier tile of a prompt: fewer keys than the last one)
    const int even = (unsigned)key_tiles / (unsigned)w.pieces, over = key_tiles - even * w.pieces;
    w.tile_lo = w.piece * even + min(w.piece, over);
    w.tile_hi = w.tile_lo + even + (w.piece < over);
    return true;
}

// ---- pages -----------------------------------------------------------------------------------------------------------------
// Block numbers of a key tile's four groups of eight rows (a page has at least eight).  Read through the scalar cache:
// the tables do not change during a launch.
struct Blocks {
    int id[4];
};
__device__ __forceinline__ Blocks blocks_of(const Attention& a, const int* table_row, int tile, int last_key) {
    typedef const __attribute__((address_space(4))) int* scalar;
    Blocks b;
#pragma unroll
    for (int p = 0; p < 4; ++p) b.id[p] = ((scalar)table_row)[min(tile * kKT + 8 * p, last_key) >> a.shift];
    return b;
}
// Address of the first of eight rows; of a place in block 0 where there is no such page (read, and not used).
template <class T>  // u16, or u8 of a pool in 8 bits
__device__ __forceinline__ const char* group_base(const Attention& a, const T* pool, int block, int key) {
    const int at = (unsigned)block < (unsigned)a.n_blocks ? block : 0;
    return uniform_ptr((const char*)(pool + at * a.block + (key & ((1 << a.shift) - 1)) * a.slot));
}
// Which of a tile's 32 rows are keys: a page that is there, at or before the last key.
__device__ __forceinline__ unsigned rows_there(const Attention& a, const Blocks& b, int tile, int last_key) {
    unsigned rows = 0;
#pragma unroll
    for (int p = 0; p < 4; ++p)
        if ((unsigned)b.id[p] < (unsigned)a.n_blocks) rows |= 0xFFu << (8 * p);
    const int n = last_key + 1 - tile * kKT;
    return n >= kKT ? rows : n <= 0 ? 0 : rows & ((1u << n) - 1);
}

__device__ inline float max_across_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float max_across_rows(float x) {  // of 16 lanes, within each half
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Eight codes as a matrix operand.
template <int CODE>
__device__ __forceinline__ bf16x8 operand(unsigned lo, unsigned hi) {
    const u32x2 a = bf16_of<CODE>(lo), b = bf16_of<CODE>(hi);
    return __builtin_bit_cast(bf16x8, (u32x4){a[0], a[1], b[0], b[1]});
}

// Transposing 8-byte LDS read: within each group of 16 lanes, lane i receives as element r element (i & 3) of the 8 bytes
// addressed by lane 4r + (i >> 2) of the group.
__device__ __forceinline__ u32x2 read_tr(unsigned lds_address) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(size_t)lds_address));
}

// ---- values that are no numbers --------------------------------------------------------------------------------------------
// The products of a tile are sums over all its 32 keys, with probability 0 where a row does not see a key; 0 times an infinity
// or a NaN is NaN.  In tiles in which some row does not see some key (masked ones: a few per workgroup) such values are
// therefore set to 0 in LDS, and what they do to the rows that do see them is added to the sums at the end, from memory.
__device__ __forceinline__ unsigned not_finite(unsigned v) {  // bits 15 and 31: an exponent of ones
    return ((v & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
}
// A 16-byte piece of a row of values in a masked tile; there: the row is a key.  True: something was taken out of it.
__device__ __forceinline__ bool clean_piece(unsigned char* at, bool there) {
    u32x4 v = *(const u32x4*)at;
    unsigned any = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) any |= not_finite(v[e]);
    if (there && !any) return false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned bad = not_finite(v[e]);
        v[e] = there ? v[e] & ~((bad & 0x8000u ? 0xFFFFu : 0u) | (bad & 0x80000000u ? 0xFFFF0000u : 0u)) : 0u;
    }
    *(u32x4*)at = v;
    return there;
}
// Of codes e4m3's 0x7F and 0xFF are no numbers (int8's are, all 256): the same with NaN in the place of what is added.
__device__ __forceinline__ unsigned not_numbers(unsigned v) {  // bits 7, 15, 23 and 31
    return ((v & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
}
__device__ __forceinline__ bool clean_codes(u32x4& v, bool there) {
    unsigned any = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned bad = not_numbers(v[e]);
        any |= bad;
        v[e] = there ? v[e] & ~((bad >> 7) * 255u) : 0u;
    }
    return there && any;
}
// What was taken out of a key's values, for four features from `feature` on (registers r .. r + 3 of sums), if the row sees the key.
template <int CODE, class V>
__device__ __forceinline__ void add_not_finite(V& sums, int r, const char* row, int feature, bool sees) {
    if constexpr (CODE == JUP_BF16) {
        const u32x2 v = *(const u32x2*)(row + feature * 2);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const unsigned bad = not_finite(v[e]);
            if (sees && (bad & 0x8000u)) sums[r + 2 * e] += bf2f((u16)v[e]);
            if (sees && (bad >> 31)) sums[r + 2 * e + 1] += bf2f((u16)(v[e] >> 16));
        }
    } else {
        const unsigned bad = not_numbers(*(const unsigned*)(row + feature));
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (sees && ((bad >> (8 * e)) & 0x80u)) sums[r + e] = __uint_as_float(0x7FC00000u);
    }
}
// Whether a row of values in memory has any (all lanes get the same).
template <int CODE>
__device__ __forceinline__ bool row_not_finite(const char* row) {
    if constexpr (CODE == JUP_BF16) return __any(not_finite(*(const unsigned*)(row + 4 * (threadIdx.x & 63))) != 0);
    else return CODE == JUP_E4M3 && __any(not_numbers(*(const unsigned*)(row + 4 * (threadIdx.x & 31))) != 0);
}

// ---- pieces of one tile put together ------------------------------------------------------------------------------------------
// The workgroups of a tile's pieces leave un-normalised sums and their softmax statistics in the scratch; the one that
// arrives last adds them in the order of the pieces (the result does not depend on who that is) and writes the rows.  Nobody
// waits.  Half a wave has a row, a lane 16 bytes of it: whole lines go to memory and back (a few bytes at 32-byte steps, as the sums lie
// in the registers, are a partial write each).  One CU takes 20 GB/s out of memory in loads of 8 bytes per lane: with 16 bytes, and no
// branches between the loads, 300 tokens behind 6000 on 8 heads, in tiles of 64 rows, took 29 µs instead of 41.

// Accesses of 16 bytes that are performed chip-wide, as load_coherent2() and store_coherent2() of 8 are.
constexpr int kCoherent = 16;  // of the buffer builtins: past L2
__device__ __forceinline__ auto scratch_of(const float* p) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)uniform_ptr((const char*)p), 0, 0x7FFFFFFF, 0x00027000);
}

// Two rows per wave at a time (a half has one, a lane four features of it: 16 bytes), N such pairs and PC pieces of each in flight at once:
// they come from memory, microseconds away.  No branches around the loads: what is not there is read twice and counts as a piece without keys.
template <int WAVES, int N, int PC>
__device__ __forceinline__ void join_rows(const Attention& a, const Work& w, int R, int kv_head, int first, int rows, const float* base, long long step) {
    const int lane = threadIdx.x & 31, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r0 = first + 2 * wave + ((threadIdx.x >> 5) & 1);
    const auto scratch = scratch_of(base);
    float m[N], l[N];
    f32x4 acc[N];
#pragma unroll
    for (int x = 0; x < N; ++x) {
        m[x] = -INFINITY;
        l[x] = 0.f;
        acc[x] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    for (int p0 = 0; p0 < w.pieces; p0 += PC) {
        u32x2 stat[N][PC];
        u32x4 val[N][PC];
#pragma unroll
        for (int x = 0; x < N; ++x)
#pragma unroll
            for (int p = 0; p < PC; ++p) {
                const unsigned at = (unsigned)(min(p0 + p, w.pieces - 1) * (int)step * 4) + min(r0 + x * 2 * WAVES, rows - 1) * (kPartRow * 4);
                stat[x][p] = __builtin_amdgcn_raw_buffer_load_b64(scratch, at + 512, 0, kCoherent);
                val[x][p] = __builtin_amdgcn_raw_buffer_load_b128(scratch, at + 16 * lane, 0, kCoherent);
            }
#pragma unroll
        for (int x = 0; x < N; ++x) {
            float top = m[x];
#pragma unroll
            for (int p = 0; p < PC; ++p) top = fmaxf(top, __uint_as_float(stat[x][p][0]));
            const float ref = top == -INFINITY ? 0.f : top;  // (nothing seen so far: the maximum stays open)
            const float back = __builtin_amdgcn_exp2f(m[x] - ref);
            l[x] *= back;
            acc[x] *= back;
#pragma unroll
            for (int p = 0; p < PC; ++p) {
                const float sum = __uint_as_float(stat[x][p][1]);
                if (p0 + p < w.pieces && sum != 0.f) {  // (0: a piece this row sees nothing of)
                    const float f = __builtin_amdgcn_exp2f(__uint_as_float(stat[x][p][0]) - ref);
                    l[x] += sum * f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[x][e] += __uint_as_float(val[x][p][e]) * f;
                }
            }
            m[x] = top;
        }
    }
#pragma unroll
    for (int x = 0; x < N; ++x) {
        const int r = r0 + x * 2 * WAVES;
        if (r >= rows) continue;
        const float inv = l[x] == 0.f ? 0.f : 1.0f / l[x];
        const int row = w.tile * R + r, token = a.group.of(row);
        u32x2 o;
        o[0] = pack_bf16x2(acc[x][0] * inv, acc[x][1] * inv);
        o[1] = pack_bf16x2(acc[x][2] * inv, acc[x][3] * inv);
        *(u32x2*)(out_piece(a, w.begin + token, (kv_head - token) * (int)a.group.d + row, lane >> 1) + 4 * (lane & 1)) = o;
    }
}

// flag: an LDS word that nobody else uses any more; all waves of the workgroup call it.
template <int R, int WAVES>
__device__ __forceinline__ void join_pieces(const Work& w, int kv_head, int* flag) {
    const Attention a = args_again();
    wait_stores_performed();
    __syncthreads();
    if (threadIdx.x == 0) {
        int* count = a.count + (long long)w.slot * a.n_kv_heads + kv_head;
        const int before = arrive_coherent(count);
        *flag = before == w.pieces - 1;
        if (before == w.pieces - 1) *count = 0;  // ready for the next launch
    }
    __syncthreads();
    if (!*flag) return;
    const long long step = (long long)a.n_kv_heads * R * kPartRow;
    const float* base = a.partial + ((long long)w.slot * a.n_kv_heads + kv_head) * R * kPartRow;
    const int rows = min(R, w.tokens * (int)a.group.d - w.tile * R);
    constexpr int N = R / (2 * WAVES) < 4 ? R / (2 * WAVES) : 4;
    if (rows <= 2 * WAVES) join_rows<WAVES, 1, 16>(a, w, R, kv_head, 0, rows, base, step);
    else
        for (int first = 0; first < rows; first += 2 * WAVES * N) join_rows<WAVES, N, 16 / N>(a, w, R, kv_head, first, rows, base, step);
}
// A workgroup's sums of row r, in LDS as `PARTS` partial ones `region` bytes apart, into their place in the scratch.
template <int PARTS, int WAVES>
__device__ __forceinline__ void store_pieces(const unsigned char* sums, int row_bytes, int region, float* place, int rows) {
    const int lane = threadIdx.x & 31;
    const auto scratch = scratch_of(place);
    for (int r = threadIdx.x >> 5; r < rows; r += 2 * WAVES) {
        f32x4 x = *(const f32x4*)(sums + r * row_bytes + lane * 16);
#pragma unroll
        for (int k = 1; k < PARTS; ++k) x += *(const f32x4*)(sums + k * region + r * row_bytes + lane * 16);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), scratch, r * kPartRow * 4 + lane * 16, 0, kCoherent);
    }
}

// ---- few rows: the waves' sums put together, as the only piece or one of several ------------------------------------------------------
// QW rows, NW waves, each with its sums of all rows; lane (c, hh) has row c's features 16 x + 4 hh .. (QW = 16) or 8 x + 4 hh .. .  LDS below kStat is free.
template <int QW, int NW, int kStat, class Acc>
__device__ __forceinline__ void merge_few(const Work& w, int kv_head, int rows, int c, int hh, float m_run, float l_run, const Acc& oacc, unsigned char* lds) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Attention e = args_again();
    constexpr int kRow = 132;
    constexpr int kRegion = QW * kRow;
    float* obuf = (float*)lds;
    float* stat_m = (float*)(lds + kStat);
    float* stat_l = stat_m + NW * QW;
    {
        float l_tot = l_run + __shfl_xor(l_run, 32, 64);
        if (QW == 16) l_tot += __shfl_xor(l_tot, 16, 64);
        if (hh == 0) {
            stat_m[wave * QW + c] = m_run;
            stat_l[wave * QW + c] = l_tot;
        }
    }
    __syncthreads();  // statistics visible; every wave is done with its slots
    const long long part = ((long long)(w.slot + w.piece) * e.n_kv_heads + kv_head) * QW;
    {
        float sm[NW], sl[NW];
#pragma unroll
        for (int x = 0; x < NW; ++x) {
            sm[x] = stat_m[x * QW + c];
            sl[x] = stat_l[x * QW + c];
        }
        float m_all = -INFINITY;
#pragma unroll
        for (int x = 0; x < NW; ++x) m_all = fmaxf(m_all, sm[x]);
        const float m_ref = m_all == -INFINITY ? 0.f : m_all;  // (a row that sees nothing of this piece)
        float l_all = 0.f;
#pragma unroll
        for (int x = 0; x < NW; ++x) l_all += sl[x] * __builtin_amdgcn_exp2f(sm[x] - m_ref);
        // the only piece: normalised here; of several: left for join_pieces
        const float f = __builtin_amdgcn_exp2f(m_run - m_ref) * (w.pieces > 1 ? 1.0f : l_all == 0.f ? 0.f : 1.0f / l_all);
        float* mine = obuf + wave * kRegion + c * kRow;
#pragma unroll
        for (int x = 0; x < (QW == 16 ? 8 : 16); ++x) {  // four consecutive features per write
            const int db = QW == 16 ? x : x >> 2, r = QW == 16 ? 0 : 4 * (x & 3);
            *(float4*)(mine + (QW == 16 ? 16 * x : 8 * x) + 4 * hh) =
                make_float4(oacc[db][r] * f, oacc[db][r + 1] * f, oacc[db][r + 2] * f, oacc[db][r + 3] * f);
        }
        if (w.pieces > 1 && wave == 0 && hh == 0 && c < rows) store_coherent2(e.partial + (part + c) * kPartRow + 128, m_all, l_all);
    }
    __syncthreads();
    if (w.pieces > 1) {
        store_pieces<NW, NW>(lds, kRow * 4, kRegion * 4, e.partial + part * kPartRow, rows);
        join_pieces<QW, NW>(w, kv_head, (int*)(lds + kStat));
        return;
    }
    for (int idx = tid; idx < rows * 16; idx += 64 * NW) {
        const int r = idx >> 4, ch = idx & 15;
        const float* src = obuf + r * kRow + ch * 8;
        float4 x = *(const float4*)src, y = *(const float4*)(src + 4);
#pragma unroll
        for (int i = 1; i < NW; ++i) {
            const float4 x2 = *(const float4*)(src + i * kRegion), y2 = *(const float4*)(src + i * kRegion + 4);
            x.x += x2.x; x.y += x2.y; x.z += x2.z; x.w += x2.w;
            y.x += y2.x; y.y += y2.y; y.z += y2.z; y.w += y2.w;
        }
        const int row = w.tile * QW + r, token = e.group.of(row);
        u32x4 o;
        o[0] = pack_bf16x2(x.x, x.y); o[1] = pack_bf16x2(x.z, x.w);
        o[2] = pack_bf16x2(y.x, y.y); o[3] = pack_bf16x2(y.z, y.w);
        *(u32x4*)out_piece(e, w.begin + token, (kv_head - token) * (int)e.group.d + row, ch) = o;
    }
}

// ---- launches ------------------------------------------------------------------------------------------------------------------
// Scratch: counters, the plan, then pieces.  Pieces wanted are P per chip, so at most P + n_kv_heads in all (find_work); a divided tile of
// attention_few has at least two, each of which is at least half as long as a piece may be: at most twice as many places are
// used.  attention_many counts a request's pieces as if all its tiles had the keys of the last one, at most twice what they
// have on average: four times.
// Calls whose requests have up to 96 rows, or that have no more tiles of 32 rows than fit the chip at once (two per CU), are attention_few's.
// In µs, attention_few and attention_many: 64 rows behind 1536 on 32 heads 16 / 20, 96 rows 17 / 20, 128 rows (of 128 tiles) 17 / 21, 192 rows 20 / 34;
// 16 requests of 96 rows behind 500 to 2100 29 / 38; 900 tokens behind 3000 on 16 heads over 2 (452 tiles) 78 / 87; four requests of 100 (416
// tiles) 34 / 32 (lost by the rule); 512 tokens behind 1536 (544 tiles) 33 / 33; 20 requests of 128 rows behind 300 to 1000 (2560 tiles) 81 / 74.
// (Tiles of codes: paged_attention8.hip.)
constexpr int kFewRows = 96;
constexpr int kFewTiles = 512;
constexpr int kShortRows = 32;
// Pieces: two workgroups per CU (one token behind 8192 27.4 µs with 768, 27.0 with 512 as with 192 of eight waves), three of
// eight waves for four CUs (16 requests behind 10 to 8000 on 8 heads 28 µs, with 256 pieces 36).
constexpr int kFewPieces = 512, kWidePieces = 192;
// Key tiles that the longest piece may have whatever the cost: 20 stay whole, 21 are divided in two of 10 and 11.  One token behind 576 (19
// tiles) takes 10.3 µs whole and 12.3 in two pieces; behind 2048 14.3 in pieces of 24 tiles, 12.8 in pieces of 20 or 16; 48 rows behind 1300
// 15.9, 14.1 and 14.1; 60 rows behind 400 11.1 whole, 13.3 in pieces of 12.  Just above 20 tiles the rule loses: one token on 32 heads behind
// 641, 672, 768, 1024 and 1056 keys takes 12.2, 10.9, 11.1, 11.7 and 12.4 µs in two pieces, 10.7, 9.2, 9.3, 11.2 and 11.8 whole.
constexpr int kLeast = 20;
// A workgroup per CU, less what the longest piece may be longer than the average.  With 128, 222 and 333: three requests of 40 to 500 tokens
// behind 2000 to 9000 86, 84 and 102 µs, five of 100 to 300 behind 10 to 20000 150, 122 and 130.
constexpr int kManyPieces = 222;
constexpr int kMostSplitHeads = 64;  // (more heads than that fill the chip without dividing keys)
constexpr int kMostFewPieces = 1024;  // of any kind of pool
constexpr int kFewPlaces = 2 * (kMostFewPieces + kMostSplitHeads), kManyPlaces = 4 * (kManyPieces + kMostSplitHeads);
constexpr size_t kPartialBytes = (size_t)(kFewPlaces * 32 > kManyPlaces * 256 ? kFewPlaces * 32 : kManyPlaces * 256) * kPartRow * 4;
constexpr size_t kPlanBytes = ((size_t)JUP_PAGED_MAX_SEQS + 2) * 8;
static_assert(kFewPlaces * 4 <= kCountBytes && kManyPlaces * 4 <= kCountBytes);

template <class K>
hipError_t with_lds(K* kernel, int bytes, bool* done) {  // once per device: a kernel's limit of dynamic LDS
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess || (dev < 64 && __atomic_load_n(done + dev, __ATOMIC_ACQUIRE))) return e;
    e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess && dev < 64) __atomic_store_n(done + dev, true, __ATOMIC_RELEASE);
    return e;
}

// tiles: at most so many tiles of rows per key/value head
template <int R, class K, class A>
hipError_t launch(K* kernel, int threads, int lds, bool* done, A a, long long tiles, int pieces, int places, int least, hipStream_t s) {
    hipError_t e = with_lds(kernel, lds, done);
    if (e != hipSuccess) return e;
    pieces = a.n_kv_heads > kMostSplitHeads ? 0 : (pieces + a.n_kv_heads - 1) / a.n_kv_heads;
    a.chunk_factor = pieces > 0 ? 1.0001f / pieces : 1e30f;
    a.most_places = places / a.n_kv_heads;
    const long long items = tiles + 2 * pieces, grid = items * a.n_kv_heads;
    if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
    a.most_items = (int)items;
    if (a.plan) hipLaunchKernelGGL(plan_work<R>, dim3(1), dim3(1024), 0, s, a, least, (int2*)a.plan);
    hipLaunchKernelGGL(kernel, grid_of(grid), dim3(threads), lds, s, a, least);
    return hipGetLastError();
}


// The call's arguments for the kernels.
inline void set_call(Attention& a, const jup_paged_pool_t& pool, const jup_paged_attention_t& c, int tiled) {
    const int shift = log2_of(pool.page_size);
    a.q = (const u16*)c.q; a.k = (const u16*)pool.k; a.v = (const u16*)pool.v; a.out = (u16*)c.out;
    a.q_row = c.q_row_stride; a.q_head = c.q_head_stride; a.out_row = c.out_row_stride; a.out_head = c.out_head_stride;
    a.block = pool.block_stride; a.head = pool.head_stride; a.slot = pool.slot_stride;
    a.tiled = tiled;
    a.row_start = c.row_start; a.lengths = c.lengths; a.table = c.table; a.table_row = c.table_stride;
    a.n_seqs = c.n_seqs; a.n_rows = c.n_rows; a.n_kv_heads = pool.n_kv_heads; a.n_blocks = pool.n_blocks; a.shift = shift;
    a.positions = c.table_width << shift;
    a.group.set(c.n_heads / pool.n_kv_heads);
    a.scale_log2e = c.scale * 1.4426950408889634f;
    a.count = (int*)c.workspace;
    a.plan = c.n_seqs > 64 ? (const int2*)((char*)c.workspace + kCountBytes) : nullptr;
    a.partial = (float*)((char*)c.workspace + kCountBytes + kPlanBytes);
    a.least_rows = 0; a.most_rows = INT32_MAX;
}

// K: the kernels of a kind of pool, few<QW, NW>() and many<KP, NT, SUB>(), the LDS that they take, pieces that fill the chip, and the most tiles of 32
// rows per call that are for few(); A: their arguments
template <class K, class A>
hipError_t launch_tiles(A a, const jup_paged_attention_t& c, hipStream_t s) {
    const long long rows = (long long)c.n_rows * a.group.d, most = (long long)c.max_new * a.group.d;
    static bool done16[64], done32[64], done16w[64], done32w[64];
    auto few = [&](A x, long long tiles16, long long tiles32) {
        const long long tiles = most <= 16 ? tiles16 : tiles32;
        if (tiles * a.n_kv_heads <= 256)  // a workgroup per CU at most: of eight waves, and pieces for three CUs in four
            return most <= 16 ? launch<16>(K::template few<16, 8>(), 512, K::template few_lds<16, 8>(), done16w, x, tiles, K::template few_pieces<16, 8>(), kFewPlaces, kLeast, s)
                              : launch<32>(K::template few<32, 8>(), 512, K::template few_lds<32, 8>(), done32w, x, tiles, K::template few_pieces<32, 8>(), kFewPlaces, kLeast, s);
        return most <= 16 ? launch<16>(K::template few<16, 4>(), 256, K::template few_lds<16, 4>(), done16, x, tiles, K::template few_pieces<16, 4>(), kFewPlaces, kLeast, s)
                          : launch<32>(K::template few<32, 4>(), 256, K::template few_lds<32, 4>(), done32, x, tiles, K::template few_pieces<32, 4>(), kFewPlaces, kLeast, s);
    };
    if (most <= kFewRows || (rows / 32 + c.n_seqs) * a.n_kv_heads <= K::kTiles) return few(a, rows / 16 + c.n_seqs, rows / 32 + c.n_seqs);
    // Up to 32 requests all go to attention_many, of more those of up to 32 rows to a launch of attention_few (an empty one costs 4 µs).  One
    // launch and two: 15 requests of one token behind 4000 and one of 512 61 and 65 µs, 32 of 1 to 300 behind 100 to 3000 171 and 180, 60 of one
    // behind 2000 and four of 300 142 and 160 (lost by the rule, which knows the number of requests alone); 63 of one behind 1000 and one of 512
    // 76 and 66, 63 behind 4000 and one of 256 804 and 760.
    const bool all = c.n_seqs <= 32;
    A longer = a;
    longer.least_rows = all ? 0 : kShortRows + 1;
    // Tiles of 256, 128 or 64 rows, by how many of 256 there are at most.  In µs, tiles of 256 / 128 / 64 rows; first the number of tiles of 256:
    //   1280 (four prompts, 40 heads) 292 / 320 / 458;  520 (16384 tokens, 8 heads) 542 / 594 / 782;  384 (2900 tokens, 32 heads) 100 / 104 / 141;
    //   360 (2048 tokens, 40 heads) 78 / 76 / 101;  320 (three chunks, 40 heads) 64 / 55 / 74;  288 (2048 tokens, 32 heads) 66 / 57 / 81;  264 (2048 behind
    //   8192, 32 heads on 8) 317 / 333 / 438;  160 (1024 tokens) 42 / 31 / 32;  128 (768 behind 1536) 54 / 61 / 57;  96 (512 behind 1536) 43 / 36 / 33.
    // (No number of tiles alone decides: 264 and 128 lose 5 and 12 % by the rule.)
    const long long groups = (rows / 256 + c.n_seqs) * a.n_kv_heads;
    static bool done256[64], done128[64], done64[64];
    hipError_t e = groups >= 384   ? launch<256>(K::template many<1, 2, 2>(), 512, K::template many_lds<1, 2, 2>(), done256, longer, rows / 256 + c.n_seqs, kManyPieces, kManyPlaces, kLeast, s)
                   : groups >= 112 ? launch<128>(K::template many<2, 2, 1>(), 512, K::template many_lds<2, 2, 1>(), done128, longer, rows / 128 + c.n_seqs, kManyPieces, kManyPlaces, kLeast, s)
                                   : launch<64>(K::template many<4, 1, 1>(), 512, K::template many_lds<4, 1, 1>(), done64, longer, rows / 64 + c.n_seqs, kManyPieces, kManyPlaces, kLeast, s);
    if (e != hipSuccess || all) return e;
    a.most_rows = kShortRows;  // (one tile each)
    return few(a, 0, c.n_seqs);
}

}  // namespace
}  // namespace jup
