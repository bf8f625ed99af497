// Attention of the new tokens of a ragged batch over a paged cache (include/jupiter_paged.h).
//
// Rows.  A key/value head serves G = n_heads / n_kv_heads query heads, so the rows that read the same keys are (token, query
// head of the group): row r of a request is token r / G, head r % G.  A workgroup has a TILE of such rows of one request and one
// key/value head and a range of its keys.
//
// Who does what is found on the GPU: lengths are known nowhere else.  Every wave reads the lengths of all requests (64 lanes, a
// prefix sum), so a launch needs no table of work and no launch before it: the host's grid is an upper bound, and the
// workgroups past the last piece of work leave.  Of more than 64 requests plan_work() makes a table first.  See find_work().
#include "paged.h"

namespace jup {
namespace {

__device__ inline f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

constexpr int kKT = 32;                // keys per tile
constexpr int kTileBytes = kKT * 256;  // a K or V tile: 32 rows of 128 bf16

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
// The arguments, read from memory where they are used: behind a main loop that needs the scalar registers itself.
__device__ __forceinline__ Attention args_again() {
    typedef const __attribute__((address_space(4))) char* kernarg;
    kernarg p = (kernarg)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const Attention*)p;
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
__device__ __forceinline__ const char* group_base(const Attention& a, const u16* pool, int block, int key) {
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
// What was taken out of a key's values, for four features from `feature` on (registers r .. r + 3 of sums), if the row sees the key.
template <class V>
__device__ __forceinline__ void add_not_finite(V& sums, int r, const char* row, int feature, bool sees) {
    const u32x2 v = *(const u32x2*)(row + feature * 2);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const unsigned bad = not_finite(v[e]);
        if (sees && (bad & 0x8000u)) sums[r + 2 * e] += bf2f((u16)v[e]);
        if (sees && (bad >> 31)) sums[r + 2 * e + 1] += bf2f((u16)(v[e] >> 16));
    }
}
// Whether a row of values in memory has any (all lanes get the same).
__device__ __forceinline__ bool row_not_finite(const char* row) {
    return __any(not_finite(*(const unsigned*)(row + 4 * (threadIdx.x & 63))) != 0);
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

// ---- few rows ----------------------------------------------------------------------------------------------------------------
// Decoding and verification: a handful of rows against a long cache, bound by reading keys and values (and calls of so few rows that
// taller tiles would leave CUs without any).  A tile has QW = 16 or
// 32 rows, and four waves divide the piece's key tiles: each works alone on the tiles wave, wave + 4, ..., with one LDS
// slot for a K and one for a V tile, and refills the K slot as soon as the scores are out of it and the V slot as soon as the products
// are.  Two workgroups share a CU, so 128 KB are in flight on it, and one's entry and merge lie under the other's loads.
// Where there is a workgroup per CU at most, eight waves divide the keys, and there are half as many pieces to put together: one token
// behind 8192 31 -> 28 µs, behind 65536 with four query heads per key head 71 -> 61.
// Keys and values of 64 requests of one token (550 MB) pass in 110 µs, 5.0 TB/s; of 16 requests of five tokens, whose lengths are
// uneven, in 45 µs, 5.4 TB/s (the last-level cache holds some of them from call to call).  One token behind 576 takes 10 µs: lengths,
// block numbers, a tile and its neighbours, the merge of the waves, each a trip to memory or through LDS behind the other.
// Transposed products, S^T = K Q^T and O^T += V^T P^T: a lane owns a row, whose statistics are scalars of the lane.
//   QW = 32, 32x32x16 (lane = 32 hh + c): A[m = c][k = 8 hh + e], B[k = 8 hh + e][n = c], D[m = 8 (i/4) + 4 hh + i%4][n = c].
//   QW = 16, 16x16x32 (lane = 16 hh + c): A[m = c][k = 8 hh + e], B[k = 8 hh + e][n = c], D[m = 4 hh + i][n = c].
// P^T is taken as the scores lie in the accumulators; V^T is read for exactly that order of keys.
// LDS tiles, rows of 256 bytes in 16 chunks of 16:  K: chunk ch of row r at position ch ^ (r & 15);  V: at (((ch >> 2) ^ (r & 3)) << 2) | (ch & 3).
template <int QW, int NW>
struct Few {
    static constexpr int kQ = NW * 2 * kTileBytes;             // the tile of rows, K layout
    static constexpr int kStat = kQ + QW * 256;                // [2][waves][QW] maxima and sums
    static constexpr int kLds = kStat + 2 * NW * QW * 4;
    static_assert(NW * QW * 132 * 4 <= kStat, "merge regions overlap the statistics");
    static_assert((8 / NW) * kLds <= 160 * 1024, "two workgroups of four waves share a CU");
};

template <int QW, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attention_few(const Attention args, int least) {
    typedef Few<QW, NW> L;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & (QW - 1), hh = lane / QW;
    // consecutive workgroups are the heads of a piece: a head's pieces meet on one XCD where the heads are a multiple of 8
    const int kv_head = (int)(block_number() % (unsigned)args.n_kv_heads), item = (int)(block_number() / (unsigned)args.n_kv_heads);
    Work w;
    if (!find_work<QW>(args, item, least, w)) return;
    w.make_uniform();
    const Attention a = args_again();
    const int G = a.group.d;
    const int rows = min(QW, w.tokens * G - w.tile * QW);
    const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_byte_address(lds));
    const int lrow = lane >> 4, lp = lane & 15;

    // the rows of q into LDS; past the last one, that one again
    for (int r0 = 4 * wave; r0 < QW; r0 += 4 * NW) {
        const int r = r0 + lrow;
        const int row = w.tile * QW + min(r, rows - 1), token = a.group.of(row);
        const u16* from = a.q + (long long)(w.begin + token) * a.q_row + (long long)(kv_head * G + row - token * G) * a.q_head;
        load_to_lds_16(from + (lp ^ (r & 15)) * 8, lds0 + L::kQ + r0 * 256);
    }
    const int last_key = w.keys - 1;
    const int my_token = a.group.of(w.tile * QW + min(c, rows - 1));
    const int q_abs = w.before + my_token;                                          // the last key this lane's row sees
    const int first_token = a.group.of(w.tile * QW);
    const int first_masked = (int)max((long long)w.before + first_token + 1, 0ll) / kKT;  // tiles before it: every row sees every key
    const int* table_row = (const int*)uniform_ptr((const char*)(a.table + w.seq * a.table_row));
    const u16* k_pool = a.k + kv_head * a.head;
    const u16* v_pool = a.v + kv_head * a.head;
    const unsigned row_bytes = (unsigned)(a.slot * 2);

    auto fill = [&](int tile, const Blocks& b, bool v_part) __attribute__((always_inline)) {
        unsigned slot = lds0 + wave * 2 * kTileBytes + (v_part ? kTileBytes : 0);
        asm volatile("" : "+v"(slot));  // (from a vector register on purpose: the compiler keeps it in one, and else hands that to the loads)
        const unsigned dst = __builtin_amdgcn_readfirstlane(slot);
#pragma unroll
        for (int j = 0; j < 8; ++j) {  // four rows (1 KB): lane i lands at row 4j + (i >> 4), position i & 15
            const char* base = group_base(a, v_part ? v_pool : k_pool, b.id[j >> 1], tile * kKT + 8 * (j >> 1));
            const unsigned ch = v_part ? (((lp >> 2) ^ lrow) << 2) | (lp & 3) : lp ^ (4 * (j & 3) + lrow);
            load_to_lds_16(base, (4 * (j & 1) + lrow) * row_bytes + ch * 16, dst + j * 1024);
        }
    };
    int tile = w.tile_lo + wave;
    Blocks here{}, next{};
    if (tile < w.tile_hi) {
        here = blocks_of(a, table_row, tile, last_key);
        fill(tile, here, false);
        fill(tile, here, true);
        if (tile + NW < w.tile_hi) next = blocks_of(a, table_row, tile + NW, last_key);
        asm volatile("s_waitcnt vmcnt(16)" ::: "memory");  // the rows of q have landed, the tiles are on their way
    } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    __builtin_amdgcn_s_barrier();

    constexpr int KS = QW == 16 ? 4 : 8;   // MFMA steps over the head's 128 features
    constexpr int NS = QW == 16 ? 8 : 16;  // scores of a tile per lane
    constexpr int DB = QW == 16 ? 8 : 4;   // output blocks of QW features
    constexpr int NR = QW == 16 ? 4 : 16;  // registers of one
    typedef float acc_t __attribute__((ext_vector_type(NR)));
    constexpr unsigned kStep = QW == 16 ? 64 : 32;  // 16-byte chunk `hh` of a K row; the next MFMA step's is an XOR away
    const unsigned k_lane = c * 256 + ((hh ^ (c & 15)) * 16);
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const bf16x8*)(lds + L::kQ + (k_lane ^ (kStep * ks)));
    acc_t oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < NR; ++r) oacc[db][r] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    const int quad = lane >> 4, s = lane & 15;
    const int vt_row = QW == 16 ? 4 * quad + (s >> 2) : 4 * (quad >> 1) + (s >> 2);
    const unsigned v_base = lds0 + wave * 2 * kTileBytes + kTileBytes;
    unsigned v_lane[4];  // by 64-byte feature group
#pragma unroll
    for (int db = 0; db < 4; ++db)
        v_lane[db] = v_base + vt_row * 256 + ((db ^ (vt_row & 3)) << 6) + ((QW == 16 ? 0 : 2 * (quad & 1)) + ((s & 3) >> 1)) * 16 + 8 * (s & 1);
    auto key_of = [](int r) { return (QW == 16 ? 16 : 8) * (r >> 2) + (r & 3); };  // of the lane's score r, less 4 hh
    const unsigned char* k_base = lds + wave * 2 * kTileBytes;
    bool special = false;  // values that are no numbers were taken out of a tile (of this lane's pieces)

    for (; tile < w.tile_hi; tile += NW) {
        const bool more = tile + NW < w.tile_hi;
        const unsigned there = rows_there(a, here, tile, last_key);
        asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // the K tile has landed; V may be in flight

        // ---- S^T = K Q^T ----
        bf16x8 kf[8];
        float sv[NS];
        if constexpr (QW == 16) {
#pragma unroll
            for (int f = 0; f < 8; ++f) kf[f] = *(const bf16x8*)(k_base + (f >> 2) * 4096 + (k_lane ^ (kStep * (f & 3))));
            f32x4 sacc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int f = 0; f < 8; ++f) sacc[f & 1] = mfma16(kf[4 * (f & 1) + (f >> 1)], qf[f >> 1], sacc[f & 1]);
#pragma unroll
            for (int r = 0; r < NS; ++r) sv[r] = sacc[r >> 2][r & 3];
        } else {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) kf[ks] = *(const bf16x8*)(k_base + (k_lane ^ (kStep * ks)));
            f32x16 sacc;
#pragma unroll
            for (int r = 0; r < 16; ++r) sacc[r] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) sacc = mfma32(kf[ks], qf[ks], sacc);
#pragma unroll
            for (int r = 0; r < NS; ++r) sv[r] = sacc[r];
        }
        if (more) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the K slot has been read
            fill(tile + NW, next, false);
        }

        // ---- online softmax ----
        const bool masked = tile >= first_masked || there != ~0u;
        if (masked) {
            // (opaque: keeps this a branch, as selects it would run for every tile, and its numbers out of the registers between tiles)
            int quarter = 4 * hh;
            asm volatile("" : "+v"(quarter));
#pragma unroll
            for (int r = 0; r < NS; ++r) {
                const int key = quarter + key_of(r);
                if (tile * kKT + key > q_abs || !((there >> key) & 1)) sv[r] = -INFINITY;
            }
        }
        float mt = -INFINITY;
#pragma unroll
        for (int r = 0; r < NS; ++r) mt = fmaxf(mt, sv[r]);
        if constexpr (QW == 16) mt = max_across_rows(mt);
        mt = max_across_halves(mt) * a.scale_log2e;  // the scale is positive
        // The reference of the exponentials moves only when a tile's maximum exceeds it by 2^8: sums are rescaled a few times per
        // piece, and the common factor goes with the normalisation.
        const bool grow = mt > m_run + 8.0f;
        const float m_new = grow ? mt : m_run;
        const float m_safe = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = grow ? __builtin_amdgcn_exp2f(m_run - m_safe) : 1.0f;
        const bool rescale = grow && m_run != -INFINITY;
        float ps = 0.f;
        bf16x8 pf[NS / 8];
#pragma unroll
        for (int r = 0; r < NS; ++r) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[r], a.scale_log2e, -m_safe));
            ps += p;
            pf[r >> 3][r & 7] = (__bf16)p;  // the operand of the second product: 2^-8 of each probability
        }
        l_run = l_run * alpha + ps;
        m_run = m_new;
        if (__any(rescale)) {
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < NR; ++r) oacc[db][r] *= alpha;
        }

        // ---- O^T += V^T P^T ----
        if (more) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // V has landed, the next K may be in flight
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (masked) {
            asm volatile("");
#pragma unroll
            for (int j = 0; j < 8; ++j)  // rows 4j .. 4j + 3
                special |= clean_piece(lds + wave * 2 * kTileBytes + kTileBytes + j * 1024 + lane * 16, (there >> (4 * j + lrow)) & 1);
        }
#pragma unroll
        for (int f = 0; f < 8; ++f) {
            // QW = 32: feature block f / 2, key half f % 2; QW = 16: feature block f, all 32 keys
            const unsigned at = v_lane[f / 2] + (QW == 16 ? (f % 2) * 32 : (f % 2) * 16 * 256);
            const u32x2 lo = read_tr(at), hi = read_tr(at + (QW == 16 ? 16 * 256 : 8 * 256));
            const bf16x8 v = __builtin_bit_cast(bf16x8, (u32x4){lo[0], lo[1], hi[0], hi[1]});
            if constexpr (QW == 16) oacc[f] = mfma16(v, pf[0], oacc[f]);
            else oacc[f / 2] = mfma32(v, pf[f % 2], oacc[f / 2]);
        }
        if (more) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the V slot has been read
            fill(tile + NW, next, true);
            here = next;
            if (tile + 2 * NW < w.tile_hi) next = blocks_of(a, table_row, tile + 2 * NW, last_key);
        }
    }

    if (__any(special)) {  // once in a blue moon
        for (tile = w.tile_lo + wave; tile < w.tile_hi; tile += NW) {
            const Blocks b = blocks_of(a, table_row, tile, last_key);
            const unsigned there = rows_there(a, b, tile, last_key);
            if (tile < first_masked && there == ~0u) continue;
            for (int k = 0; k < kKT; ++k) {
                if (!((there >> k) & 1)) continue;
                const char* row = group_base(a, v_pool, table_row[(tile * kKT + k) >> a.shift], tile * kKT + (k & ~7)) + (k & 7) * row_bytes;
                if (!row_not_finite(row)) continue;
#pragma unroll
                for (int x = 0; x < (QW == 16 ? 8 : 16); ++x) {
                    const int db = QW == 16 ? x : x >> 2, r = QW == 16 ? 0 : 4 * (x & 3);
                    add_not_finite(oacc[db], r, row, (QW == 16 ? 16 * x : 8 * x) + 4 * hh, tile * kKT + k <= q_abs);
                }
            }
        }
    }

    // ---- the waves' sums put together ----
    const Attention e = args_again();
    constexpr int kRow = 132;
    constexpr int kRegion = QW * kRow;
    float* obuf = (float*)lds;
    float* stat_m = (float*)(lds + L::kStat);
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
        join_pieces<QW, NW>(w, kv_head, (int*)(lds + L::kStat));
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

// ---- many rows -----------------------------------------------------------------------------------------------------------------
// Prompts and long chunks, bound by the matrix cores.  Eight waves of 32 rows each; keys come in steps, K and V in LDS for all
// waves, and the waves meet once per step.  Two waves share a SIMD: one's exponentials lie under the other's products.
// KP parts of the keys: a workgroup has 256 / KP rows, and KP waves divide the keys of 32 of them and add up through LDS at the
// end.  One part reads a key for the most rows; more parts make more workgroups of fewer rows, where rows are few or
// where triangles of different sizes are to be dealt to the CUs.  Where one request's keys are far more than the others', they are divided
// among workgroups: five requests of 100 to 300 tokens behind 10 to 20000 take 114 µs instead of 342, three of 40 to 500 behind 2000 to 9000
// 78 instead of 138 (but six of 1 to 600 behind 10 to 32000 589 instead of 580: 320 equal pieces for 256 CUs).
// Measured: a prompt of 16384 tokens on 8 heads in 540 µs, 1019 TFLOP/s, matrix cores busy 44 % of the clocks, LDS 22 %.  Without loads
// from memory it takes 92 % of that, without exponentials 89 %, without LDS reads 73 %, without products 95 %: no one unit binds it, but the
// waves wait for one another's, as registers leave room for two per SIMD.  (The shapes of 128 and 64 rows were not taken apart like this.)
// Three per SIMD of half the keys each: 970 instead of 1050 TFLOP/s.  One wave per SIMD of 64 rows: 789.  Half the waves a product behind the
// others: 632 instead of 590 µs.  Four prompts of 700 to 4100 tokens (40 heads, 292 µs, 735 TFLOP/s) have 1240 such tiles of 10 steps each,
// whose entry and end (15 of 60 µs) nothing overlaps: LDS has room for one workgroup, and a workgroup has one tile.
template <int NW, int KP, int NT, int SUB>
struct Many {
    static constexpr int kWaves = NW;
    static constexpr int kRows = 32 * NW / KP;
    static constexpr int kSubTiles = KP * NT;                // a wave works through NT tiles at a time, SUB times between two meetings
    static constexpr int kStepTiles = SUB * kSubTiles;
    static constexpr int kStep = kStepTiles * kKT;           // keys of a step
    static constexpr int kHalf = kStepTiles * kTileBytes;    // K tiles, then V tiles
    static constexpr int kGroups = kStepTiles * 4 / kWaves;  // groups of eight rows that a wave fetches per step: wave, wave + NW
    static_assert(kGroups * kWaves == kStepTiles * 4);
    static constexpr int kRowBytes = 132 * 4;                // a row of a part's sums
    static constexpr int kSteps = 2 * 2 * kHalf, kSums = 32 * NW * kRowBytes, kQ = 32 * NW * 256;
    static constexpr int kThere = (kSteps > kSums ? kSteps > kQ ? kSteps : kQ : kSums);  // [2][kStepTiles * 4] bytes: which rows of a step's groups are keys
    static constexpr int kFlag = kThere + 64;
    static constexpr int kStat = kFlag + 64;                 // [2][waves][32] maxima and sums
    static constexpr int kLds = kStat + (KP > 1 ? 2 * 32 * NW * 4 : 0);
    // queries go through the second step's place, the first step is fetched beside them
    static constexpr int kQAt = kThere - kQ;
    static_assert(kLds <= 160 * 1024 && 2 * kStepTiles * 4 <= 64 && kQAt >= 2 * kHalf);
};

template <int NW, int KP, int NT, int SUB, int OCC>
__global__ __launch_bounds__(64 * NW, OCC) void attention_many(const Attention args, int least) {
    typedef Many<NW, KP, NT, SUB> L;
    constexpr int kHalf = L::kHalf, kStep = L::kStep, kRows = L::kRows;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 31, hh = lane >> 5;
    const int part = wave % KP, r_wave = wave / KP * 32;  // this wave's keys of a step, and its rows
    const int kv_head = (int)(block_number() % (unsigned)args.n_kv_heads), item = (int)(block_number() / (unsigned)args.n_kv_heads);
    Work w;
    if (!find_work<kRows>(args, item, least, w)) return;
    w.make_uniform();
    const Attention a = args_again();
    const int G = a.group.d;
    const int rows = min(kRows, w.tokens * G - w.tile * kRows);
    const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_byte_address(lds));
    const int lrow = lane >> 4, lp = lane & 15;

    // this wave's eight rows of a step: group `wave` (and wave + 8)
    const int last_key = w.keys - 1, first_key = w.tile_lo * kKT;
    const int n = (w.tile_hi - w.tile_lo + L::kStepTiles - 1) / L::kStepTiles;
    const int* table_row = (const int*)uniform_ptr((const char*)(a.table + w.seq * a.table_row));
    typedef const __attribute__((address_space(4))) int* scalar;
    const u16* k_pool = a.k + kv_head * a.head;
    const u16* v_pool = a.v + kv_head * a.head;
    // keys of this piece: up to the last key, or where the next piece begins
    const int end_key = min(last_key + 1, w.tile_hi * kKT);
    unsigned k_off[2], v_off[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const unsigned row = (unsigned)(a.slot * 2) * (4 * j + lrow);
        k_off[j] = row + (lp ^ ((8 * wave + 4 * j + lrow) & 15)) * 16;
        v_off[j] = row + ((((lp >> 2) ^ lrow) << 2) | (lp & 3)) * 16;
    }
    struct Ids {
        int id[L::kGroups];
    };
    auto ids_of = [&](int i) {
        Ids x;
#pragma unroll
        for (int g = 0; g < L::kGroups; ++g) x.id[g] = ((scalar)table_row)[min(first_key + i * kStep + 8 * NW * g + 8 * wave, last_key) >> a.shift];
        return x;
    };
    unsigned hole = 0;  // bit: in that slot, some of this wave's rows are no keys
    // K of step i, or V, and which rows are keys
    auto fill = [&](int i, const Ids& ids, bool v_part) __attribute__((always_inline)) {
        if (v_part) hole &= ~(1u << (i & 1));
#pragma unroll
        for (int g = 0; g < L::kGroups; ++g) {
            const int mine = first_key + i * kStep + 8 * NW * g + 8 * wave, key = min(mine, last_key & ~7);  // (groups behind the last key repeat its own)
            unsigned slot = lds0 + (unsigned)(i & 1) * 2 * kHalf + (v_part ? kHalf : 0) + (NW * g + wave) * 2048;
            asm volatile("" : "+v"(slot));  // (see attention_few)
            const unsigned dst = __builtin_amdgcn_readfirstlane(slot);
            const char* base = group_base(a, v_part ? v_pool : k_pool, ids.id[g], key);
#pragma unroll
            for (int j = 0; j < 2; ++j) load_to_lds_16(base, v_part ? v_off[j] : k_off[j], dst + j * 1024);
            if (!v_part) continue;
            const int left = end_key - mine;
            const unsigned there = (unsigned)ids.id[g] >= (unsigned)a.n_blocks || left <= 0 ? 0u : left >= 8 ? 0xFFu : (1u << left) - 1;
            hole |= there == 0xFFu ? 0u : 1u << (i & 1);
            if (lane == 0) lds[L::kThere + (i & 1) * L::kStepTiles * 4 + NW * g + wave] = (unsigned char)there;
        }
    };
    // Queries: this wave's 32 rows go through LDS (the second half of the steps' places) into B operands; rows past the last one repeat it.
    // (As plain loads they would be waited for with everything issued behind them: the compiler does not know of the tiles.)
    unsigned char* q_lds = lds + L::kQAt + wave * 8192;
    const unsigned q_at = lds0 + L::kQAt + wave * 8192;
    for (int r0 = 0; r0 < 32; r0 += 4) {
        const int row = w.tile * kRows + min(r_wave + r0 + lrow, rows - 1), token = a.group.of(row);
        const u16* from = a.q + (long long)(w.begin + token) * a.q_row + (long long)(kv_head * G + row - token * G) * a.q_head;
        load_to_lds_16(from + (lp ^ ((r0 + lrow) & 15)) * 8, __builtin_amdgcn_readfirstlane(q_at + r0 * 256));
    }
    if (tid == 0) lds[L::kFlag] = 0;
    Ids ids{};
    if (n > 0) ids = ids_of(0);
    auto fill_next = [&](int i, bool k_part, bool v_part) __attribute__((always_inline)) {  // step i, then the block numbers of the one behind it
        if (i >= n) return;
        if (k_part) fill(i, ids, false);
        if (v_part) {
            const Ids next = ids_of(i + 1);
            fill(i, ids, true);
            ids = next;
        }
    };
    fill_next(0, true, true);

    // Sub-steps (NT tiles per part) before this one: every row of the workgroup sees all their keys.
    constexpr int kSub = L::kSubTiles * kKT;
    const int open = __builtin_amdgcn_readfirstlane((int)min(max(max((long long)w.before + a.group.of(w.tile * kRows) + 1, 0ll) - first_key, 0ll) / kSub, (long long)n * SUB));
    // Behind the wait for this wave's rows of step i: rows that are no keys become 0, and where some row sees some key and another
    // does not, values that are no numbers do.
    bool special = false;
    auto clean = [&](int i) __attribute__((always_inline)) {
        if ((i + 1) * SUB <= open && !((hole >> (i & 1)) & 1)) return;
#pragma unroll
        for (int g = 0; g < L::kGroups; ++g) {
            const unsigned there = lds[L::kThere + (i & 1) * L::kStepTiles * 4 + NW * g + wave];
            unsigned char* at = lds + (i & 1) * 2 * kHalf + kHalf + (NW * g + wave) * 2048 + lane * 16;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const bool key = (there >> (4 * j + lrow)) & 1;
                if (i * SUB + (NW * g + wave) / (4 * L::kSubTiles) >= open || !key) special |= clean_piece(at + j * 1024, key);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    // the last key that this lane's row sees; sub-steps that some row of this wave sees
    const int sees_to = w.before + a.group.of(w.tile * kRows + min(r_wave + c, rows - 1));
    const long long seen = (long long)w.before + a.group.of(w.tile * kRows + min(r_wave + 31, rows - 1)) + 1 - first_key;
    const int mine = __builtin_amdgcn_readfirstlane(r_wave >= rows ? 0 : (int)min(max((seen + kSub - 1) / kSub, 0ll), (long long)n * SUB));

    f32x16 o[4];
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] = 0.f;
    const unsigned k_lane = c * 256 + ((hh ^ (c & 15)) * 16);
    const int quad = lane >> 4, sl = lane & 15;
    const int vt_row = 4 * (quad >> 1) + (sl >> 2);
    unsigned v_lane[4];
#pragma unroll
    for (int db = 0; db < 4; ++db)
        v_lane[db] = lds0 + kHalf + vt_row * 256 + ((db ^ (vt_row & 3)) << 6) + (2 * (quad & 1) + ((sl & 3) >> 1)) * 16 + 8 * (sl & 1);
    bf16x8 qf[8];
    // the queries have landed, the first step's loads may be in flight
    if (n > 0) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * L::kGroups) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) qf[ks] = *(const bf16x8*)(q_lds + (k_lane ^ (32 * ks)));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();  // every wave has its queries: the second step may go there
    asm volatile("" ::: "memory");

    for (int i = 0; i < n; ++i) {
        // step i is there for all, and step i - 1 has been read by all
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        clean(i);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // Step i + 1 goes where step i - 1 was.  (Its loads are put between the products: the address path of a CU takes 64 bytes per
        // clock, and with all waves' loads behind the meeting every wave would wait for it there.)
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        if (i * SUB + u >= mine) {
            fill_next(i + 1, u == 0, u == SUB - 1);
            continue;
        }
        const int first_tile = (u * KP + part) * NT;  // of this wave's keys of the sub-step
        const unsigned char* k_base = lds + (i & 1) * 2 * kHalf + first_tile * kTileBytes;
        const unsigned v_slot = (unsigned)(i & 1) * 2 * kHalf + first_tile * kTileBytes;
        const int key0 = first_key + i * kStep + first_tile * kKT;
        unsigned there[NT], whole = ~0u;
#pragma unroll
        for (int t = 0; t < NT; ++t) there[t] = *(const unsigned*)(lds + L::kThere + (i & 1) * L::kStepTiles * 4 + (first_tile + t) * 4);

        // ---- S^T = K Q^T ----
        f32x16 s[NT];
        bf16x8 kf[NT][8];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) kf[t][ks] = *(const bf16x8*)(k_base + t * kTileBytes + (k_lane ^ (32 * ks)));
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) s[t] = mfma32(kf[t][ks], qf[ks], s[t]);
        }
        // the first tile's values are on their way under the exponentials
        u32x4 vf[8];
        auto read_v = [&](int t) __attribute__((always_inline)) {
#pragma unroll
            for (int f = 0; f < 8; ++f) {  // feature block f / 2, key half f % 2
                const unsigned at = v_slot + t * kTileBytes + v_lane[f / 2] + (f % 2) * 16 * 256;
                const u32x2 lo = read_tr(at), hi = read_tr(at + 8 * 256);
                vf[f] = (u32x4){lo[0], lo[1], hi[0], hi[1]};
            }
        };
        read_v(0);

        fill_next(i + 1, u == 0, false);

        // ---- online softmax (see attention_few) ----
        float sv[16 * NT];
#pragma unroll
        for (int r = 0; r < 16 * NT; ++r) sv[r] = s[r >> 4][r & 15];
#pragma unroll
        for (int t = 0; t < NT; ++t) whole &= there[t] = __builtin_amdgcn_readfirstlane(there[t]);
        if (i * SUB + u >= open || whole != ~0u) {
            int quarter = 4 * hh;
            asm volatile("" : "+v"(quarter));
#pragma unroll
            for (int r = 0; r < 16 * NT; ++r) {
                const int key = quarter + 8 * ((r & 15) >> 2) + (r & 3);
                if (key0 + 32 * (r >> 4) + key > sees_to || !((there[r >> 4] >> key) & 1)) sv[r] = -INFINITY;
            }
        }
        float mt = sv[0];
#pragma unroll
        for (int r = 1; r < 16 * NT; ++r) mt = fmaxf(mt, sv[r]);
        mt = max_across_halves(mt) * a.scale_log2e;
        const bool grow = mt > m_run + 8.0f;
        const float m_new = grow ? mt : m_run;
        const float m_safe = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = grow ? __builtin_amdgcn_exp2f(m_run - m_safe) : 1.0f;
        if (__any(grow && m_run != -INFINITY)) {
#pragma unroll
            for (int db = 0; db < 4; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
        }
        float ps = 0.f;
        bf16x8 p[2 * NT];
#pragma unroll
        for (int r = 0; r < 16 * NT; ++r) {
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[r], a.scale_log2e, -m_safe));
            ps += x;
            p[r >> 3][r & 7] = (__bf16)x;
        }
        l_run = l_run * alpha + ps;
        m_run = m_new;

        fill_next(i + 1, false, u == SUB - 1);

        // ---- O^T += V^T P^T ----
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int f = 0; f < 8; ++f) o[f / 2] = mfma32(__builtin_bit_cast(bf16x8, vf[f]), p[2 * t + f % 2], o[f / 2]);
            if (t + 1 < NT) read_v(t + 1);
        }
      }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the step has been read
    }
    if (__any(special)) lds[L::kFlag] = 1;

    // ---- results -------------------------------------------------------------------------------------------------------------
    const Attention e = args_again();
    __syncthreads();  // every wave is done with the steps
    if (lds[L::kFlag]) {  // once in a blue moon: what clean() took out
        for (int tile = w.tile_lo + L::kSubTiles * open; tile < min(w.tile_hi, w.tile_lo + L::kSubTiles * mine); ++tile) {
            if ((tile - w.tile_lo) / NT % KP != part) continue;
            const Blocks ids = blocks_of(a, table_row, tile, last_key);
            const unsigned there = rows_there(a, ids, tile, last_key);
            for (int k = 0; k < kKT; ++k) {
                if (!((there >> k) & 1)) continue;
                const char* row = group_base(a, v_pool, table_row[(tile * kKT + k) >> a.shift], tile * kKT + (k & ~7)) + (k & 7) * (unsigned)(a.slot * 2);
                if (!row_not_finite(row)) continue;
#pragma unroll
                for (int x = 0; x < 16; ++x) add_not_finite(o[x >> 2], 4 * (x & 3), row, 8 * x + 4 * hh, tile * kKT + k <= sees_to);
            }
        }
    }
    float l = l_run + __shfl_xor(l_run, 32, 64), m = m_run;
    float f = 1.0f;  // what this wave's sums are multiplied by
    if (KP > 1) {
        float* stat = (float*)(lds + L::kStat);
        if (hh == 0) {
            stat[wave * 32 + c] = m_run;
            stat[32 * NW + wave * 32 + c] = l;
        }
        __syncthreads();
        const int first = wave / KP * KP;
        m = -INFINITY;
#pragma unroll
        for (int x = 0; x < KP; ++x) m = fmaxf(m, stat[(first + x) * 32 + c]);
        const float ref = m == -INFINITY ? 0.f : m;
        l = 0.f;
#pragma unroll
        for (int x = 0; x < KP; ++x) l += stat[32 * NW + (first + x) * 32 + c] * __builtin_amdgcn_exp2f(stat[(first + x) * 32 + c] - ref);
        f = __builtin_amdgcn_exp2f(m_run - ref);
    }
    const bool pieces = w.pieces > 1;
    if (!pieces) f *= l == 0.f ? 0.f : 1.0f / l;
    const long long place = ((long long)(w.slot + w.piece) * e.n_kv_heads + kv_head) * kRows;
    if (pieces && part == 0 && hh == 0 && r_wave + c < rows) store_coherent2(e.partial + (place + r_wave + c) * kPartRow + 128, m, l);
    if (KP == 1 && !pieces) {  // rows as they are, through LDS to whole lines (a wave reads its own rows only)
        unsigned char* to = lds + (r_wave + c) * 256;  // 16-byte pieces as in a K tile
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            u32x2 y;
            y[0] = pack_bf16x2(o[x >> 2][4 * (x & 3)] * f, o[x >> 2][4 * (x & 3) + 1] * f);
            y[1] = pack_bf16x2(o[x >> 2][4 * (x & 3) + 2] * f, o[x >> 2][4 * (x & 3) + 3] * f);
            *(u32x2*)(to + (x ^ (c & 15)) * 16 + 8 * hh) = y;
        }
        for (int r0 = 0; r0 < 32; r0 += 4) {
            const int r = r_wave + r0 + lrow, row = w.tile * kRows + r;
            if (r >= rows) break;
            const int token = e.group.of(row);
            *(u32x4*)out_piece(e, w.begin + token, (kv_head - token) * (int)e.group.d + row, lp) =
                *(const u32x4*)(lds + r * 256 + (lp ^ (r & 15)) * 16);
        }
        return;
    }
    float* to = (float*)(lds + (part * kRows + r_wave + c) * L::kRowBytes);
#pragma unroll
    for (int x = 0; x < 16; ++x)
        *(float4*)(to + 8 * x + 4 * hh) = make_float4(o[x >> 2][4 * (x & 3)] * f, o[x >> 2][4 * (x & 3) + 1] * f, o[x >> 2][4 * (x & 3) + 2] * f, o[x >> 2][4 * (x & 3) + 3] * f);
    __syncthreads();
    if (pieces) {
        store_pieces<KP, NW>(lds, L::kRowBytes, kRows * L::kRowBytes, e.partial + place * kPartRow, rows);
        join_pieces<kRows, NW>(w, kv_head, (int*)(lds + L::kFlag));
        return;
    }
    for (int idx = tid; idx < rows * 16; idx += 64 * NW) {
        const int r = idx >> 4, ch = idx & 15;
        const char* from = (const char*)lds + r * L::kRowBytes + ch * 32;
        float4 x = *(const float4*)from, y = *(const float4*)(from + 16);
#pragma unroll
        for (int k = 1; k < KP; ++k) {
            const float4 x2 = *(const float4*)(from + k * kRows * L::kRowBytes), y2 = *(const float4*)(from + k * kRows * L::kRowBytes + 16);
            x.x += x2.x; x.y += x2.y; x.z += x2.z; x.w += x2.w;
            y.x += y2.x; y.y += y2.y; y.z += y2.z; y.w += y2.w;
        }
        const int row = w.tile * kRows + r, token = e.group.of(row);
        u32x4 z;
        z[0] = pack_bf16x2(x.x, x.y); z[1] = pack_bf16x2(x.z, x.w);
        z[2] = pack_bf16x2(y.x, y.y); z[3] = pack_bf16x2(y.z, y.w);
        *(u32x4*)out_piece(e, w.begin + token, (kv_head - token) * (int)e.group.d + row, ch) = z;
    }
}

// Check mode.  One wave per (row, query head): 64 keys at a time, a lane has a key's score, then D / 64 columns of the output (rounded up).
__global__ __launch_bounds__(64) void attention_f32(const jup_paged_pool_t pool, const jup_paged_attention_t a, int shift) {
    __shared__ float q[256];
    const int lane = threadIdx.x, row = (int)(block_number() / (unsigned)a.n_heads), head = (int)block_number() - row * a.n_heads;
    if (row >= a.n_rows) return;
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
    for (int i = lane; i < D; i += 64) q[i] = ((const float*)a.q)[row * a.q_row_stride + head * a.q_head_stride + i];
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
                const float* k = (const float*)pool.k + at;
                float sum = 0.f;
                for (int i = 0; i < D; ++i) sum = __builtin_fmaf(q[i], k[i], sum);
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
                if (lane + 64 * c < D) acc[c] = __builtin_fmaf(w, ((const float*)pool.v)[from + lane + 64 * c], acc[c]);
        }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (lane + 64 * c < D) ((float*)a.out)[row * a.out_row_stride + head * a.out_head_stride + lane + 64 * c] = l == 0.f ? 0.f : acc[c] / l;
}

}  // namespace

// ---- launches ------------------------------------------------------------------------------------------------------------------
namespace {

// Scratch: counters, the plan, then pieces.  Pieces wanted are P per chip, so at most P + n_kv_heads in all (find_work); a divided tile of
// attention_few has at least two, each of which is at least half as long as a piece may be: at most twice as many places are
// used.  attention_many counts a request's pieces as if all its tiles had the keys of the last one, at most twice what they
// have on average: four times.
// Calls whose requests have up to 96 rows, or that have no more tiles of 32 rows than fit the chip at once (two per CU), are attention_few's.
// In µs, attention_few and attention_many: 64 rows behind 1536 on 32 heads 16 / 20, 96 rows 17 / 20, 128 rows (of 128 tiles) 17 / 21, 192 rows 20 / 34;
// 16 requests of 96 rows behind 500 to 2100 29 / 38; 900 tokens behind 3000 on 16 heads over 2 (452 tiles) 78 / 87; four requests of 100 (416
// tiles) 34 / 32 (lost by the rule); 512 tokens behind 1536 (544 tiles) 33 / 33; 20 requests of 128 rows behind 300 to 1000 (2560 tiles) 81 / 74.
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
constexpr int kFewPlaces = 2 * (kFewPieces + kMostSplitHeads), kManyPlaces = 4 * (kManyPieces + kMostSplitHeads);
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
template <int R, class K>
hipError_t launch(K* kernel, int threads, int lds, bool* done, Attention a, long long tiles, int pieces, int places, int least, hipStream_t s) {
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

}  // namespace

hipError_t launch_paged_attention(const jup_paged_pool_t& pool, const jup_paged_attention_t& c, hipStream_t s, int tiled) {
    const int shift = log2_of(pool.page_size);
    if (pool.dtype == JUP_F32) {
        hipLaunchKernelGGL(attention_f32, grid_of((long long)c.n_rows * c.n_heads), dim3(64), 0, s, pool, c, shift);
        return hipGetLastError();
    }
    Attention a{};
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
    const long long rows = (long long)c.n_rows * a.group.d, most = (long long)c.max_new * a.group.d;
    static bool done16[64], done32[64], done16w[64], done32w[64];
    auto few = [&](Attention x, long long tiles16, long long tiles32) {
        const long long tiles = most <= 16 ? tiles16 : tiles32;
        if (tiles * pool.n_kv_heads <= 256)  // a workgroup per CU at most: of eight waves, and pieces for three CUs in four
            return most <= 16 ? launch<16>(attention_few<16, 8>, 512, Few<16, 8>::kLds, done16w, x, tiles, kWidePieces, kFewPlaces, kLeast, s)
                              : launch<32>(attention_few<32, 8>, 512, Few<32, 8>::kLds, done32w, x, tiles, kWidePieces, kFewPlaces, kLeast, s);
        return most <= 16 ? launch<16>(attention_few<16, 4>, 256, Few<16, 4>::kLds, done16, x, tiles, kFewPieces, kFewPlaces, kLeast, s)
                          : launch<32>(attention_few<32, 4>, 256, Few<32, 4>::kLds, done32, x, tiles, kFewPieces, kFewPlaces, kLeast, s);
    };
    if (most <= kFewRows || (rows / 32 + c.n_seqs) * pool.n_kv_heads <= kFewTiles) return few(a, rows / 16 + c.n_seqs, rows / 32 + c.n_seqs);
    // Up to 32 requests all go to attention_many, of more those of up to 32 rows to a launch of attention_few (an empty one costs 4 µs).  One
    // launch and two: 15 requests of one token behind 4000 and one of 512 61 and 65 µs, 32 of 1 to 300 behind 100 to 3000 171 and 180, 60 of one
    // behind 2000 and four of 300 142 and 160 (lost by the rule, which knows the number of requests alone); 63 of one behind 1000 and one of 512
    // 76 and 66, 63 behind 4000 and one of 256 804 and 760.
    const bool all = c.n_seqs <= 32;
    Attention longer = a;
    longer.least_rows = all ? 0 : kShortRows + 1;
    // Tiles of 256, 128 or 64 rows, by how many of 256 there are at most.  In µs, tiles of 256 / 128 / 64 rows; first the number of tiles of 256:
    //   1280 (four prompts, 40 heads) 292 / 320 / 458;  520 (16384 tokens, 8 heads) 542 / 594 / 782;  384 (2900 tokens, 32 heads) 100 / 104 / 141;
    //   360 (2048 tokens, 40 heads) 78 / 76 / 101;  320 (three chunks, 40 heads) 64 / 55 / 74;  288 (2048 tokens, 32 heads) 66 / 57 / 81;  264 (2048 behind
    //   8192, 32 heads on 8) 317 / 333 / 438;  160 (1024 tokens) 42 / 31 / 32;  128 (768 behind 1536) 54 / 61 / 57;  96 (512 behind 1536) 43 / 36 / 33.
    // (No number of tiles alone decides: 264 and 128 lose 5 and 12 % by the rule.)
    const long long groups = (rows / 256 + c.n_seqs) * pool.n_kv_heads;
    static bool done256[64], done128[64], done64[64];
    hipError_t e = groups >= 384   ? launch<256>(attention_many<8, 1, 2, 2, 2>, 512, Many<8, 1, 2, 2>::kLds, done256, longer, rows / 256 + c.n_seqs, kManyPieces, kManyPlaces, kLeast, s)
                   : groups >= 112 ? launch<128>(attention_many<8, 2, 2, 1, 2>, 512, Many<8, 2, 2, 1>::kLds, done128, longer, rows / 128 + c.n_seqs, kManyPieces, kManyPlaces, kLeast, s)
                                   : launch<64>(attention_many<8, 4, 1, 1, 2>, 512, Many<8, 4, 1, 1>::kLds, done64, longer, rows / 64 + c.n_seqs, kManyPieces, kManyPlaces, kLeast, s);
    if (e != hipSuccess || all) return e;
    a.most_rows = kShortRows;  // (one tile each)
    return few(a, 0, c.n_seqs);
}

}  // namespace jup

extern "C" size_t jup_paged_workspace_bytes(void) {
    return jup::kCountBytes + (jup::kPlanBytes + jup::kPartialBytes > jup::kVerifyBytes ? jup::kPlanBytes + jup::kPartialBytes : jup::kVerifyBytes);
}
