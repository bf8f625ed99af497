// Attention of the new tokens of a ragged batch over a paged cache of bf16 values (include/jupiter_paged.h); rows, tiles and pieces:
// paged_work.h.
#include "paged_many.h"

namespace jup {
namespace {

constexpr int kTileBytes = kValueTile;

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
                if (!row_not_finite<JUP_BF16>(row)) continue;
#pragma unroll
                for (int x = 0; x < (QW == 16 ? 8 : 16); ++x) {
                    const int db = QW == 16 ? x : x >> 2, r = QW == 16 ? 0 : 4 * (x & 3);
                    add_not_finite<JUP_BF16>(oacc[db], r, row, (QW == 16 ? 16 * x : 8 * x) + 4 * hh, tile * kKT + k <= q_abs);
                }
            }
        }
    }

    // ---- the waves' sums put together ----
    merge_few<QW, NW, L::kStat>(w, kv_head, rows, c, hh, m_run, l_run, oacc, lds);
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

struct Kernels {
    static constexpr int kTiles = kFewTiles;
    template <int QW, int NW> static auto few() { return attention_few<QW, NW>; }
    template <int QW, int NW> static constexpr int few_lds() { return Few<QW, NW>::kLds; }
    template <int QW, int NW> static constexpr int few_pieces() { return NW == 8 ? kWidePieces : kFewPieces; }
    template <int KP, int NT, int SUB> static auto many() { return attention_many<JUP_BF16, 8, KP, NT, SUB, 2>; }
    template <int KP, int NT, int SUB> static constexpr int many_lds() { return Many<8, KP, NT, SUB, false>::kLds; }
};

}  // namespace

hipError_t launch_paged_attention(const jup_paged_pool_t& pool, const jup_paged_attention_t& c, hipStream_t s, int tiled) {
    if (pool.dtype == JUP_F32) {
        hipLaunchKernelGGL(attention_f32, grid_of((long long)c.n_rows * c.n_heads), dim3(64), 0, s, pool, c, log2_of(pool.page_size));
        return hipGetLastError();
    }
    Attention a{};
    set_call(a, pool, c, tiled);
    return launch_tiles<Kernels>(a, c, s);
}

}  // namespace jup

// what other calls take of a workspace: maps of 2^26 blocks (paged_reorder.hip), lists of 16384 slices of rows (paged_beams.hip)
static_assert(jup::kPartialBytes >= JUP_PAGED_MAX_SEQS * 4ull + 2 * (1ull << 26) && jup::kPartialBytes >= JUP_PAGED_MAX_SEQS * (2ull + JUP_BEAM_MOST) * 8);

extern "C" size_t jup_paged_workspace_bytes(void) {
    return jup::kCountBytes + (jup::kPlanBytes + jup::kPartialBytes > jup::kVerifyBytes ? jup::kPlanBytes + jup::kPartialBytes : jup::kVerifyBytes);
}
