// Attention of the new tokens of a ragged batch over a paged cache of 8-bit codes (include/jupiter_paged.h); rows, tiles and pieces:
// paged_work.h.
//
// Codes are exact in bf16, so products are those of bf16 operands.  Scores are sums over a key's codes times the key's scale; a value's scale goes
// with its probability, s_j p_j, as an operand of the second product, which is bf16.  Tiles of up to 32 rows take it as two: its first eight bits, cut
// off, and the rest of it, which is exact in fp32, rounded (2^-15 is left).  Results are then as far from the formula as their own rounding, 1.66e-3 of the
// whole; with one rounded operand 2.2e-3 to 2.5e-3, and up to 1.54 times as far as that rounding for a few short int8 prompts.  In µs, one operand / two: 512
// int8 tokens behind 1536 42.1 / 46.0 (with the first operand rounded, and the rest looked at for infinities, 48.7), 768 66 / 70, a prompt of 1024 32.7 / 34.1, 64
// behind 576 11.6 / 12.0, 16 requests of five with four heads to a key head 18.0 / 18.3.  Tall tiles (attention_many) round one operand, 2^-8 of it, as they
// do over bf16 values: with two, four prompts of 700 to 4100 tokens take 401 in place of 337.
#include "paged_many.h"

namespace jup {
namespace {

constexpr int kTileBytes = kKT * 128;  // a K or V tile: 32 rows of 128 codes

// Transposing 8-byte LDS read: within each group of 16 lanes, lane i receives as byte r byte (i & 7) of the 8 bytes addressed by lane
// 2r + (i >> 3) of the group.
__device__ __forceinline__ u32x2 read_tr8(unsigned lds_address) {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) i32x2* lds_ptr;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_ptr)(size_t)lds_address));
}

// 4 bytes per lane straight into LDS (see load_to_lds_16).
__device__ inline void load_to_lds_4(const void* gptr, unsigned lds_base) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(gptr), "s"(lds_base) : "memory", "m0");
}

// A 16-byte piece of a row of values in a masked tile; there: the row is a key.  True: something was taken out of it.
__device__ __forceinline__ bool clean_piece8(unsigned char* at, bool there) {
    u32x4 v = *(const u32x4*)at;
    const bool taken = clean_codes(v, there);
    if (taken || !there) *(u32x4*)at = v;
    return taken;
}

// ---- few rows ----------------------------------------------------------------------------------------------------------------
// As attention_few: a tile has QW = 16 or 32 rows, and the waves divide the piece's key tiles, each alone with its own places in LDS.  A tile is half
// as long in bytes, so as many bytes are in flight on a CU with two places per wave, or with one and four workgroups on the CU.  That is what 16 rows
// and four waves have: one workgroup's entry and merge then lie under three others' loads.  In µs, two places and one: 64 requests of one
// token behind 16 to 8192, 32 heads on 8 73.7 / 70.4 (68.2 with twice as many pieces, 70.1 without a product), 16 of five behind 500 to 2100 41.3 /
// 35.7; behind 4096 each 114 / 117 (4.7 TB/s).
// LDS tiles, rows of 128 bytes in 8 chunks of 16:  K: chunk ch of row r at position ch ^ (r / 2 & 7);  V: at ch ^ turn(r), such that the rows of a
// transposing read lie in different banks.  Behind them the scales of the tile's keys and values, 32 each.
// K is read 16 codes at a time, two steps of the product: step (j, s) has the features 16 (chunk of j) + 8 s .. + 7, and queries are read so too.
template <int QW, int NW>
struct Few8 {
    static constexpr int kPlaces = QW == 16 && NW == 4 ? 1 : 2;
    static constexpr int kGroups = QW == 16 && NW == 4 ? 4 : 8 / NW;  // workgroups on a CU
    static constexpr int kScales = 2 * kTileBytes;             // of a place: K tile, V tile, scales
    static constexpr int kPlace = kScales + 256;
    static constexpr int kWave = kPlaces * kPlace;
    static constexpr int kQ = NW * kWave;                      // the tile of rows: 256 bytes each, chunk ch at position ch ^ (r & 15)
    static constexpr int kStat = kQ + QW * 256;                // [2][waves][QW] maxima and sums
    static constexpr int kLds = kStat + 2 * NW * QW * 4;
    static_assert(NW * QW * 132 * 4 <= kStat, "merge regions overlap the statistics");
    static_assert(kGroups * kLds <= 160 * 1024, "workgroups that share a CU");
    // position of 16-byte chunk ch of V row r: ch ^ turn(r)
    static __device__ __forceinline__ int turn(int r) {
        return QW == 16 ? ((r >> 1) & 3) | ((r >> 4) & 1) << 2 : ((r >> 1) & 1) << 1 | ((r >> 3) & 1) << 2;
    }
};

template <int CODE, int QW, int NW>
__global__ __launch_bounds__(64 * NW, (Few8<QW, NW>::kGroups * NW / 4)) void attention_few8(const Attention8 args, int least) {
    typedef Few8<QW, NW> L;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & (QW - 1), hh = lane / QW;
    const int kv_head = (int)(block_number() % (unsigned)args.n_kv_heads), item = (int)(block_number() / (unsigned)args.n_kv_heads);
    Work w;
    if (!find_work<QW>(args, item, least, w)) return;
    w.make_uniform();
    const Attention8 a = args_again<Attention8>();
    const int G = a.group.d;
    const int rows = min(QW, w.tokens * G - w.tile * QW);
    const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_byte_address(lds));

    // the rows of q into LDS; past the last one, that one again
    {
        const int lrow = lane >> 4, lp = lane & 15;
        for (int r0 = 4 * wave; r0 < QW; r0 += 4 * NW) {
            const int r = r0 + lrow;
            const int row = w.tile * QW + min(r, rows - 1), token = a.group.of(row);
            const u16* from = a.q + (long long)(w.begin + token) * a.q_row + (long long)(kv_head * G + row - token * G) * a.q_head;
            load_to_lds_16(from + (lp ^ (r & 15)) * 8, lds0 + L::kQ + r0 * 256);
        }
    }
    const int last_key = w.keys - 1;
    const int my_token = a.group.of(w.tile * QW + min(c, rows - 1));
    const int q_abs = w.before + my_token;                                          // the last key this lane's row sees
    const int first_token = a.group.of(w.tile * QW);
    const int first_masked = (int)max((long long)w.before + first_token + 1, 0ll) / kKT;  // tiles before it: every row sees every key
    const int* table_row = (const int*)uniform_ptr((const char*)(a.table + w.seq * a.table_row));
    const u8* k_pool = (const u8*)a.k + kv_head * a.head;
    const u8* v_pool = (const u8*)a.v + kv_head * a.head;
    const unsigned row_bytes = (unsigned)a.slot;
    const float* my_scales = (lane < 32 ? a.k_scale : a.v_scale) + kv_head * a.scale_head;  // (a lane has a key's or a value's)
    const int lrow = lane >> 3, lp = lane & 7;

    constexpr int P = L::kPlaces;
    // where tile number n (of this wave) lies: places take turns
    auto place = [&](int n) __attribute__((always_inline)) { return lds0 + wave * L::kWave + (P == 1 ? 0 : (n & 1) * L::kPlace); };
    auto fill = [&](int tile, int n, const Blocks& b, bool v_part) __attribute__((always_inline)) {
        unsigned slot = place(n) + (v_part ? kTileBytes : 0);
        asm volatile("" : "+v"(slot));  // (see attention_few)
        const unsigned dst = __builtin_amdgcn_readfirstlane(slot);
        if (!v_part) {
            const int g = (lane >> 3) & 3, block = g == 0 ? b.id[0] : g == 1 ? b.id[1] : g == 2 ? b.id[2] : b.id[3];
            const int at = (unsigned)block < (unsigned)a.n_blocks ? block : 0;
            load_to_lds_4(my_scales + at * a.scale_block + ((tile * kKT + (lane & 31)) & ((1 << a.shift) - 1)), dst + L::kScales);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // eight rows (1 KB): lane i lands at row 8j + (i >> 3), position i & 7
            const char* base = group_base(a, v_part ? v_pool : k_pool, b.id[j], tile * kKT + 8 * j);
            const int r = 8 * j + lrow;
            load_to_lds_16(base, lrow * row_bytes + (lp ^ (v_part ? L::turn(r) : (r >> 1) & 7)) * 16, dst + j * 1024);
        }
    };
    // loads of a tile, in order: scales and K (5), V (4); P tiles are on their way.  Block numbers: of this tile and the P behind it
    int tile = w.tile_lo + wave, n = 0;
    Blocks here{}, next{}, third{};
    if (tile < w.tile_hi) {
        here = blocks_of(a, table_row, tile, last_key);
        if (tile + NW < w.tile_hi) next = blocks_of(a, table_row, tile + NW, last_key);
        fill(tile, 0, here, false);
        fill(tile, 0, here, true);
        if (P == 2 && tile + NW < w.tile_hi) {
            fill(tile + NW, 1, next, false);
            fill(tile + NW, 1, next, true);
            if (tile + 2 * NW < w.tile_hi) third = blocks_of(a, table_row, tile + 2 * NW, last_key);
            asm volatile("s_waitcnt vmcnt(18)" ::: "memory");  // the rows of q have landed, the tiles are on their way
        } else {
            asm volatile("s_waitcnt vmcnt(9)" ::: "memory");
        }
    } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");

    constexpr int KS = QW == 16 ? 4 : 8;   // MFMA steps over the head's 128 features
    constexpr int NS = QW == 16 ? 8 : 16;  // scores of a tile per lane
    constexpr int DB = QW == 16 ? 8 : 4;   // output blocks of QW features
    constexpr int NR = QW == 16 ? 4 : 16;  // registers of one
    typedef float acc_t __attribute__((ext_vector_type(NR)));
    // step 2 j + s has the features 16 ch + 8 s .., ch = hh + 4 j (QW = 16) or hh + 2 j
    constexpr int kNext = QW == 16 ? 4 : 2;
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
        qf[ks] = *(const bf16x8*)(lds + L::kQ + c * 256 + (((2 * (hh + kNext * (ks >> 1)) + (ks & 1)) ^ (c & 15)) * 16));
    acc_t oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < NR; ++r) oacc[db][r] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    const unsigned k_lane = c * 128 + ((hh ^ ((c >> 1) & 7)) * 16);
    // transposing reads: lane 2 r + x of a group of 16 addresses half x of row r's chunk; rows are keys in the order of the scores
    const int quad = lane >> 4, s = lane & 15;
    const int vt_row = QW == 16 ? 4 * quad + 16 * (s >> 3) + ((s >> 1) & 3) : 4 * (quad >> 1) + 8 * (s >> 3) + ((s >> 1) & 3);
    const unsigned v_lane = kTileBytes + vt_row * 128 + (((QW == 16 ? 0 : quad & 1) ^ L::turn(vt_row)) * 16) + 8 * (s & 1);
    auto key_of = [](int r) { return (QW == 16 ? 16 : 8) * (r >> 2) + (r & 3); };  // of the lane's score r, less 4 hh
    bool special = false;  // codes that are no numbers were taken out of a tile (of this lane's pieces)

    for (; tile < w.tile_hi; tile += NW, ++n) {
        const bool more = tile + NW < w.tile_hi, further = tile + 2 * NW < w.tile_hi;
        const unsigned there = rows_there(a, here, tile, last_key);
        const unsigned my_place = place(n);
        const unsigned char* k_base = lds + (my_place - lds0);
        if (P == 2 && more) asm volatile("s_waitcnt vmcnt(13)" ::: "memory");  // the scales and the K tile have landed
        else asm volatile("s_waitcnt vmcnt(4)" ::: "memory");

        // ---- S^T = K Q^T, and both kinds of scales ----
        float sv[NS], vs[NS];
        {
            f32x4 ks[NS / 4], vx[NS / 4];
#pragma unroll
            for (int x = 0; x < NS / 4; ++x) {
                ks[x] = *(const f32x4*)(k_base + L::kScales + ((QW == 16 ? 16 : 8) * x + 4 * hh) * 4);
                vx[x] = *(const f32x4*)(k_base + L::kScales + 128 + ((QW == 16 ? 16 : 8) * x + 4 * hh) * 4);
            }
            u32x4 kc[4];
            if constexpr (QW == 16) {
#pragma unroll
                for (int f = 0; f < 4; ++f) kc[f] = *(const u32x4*)(k_base + (f >> 1) * 2048 + (k_lane ^ (64 * (f & 1))));  // key half, j
                f32x4 sacc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int half = x & 1, step = x >> 1;
                    const u32x4 k4 = kc[2 * half + (step >> 1)];
                    sacc[half] = mfma16(operand<CODE>(k4[2 * (step & 1)], k4[2 * (step & 1) + 1]), qf[step], sacc[half]);
                }
#pragma unroll
                for (int r = 0; r < NS; ++r) sv[r] = sacc[r >> 2][r & 3];
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) kc[j] = *(const u32x4*)(k_base + (k_lane ^ (32 * j)));
                f32x16 sacc;
#pragma unroll
                for (int r = 0; r < 16; ++r) sacc[r] = 0.f;
#pragma unroll
                for (int step = 0; step < 8; ++step)
                    sacc = mfma32(operand<CODE>(kc[step >> 1][2 * (step & 1)], kc[step >> 1][2 * (step & 1) + 1]), qf[step], sacc);
#pragma unroll
                for (int r = 0; r < NS; ++r) sv[r] = sacc[r];
            }
#pragma unroll
            for (int r = 0; r < NS; ++r) {
                sv[r] *= ks[r >> 2][r & 3];
                vs[r] = vx[r >> 2][r & 3];
            }
        }
        const bool refill = P == 1 ? more : further;
        if (refill) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the K tile and the scales have been read
            fill(tile + P * NW, n, P == 1 ? next : third, false);
        }

        // ---- online softmax (see attention_few) ----
        const bool masked = tile >= first_masked || there != ~0u;
        if (masked) {
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
        const bool grow = mt > m_run + 8.0f;
        const float m_new = grow ? mt : m_run;
        const float m_safe = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = grow ? __builtin_amdgcn_exp2f(m_run - m_safe) : 1.0f;
        const bool rescale = grow && m_run != -INFINITY;
        float ps = 0.f;
        u32x4 pf[NS / 8], rest[NS / 8];  // the operands of the second product
#pragma unroll
        for (int r = 0; r < NS; r += 2) {
            float x[2], hi[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[r + e], a.scale_log2e, -m_safe));
                ps += p;
                x[e] = scaled(p, vs[r + e]);
                hi[e] = __uint_as_float(__float_as_uint(x[e]) & 0xFFFF0000u);
            }
            pf[r >> 3][(r & 7) / 2] = __builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302);
            rest[r >> 3][(r & 7) / 2] = pack_bf16x2(x[0] - hi[0], x[1] - hi[1]);
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
        if (refill) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(P == 1 ? 5 : 14) : "memory");  // V has landed
        else if (P == 2 && more) asm volatile("s_waitcnt vmcnt(9)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (CODE == JUP_E4M3 && masked) {
            asm volatile("");
#pragma unroll
            for (int j = 0; j < 4; ++j)  // rows 8j .. 8j + 7
                special |= clean_piece8(lds + (my_place - lds0) + kTileBytes + j * 1024 + lane * 16, (there >> (8 * j + lrow)) & 1);
        }
#pragma unroll
        for (int f = 0; f < 8; ++f) {
            // QW = 32: feature block f / 2, key half f % 2; QW = 16: feature block f, all 32 keys
            const u32x2 codes = read_tr8(my_place + (QW == 16 ? v_lane ^ (16 * f) : (v_lane ^ (32 * (f / 2))) + (f % 2) * 2048));
            const bf16x8 v = operand<CODE>(codes[0], codes[1]);
            if constexpr (QW == 16) oacc[f] = mfma16(v, __builtin_bit_cast(bf16x8, rest[0]), mfma16(v, __builtin_bit_cast(bf16x8, pf[0]), oacc[f]));
            else oacc[f / 2] = mfma32(v, __builtin_bit_cast(bf16x8, rest[f % 2]), mfma32(v, __builtin_bit_cast(bf16x8, pf[f % 2]), oacc[f / 2]));
        }
        here = next;
        if (P == 2) next = third;
        if (refill) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the V tile has been read
            fill(tile + P * NW, n, P == 1 ? here : next, true);
            if (tile + (P + 1) * NW < w.tile_hi) (P == 1 ? next : third) = blocks_of(a, table_row, tile + (P + 1) * NW, last_key);
        }
    }

    if (CODE == JUP_E4M3 && __any(special)) {  // once in a blue moon
        for (tile = w.tile_lo + wave; tile < w.tile_hi; tile += NW) {
            const Blocks b = blocks_of(a, table_row, tile, last_key);
            const unsigned there = rows_there(a, b, tile, last_key);
            if (tile < first_masked && there == ~0u) continue;
            for (int k = 0; k < kKT; ++k) {
                if (!((there >> k) & 1)) continue;
                const char* row = group_base(a, v_pool, table_row[(tile * kKT + k) >> a.shift], tile * kKT + (k & ~7)) + (k & 7) * row_bytes;
                if (!row_not_finite<CODE>(row)) continue;
#pragma unroll
                for (int x = 0; x < (QW == 16 ? 8 : 16); ++x) {
                    const int db = QW == 16 ? x : x >> 2, r = QW == 16 ? 0 : 4 * (x & 3);
                    add_not_finite<CODE>(oacc[db], r, row, (QW == 16 ? 16 * x : 8 * x) + 4 * hh, tile * kKT + k <= q_abs);
                }
            }
        }
    }

    // ---- the waves' sums put together ----
    merge_few<QW, NW, L::kStat>(w, kv_head, rows, c, hh, m_run, l_run, oacc, lds);
}

// Codes become bf16 values once per workgroup of attention_many and once per wave of attention_few8, but there the waves do not meet: tiles of 32 rows are
// faster up to three rounds of them.  In µs, attention_few8 and attention_many, int8: 300 tokens behind 1536 on 32 heads 41 / 51, 512 45 / 45 (e4m3 39 / 45),
// 768 70 / 81 (62 / 81), prompts of 800 26 / 29, of 1024 34 / 36, of 1200 on 40 heads (1520 tiles) 54 / 50 (lost by the rule), of 2048 (2600 tiles) 120 / 95.
constexpr int kFewTiles8 = 1536;

template <int CODE>
struct Kernels8 {
    static constexpr int kTiles = kFewTiles8;
    template <int QW, int NW> static auto few() { return attention_few8<CODE, QW, NW>; }
    template <int QW, int NW> static constexpr int few_lds() { return Few8<QW, NW>::kLds; }
    template <int QW, int NW> static constexpr int few_pieces() { return NW == 8 ? kWidePieces : 256 * Few8<QW, NW>::kGroups; }
    template <int KP, int NT, int SUB> static auto many() { return attention_many<CODE, 8, KP, NT, SUB, 2>; }
    template <int KP, int NT, int SUB> static constexpr int many_lds() { return Many<8, KP, NT, SUB, true>::kLds; }
};

}  // namespace

hipError_t launch_paged_attention8(const jup_paged_pool_t& pool, const jup_paged_scales_t& scales, const jup_paged_attention_t& c, hipStream_t s, int tiled) {
    Attention8 a{};
    set_call(a, pool, c, tiled);
    a.k_scale = scales.k; a.v_scale = scales.v;
    a.scale_block = scales.block_stride; a.scale_head = scales.head_stride;
    return pool.dtype == JUP_I8 ? launch_tiles<Kernels8<JUP_I8>>(a, c, s) : launch_tiles<Kernels8<JUP_E4M3>>(a, c, s);
}

}  // namespace jup
