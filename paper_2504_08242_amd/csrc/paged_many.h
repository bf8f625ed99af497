// Attention over a paged cache in tiles of many rows (paged_attention.hip, paged_attention8.hip): the kernel that both kinds of pools share, JUP_BF16
// values that are fetched straight into LDS, or codes that become such values on the way.
#pragma once

#include "paged_work.h"

namespace jup {
namespace {

constexpr int kValueTile = kKT * 256;  // a K or V tile in LDS: 32 rows of 128 bf16

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
template <int NW, int KP, int NT, int SUB, bool SCALES>
struct Many {
    static constexpr int kWaves = NW;
    static constexpr int kRows = 32 * NW / KP;
    static constexpr int kSubTiles = KP * NT;                // a wave works through NT tiles at a time, SUB times between two meetings
    static constexpr int kStepTiles = SUB * kSubTiles;
    static constexpr int kStep = kStepTiles * kKT;           // keys of a step
    static constexpr int kHalf = kStepTiles * kValueTile;    // K tiles, then V tiles
    static constexpr int kGroups = kStepTiles * 4 / kWaves;  // groups of eight rows that a wave fetches per step: wave, wave + NW
    static_assert(kGroups * kWaves == kStepTiles * 4);
    static constexpr int kRowBytes = 132 * 4;                // a row of a part's sums
    static constexpr int kSteps = 2 * 2 * kHalf, kSums = 32 * NW * kRowBytes, kQ = 32 * NW * 256;
    static constexpr int kThere = (kSteps > kSums ? kSteps > kQ ? kSteps : kQ : kSums);  // [2][kStepTiles * 4] bytes: which rows of a step's groups are keys
    static constexpr int kFlag = kThere + 64;
    static constexpr int kStat = kFlag + 64;                 // [2][waves][32] maxima and sums
    static constexpr int kScales = kStat + (KP > 1 ? 2 * 32 * NW * 4 : 0);  // [2][keys of a step] K's, then V's (pools in 8 bits)
    static constexpr int kLds = kScales + (SCALES ? 2 * 2 * kStep * 4 : 0);
    // queries go through the second step's place, the first step is fetched beside them
    static constexpr int kQAt = kThere - kQ;
    static_assert(kLds <= 160 * 1024 && 2 * kStepTiles * 4 <= 64 && kQAt >= 2 * kHalf);
};

template <int CODE, int NW, int KP, int NT, int SUB, int OCC>
__global__ __launch_bounds__(64 * NW, OCC) void attention_many(const ArgsOf<CODE> args, int least) {
    constexpr bool kCodes = CODE != JUP_BF16;
    typedef Many<NW, KP, NT, SUB, kCodes> L;
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
    const ArgsOf<CODE> a = args_again<ArgsOf<CODE>>();
    const int G = a.group.d;
    const int rows = min(kRows, w.tokens * G - w.tile * kRows);
    const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_byte_address(lds));
    const int lrow = lane >> 4, lp = lane & 15;

    // this wave's eight rows of a step: group `wave` (and wave + 8)
    const int last_key = w.keys - 1, first_key = w.tile_lo * kKT;
    const int n = (w.tile_hi - w.tile_lo + L::kStepTiles - 1) / L::kStepTiles;
    const int* table_row = (const int*)uniform_ptr((const char*)(a.table + w.seq * a.table_row));
    typedef const __attribute__((address_space(4))) int* scalar;
    const auto* k_pool = pool_of<CODE>(a.k) + kv_head * a.head;
    const auto* v_pool = pool_of<CODE>(a.v) + kv_head * a.head;
    // keys of this piece: up to the last key, or where the next piece begins
    const int end_key = min(last_key + 1, w.tile_hi * kKT);
    unsigned k_off[2], v_off[2];  // of the pieces of a row that a lane fetches
    if constexpr (!kCodes) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const unsigned row = (unsigned)(a.slot * 2) * (4 * j + lrow);
            k_off[j] = row + (lp ^ ((8 * wave + 4 * j + lrow) & 15)) * 16;
            v_off[j] = row + ((((lp >> 2) ^ lrow) << 2) | (lp & 3)) * 16;
        }
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
    // Sub-steps (NT tiles per part) before this one: every row of the workgroup sees all their keys.
    constexpr int kSub = L::kSubTiles * kKT;
    const int open = __builtin_amdgcn_readfirstlane((int)min(max(max((long long)w.before + a.group.of(w.tile * kRows) + 1, 0ll) - first_key, 0ll) / kSub, (long long)n * SUB));
    unsigned hole = 0;  // bit: in that slot, some of this wave's rows are no keys
    auto note_keys = [&](int i, int g, const Ids& ids, int mine) __attribute__((always_inline)) {
        const int left = end_key - mine;
        const unsigned there = (unsigned)ids.id[g] >= (unsigned)a.n_blocks || left <= 0 ? 0u : left >= 8 ? 0xFFu : (1u << left) - 1;
        hole |= there == 0xFFu ? 0u : 1u << (i & 1);
        if (lane == 0) lds[L::kThere + (i & 1) * L::kStepTiles * 4 + NW * g + wave] = (unsigned char)there;
        return there;
    };
    // K of step i, or V, and which rows are keys
    auto fill = [&](int i, const Ids& ids, bool v_part) __attribute__((always_inline)) {
        if (v_part) hole &= ~(1u << (i & 1));
#pragma unroll
        for (int g = 0; g < L::kGroups; ++g) {
            const int mine = first_key + i * kStep + 8 * NW * g + 8 * wave, key = min(mine, last_key & ~7);  // (groups behind the last key repeat its own)
            unsigned slot = lds0 + (unsigned)(i & 1) * 2 * kHalf + (v_part ? kHalf : 0) + (NW * g + wave) * 2048;
            asm volatile("" : "+v"(slot));  // (from a vector register on purpose: the compiler keeps it in one, and else hands that to the loads)
            const unsigned dst = __builtin_amdgcn_readfirstlane(slot);
            const char* base = group_base(a, v_part ? v_pool : k_pool, ids.id[g], key);
#pragma unroll
            for (int j = 0; j < 2; ++j) load_to_lds_16(base, v_part ? v_off[j] : k_off[j], dst + j * 1024);
            if (!v_part) continue;
            note_keys(i, g, ids, mine);
        }
    };
    // Codes are fetched into registers, half a step ahead of their use, and go into LDS as the bf16 values that they are: once for all waves, where
    // a conversion behind LDS would be made by every wave that reads them.  (Four prompts of 700 to 4100 tokens, e4m3, take 338 µs, bf16 values 292.  What
    // comes on top, measured one at a time at 371 µs, when some registers were still spilled: conversions and stores to LDS 46, scales 33, loads 28.
    // Values put behind the products take 349, both kinds fetched a whole step ahead 354, and there int8 runs out of registers.)
    // A lane has 16 codes of a row of each of its wave's groups; of the scales lanes 0 to 7 and 16 to 23 have one of a key in the first and second
    // group, the eight behind each one of a value.
    u32x4 pending[L::kGroups];
    float pending_scale = 0.f;
    // (What a lane makes of its number is made again each time: there are no registers to keep it in, and spilled ones cost 15 µs.  Two of eight lanes
    // store to the same banks; without that, with 8 codes of either half of a row per lane, it takes as long, int8 2 % longer.)
    auto my_lane = [&]() __attribute__((always_inline)) {
        int x = lane;
        asm volatile("" : "+v"(x));
        return x;
    };
    bool special = false;  // values that are no numbers were taken out
    auto fetch = [&](int i, const Ids& ids, bool v_part) __attribute__((always_inline)) {
        const int me = my_lane();
#pragma unroll
        for (int g = 0; g < L::kGroups; ++g) {
            const int key = min(first_key + i * kStep + 8 * NW * g + 8 * wave, last_key & ~7);  // (groups behind the last key repeat its own)
            const char* base = group_base(a, v_part ? v_pool : k_pool, ids.id[g], key);
            pending[g] = load_at<u32x4>(base, (me >> 3) * (unsigned)a.slot + (me & 7) * 16);
        }
        if constexpr (kCodes) {
            if (!v_part) {
                const int g = (me >> 4) & 1, block = g == 0 ? ids.id[0] : ids.id[L::kGroups - 1];
                const int key = min(first_key + i * kStep + 8 * NW * g + 8 * wave, last_key & ~7);
                const long long at = (unsigned)block < (unsigned)a.n_blocks ? block : 0;
                const float* scales = (me & 8 ? a.v_scale : a.k_scale) + kv_head * a.scale_head;
                pending_scale = scales[at * a.scale_block + (key & ((1 << a.shift) - 1)) + (me & 7)];
            }
        }
    };
    auto put = [&](int i, const Ids& ids, bool v_part) __attribute__((always_inline)) {
        if constexpr (kCodes) {
            const int me = my_lane();
            if (v_part) hole &= ~(1u << (i & 1));
            else if (me < 16 * L::kGroups)
                *(float*)(lds + L::kScales + (i & 1) * 2 * kStep * 4 + (me & 8 ? kStep * 4 : 0) + (8 * NW * (me >> 4) + 8 * wave + (me & 7)) * 4) =
                    pending_scale;
#pragma unroll
            for (int g = 0; g < L::kGroups; ++g) {
                const int group = NW * g + wave, r = 8 * (group & 3) + (me >> 3);
                const u32x4 codes = pending[g];
                if (v_part) note_keys(i, g, ids, first_key + i * kStep + 8 * group);
                unsigned char* at = lds + (i & 1) * 2 * kHalf + (v_part ? kHalf : 0) + (group >> 2) * kValueTile + r * 256;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int ch = 2 * (me & 7) + x;
                    *(bf16x8*)(at + (v_part ? (((ch >> 2) ^ (r & 3)) << 2) | (ch & 3) : ch ^ (r & 15)) * 16) = operand<CODE>(codes[2 * x], codes[2 * x + 1]);
                }
            }
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
        if constexpr (kCodes) {  // what was fetched half a step ago goes into its place, the other half is fetched
            if (k_part) {
                put(i, ids, false);
                fetch(i, ids, true);
            }
            if (v_part) {
                const Ids next = ids_of(i + 1);
                put(i, ids, true);
                ids = next;
                if (i + 1 < n) fetch(i + 1, ids, false);
            }
            return;
        }
        if (k_part) fill(i, ids, false);
        if (v_part) {
            const Ids next = ids_of(i + 1);
            fill(i, ids, true);
            ids = next;
        }
    };
    if (kCodes && n > 0) fetch(0, ids, false);
    fill_next(0, true, true);

    // Behind the wait for this wave's rows of step i: rows that are no keys become 0, and where some row sees some key and another
    // does not, values that are no numbers do.
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
    if (n > 0 && !kCodes) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * L::kGroups) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) qf[ks] = *(const bf16x8*)(q_lds + (k_lane ^ (32 * ks)));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();  // every wave has its queries: the second step may go there
    asm volatile("" ::: "memory");

    for (int i = 0; i < n; ++i) {
        // step i is there for all, and step i - 1 has been read by all
        if constexpr (kCodes) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if constexpr (CODE != JUP_I8) clean(i);  // (the codes of int8 are numbers, and their scales do not get here)
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
        const unsigned char* k_base = lds + (i & 1) * 2 * kHalf + first_tile * kValueTile;
        const unsigned v_slot = (unsigned)(i & 1) * 2 * kHalf + first_tile * kValueTile;
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
            for (int ks = 0; ks < 8; ++ks) kf[t][ks] = *(const bf16x8*)(k_base + t * kValueTile + (k_lane ^ (32 * ks)));
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
                const unsigned at = v_slot + t * kValueTile + v_lane[f / 2] + (f % 2) * 16 * 256;
                const u32x2 lo = read_tr(at), hi = read_tr(at + 8 * 256);
                vf[f] = (u32x4){lo[0], lo[1], hi[0], hi[1]};
            }
        };
        read_v(0);

        fill_next(i + 1, u == 0, false);

        // ---- online softmax (see attention_few) ----
        float sv[16 * NT];
        const unsigned char* scales = lds + L::kScales + (i & 1) * 2 * kStep * 4 + (first_tile * kKT + 4 * hh) * 4;  // (pools in 8 bits)
        if constexpr (kCodes) {
#pragma unroll
            for (int x = 0; x < 4 * NT; ++x) {  // keys 8 x + 4 hh .. + 3
                const f32x4 ks = *(const f32x4*)(scales + x * 32);
#pragma unroll
                for (int e = 0; e < 4; ++e) sv[4 * x + e] = s[x >> 2][4 * (x & 3) + e] * ks[e];
            }
        } else {
#pragma unroll
            for (int r = 0; r < 16 * NT; ++r) sv[r] = s[r >> 4][r & 15];
        }
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
        if constexpr (kCodes) {
#pragma unroll
            for (int y = 0; y < 4 * NT; ++y) {
                const f32x4 vx = *(const f32x4*)(scales + kStep * 4 + y * 32);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[4 * y + e], a.scale_log2e, -m_safe));
                    ps += x;
                    p[y >> 1][4 * (y & 1) + e] = (__bf16)scaled(x, vx[e]);
                }
            }
        } else {
#pragma unroll
            for (int r = 0; r < 16 * NT; ++r) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[r], a.scale_log2e, -m_safe));
                ps += x;
                p[r >> 3][r & 7] = (__bf16)x;
            }
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
    const Attention e = args_again<Attention>();
    __syncthreads();  // every wave is done with the steps
    if (lds[L::kFlag]) {  // once in a blue moon: what clean() took out
        for (int tile = w.tile_lo + L::kSubTiles * open; tile < min(w.tile_hi, w.tile_lo + L::kSubTiles * mine); ++tile) {
            if ((tile - w.tile_lo) / NT % KP != part) continue;
            const Blocks ids = blocks_of(a, table_row, tile, last_key);
            const unsigned there = rows_there(a, ids, tile, last_key);
            for (int k = 0; k < kKT; ++k) {
                if (!((there >> k) & 1)) continue;
                const char* row = group_base(a, v_pool, table_row[(tile * kKT + k) >> a.shift], tile * kKT + (k & ~7)) + (k & 7) * (unsigned)(a.slot * (kCodes ? 1 : 2));
                if (!row_not_finite<CODE>(row)) continue;
#pragma unroll
                for (int x = 0; x < 16; ++x) add_not_finite<CODE>(o[x >> 2], 4 * (x & 3), row, 8 * x + 4 * hh, tile * kKT + k <= sees_to);
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

}  // namespace
}  // namespace jup
