// The end of a step of a beam search (include/jupiter_paged.h).
//
// score(b, j) = scores[b] + x_bj - L_b with L_b = m_b + log sum_j exp(x_bj - m_b).  Within a row the order of the scores is that of
// the logits, so one pass over a row leaves its n_keep largest logits and (m, sum); the workgroup of a request that is done last puts the rows'
// together.  Keys, larger is better: a logit's bits in an order that integers have, then the lower token.
#include "paged.h"

namespace jup {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMost = JUP_BEAM_MOST;
constexpr unsigned kTokens = (1u << 30) - 1;
static_assert(kMost == 64, "six bits of a candidate are its beam");
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ u64 key_of(float x, int token) {  // x finite, -0 as 0
    const unsigned bits = __float_as_uint(x + 0.0f);
    return (u64)(bits ^ ((bits >> 31) ? 0xFFFFFFFFu : 0x80000000u)) << 32 | (unsigned)~token;
}
__device__ __forceinline__ float value_of(u64 key) {
    const unsigned bits = (unsigned)(key >> 32);
    return __uint_as_float(bits ^ ((bits >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}

// What a workgroup leaves of a slice of a row: the statistics and n_keep keys, best first, 0 where there are fewer.
constexpr int kLeft = 2 + kMost;
__device__ __forceinline__ void leave(u64* at, u64 x) { store_coherent2((float*)at, __uint_as_float((unsigned)x), __uint_as_float((unsigned)(x >> 32))); }
__device__ __forceinline__ u64 left(const u64* at) {
    const float2 x = load_coherent2((const float*)at);
    return (u64)__float_as_uint(x.y) << 32 | __float_as_uint(x.x);
}

// A wave's best keys so far.  Candidates are collected as they come; where they might not fit any more, the n_keep best stay (their ranks are
// counted, all lanes at once) and the last of these is the limit for those that follow.  Indices only rise: what equals the limit is behind it.
constexpr int kStep = 64 * 8;  // logits of a wave at a time, at most
struct Best {
    u64 found[kMost + kMost / 2 + kStep + 8], kept[kMost];
};
// Candidates are put in order when there are so many: the limit rises, and fewer logits get so far.  (When there are 64, whatever n_keep is: 65 µs in
// place of 52 for 512 rows of 131072 with eight kept, as some logit of nearly every 512 was above a limit that old.)
__device__ __forceinline__ int enough(int keep) { return keep + max(8, keep / 2); }
__device__ __forceinline__ void in_order() {  // LDS accesses of a wave are in order; so are the compiler's
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ int lanes_below(u64 lanes) {  // how many of them are before this one
    return __builtin_amdgcn_mbcnt_hi((unsigned)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)lanes, 0));
}
// How many of n keys are above one; eight at a time, the places behind the last hold 0.
__device__ __forceinline__ int above(const u64* keys, int n, u64 key) {
    typedef u64 u64x2 __attribute__((ext_vector_type(2)));
    int rank = 0;
    for (int j = 0; j < n; j += 8) {
        u64x2 x[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) x[y] = *(const u64x2*)(keys + j + 2 * y);
#pragma unroll
        for (int y = 0; y < 4; ++y) rank += (x[y][0] > key) + (x[y][1] > key);
    }
    return rank;
}
__device__ __forceinline__ int keep_best(Best& b, int n, int keep, float& limit) {
    const int lane = threadIdx.x & 63;
    if (lane < 8) b.found[n + lane] = 0;
    in_order();
    for (int i = lane; i < n; i += 64) {
        const u64 mine = b.found[i];
        const int rank = above(b.found, n, mine);
        if (rank < keep) b.kept[rank] = mine;
    }
    in_order();
    n = min(n, keep);
    if (lane < n) b.found[lane] = b.kept[lane];
    in_order();
    if (n == keep) limit = fmaxf(limit, __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(value_of(b.found[n - 1])))));
    return n;
}

// The largest of a wave; the least of the largest of its groups of `group` lanes (a power of two).  Every lane gets the same, and the compiler knows.
__device__ __forceinline__ float pair_up(float x, int by, bool largest) {
    float y;
    if (by == 1) y = dpp_move<0xB1>(x);
    else if (by == 2) y = dpp_move<0x4E>(x);
    else if (by == 4) y = dpp_move<0x141>(x);  // (the four lanes that are alike, mirrored)
    else if (by == 8) y = dpp_move<0x140>(x);
    else if (by == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return largest ? fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])) : fminf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return largest ? fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])) : fminf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return largest ? fmaxf(x, y) : fminf(x, y);
}
__device__ __forceinline__ float least_of_groups(float x, int group) {
#pragma unroll
    for (int by = 1; by < 64; by *= 2) x = pair_up(x, by, by < group);
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}
__device__ __forceinline__ float wave_max(float x) { return least_of_groups(x, 64); }

struct __attribute__((aligned(16))) Shared {
    Best best[kWaves];
    int n[kWaves];
    float m[kWaves];
    double sum[kWaves];
    int flag;
};

// The last one done has all rows' statistics and keys.  A candidate, larger is better, 128 bits: its score as an integer of the same order, less its last
// four bits (2^-48 of it), then the lower beam (6 bits), the larger logit (32) and the lower token (30).  Scores of a beam are its logits' up to rounding, so
// this is the order of its keys however far from its logits the score is: the order of the lists, and one for all of them.
struct __attribute__((aligned(16))) Candidate {
    u64 score, place;
    __device__ __forceinline__ bool operator>(const Candidate& o) const { return score > o.score || (score == o.score && place > o.place); }
    __device__ __forceinline__ int beam() const { return (kMost - 1) ^ (int)((score & 15) << 2 | place >> 62); }
    __device__ __forceinline__ int token() const { return (int)(~(unsigned)place & kTokens); }
};
__device__ __forceinline__ Candidate candidate_of(double score, int beam, u64 key) {
    const u64 bits = __builtin_bit_cast(u64, score + 0.0), order = bits ^ ((bits >> 63) ? ~0ull : 1ull << 63);
    const u64 back = (u64)((kMost - 1) ^ beam);
    return {(order & ~15ull) | back >> 2, back << 62 | (key >> 32) << 30 | (key & kTokens)};
}
__device__ __forceinline__ double score_of(u64 order) {  // (the last bits are 0 again: an fp32 score comes back as it was)
    return __builtin_bit_cast(double, (order >> 63) ? (order & ~15ull) ^ 1ull << 63 : ~(order | 15ull));
}

constexpr int kMostLists = 1024;  // slices of a request's rows
constexpr int kEach = 4;          // candidates of a thread, where they are looked at all at once
struct Merge {
    union {
        Candidate best[kWaves][kMost + 64];
        struct {
            u64 all[kThreads];
            Candidate chosen[kThreads], ordered[kThreads];
            int counts[kEach][kWaves];
            float bound[kWaves];
        };
    };
    double part[kMostLists];
    float m[kMostLists], top[kMost];
    double log_sum[kMost], score[kMost];
    int ended[kMost], n[kWaves], disorder;
};

union Lds {
    Shared s;
    Merge m;
};

template <class T>
struct Logits;
template <>
struct Logits<float> {
    static constexpr int V = 4;  // of a 16-byte load
    typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ float value(float x) { return x; }
};
template <>
struct Logits<u16> {
    static constexpr int V = 8;
    typedef u16 vec __attribute__((ext_vector_type(8), aligned(2)));
    static __device__ __forceinline__ float value(u16 x) { return bf2f(x); }
};

// `slices` workgroups per row, each with `length` logits of it, U pieces of 16 bytes per thread at a time (the next ones are on their way meanwhile; with
// two in place of four 64 rows of 32000 in bf16 take 17 µs in place of 14, 512 of 131072 48 in place of 47).
// Four rows of 32000 fp32 logits take 12 µs: 8 up to the arrival, 4 for the last workgroup, trips to memory most of it (with slices of 2048 logits
// 14, as twice as many lists are put together).  512 rows of 131072 in bf16, of which a fifth are not read, 107 MB, take 45: reading alone takes 28 (3.8
// TB/s, as workgroups of rows that are not read leave holes), exponentials 5 of the others and candidates 10 (without either, less than the sum).
template <class T, int U>
__global__ __launch_bounds__(kThreads) void select(const jup_beam_select_t a, int slices, int length, int* count, u64* scratch) {
    typedef Logits<T> L;
    constexpr int V = L::V;
    typedef typename L::vec vec;
    __shared__ Lds lds;
    Shared& s = lds.s;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = (int)(block_number() / (unsigned)slices), slice = (int)(block_number() - (unsigned)row * slices);
    if (row >= a.n_seqs * a.n_beams) return;
    const int request = row / a.n_beams, keep = a.n_keep;
    u64* mine = scratch + ((long long)row * slices + slice) * kLeft;
    const float so_far = a.scores[row];
    const bool reads = fabsf(so_far) < INFINITY && !(a.ended && a.ended[row]);
    // statistics: a lane's sum of exp(x - m); m is the wave's, within 1 of the largest so far
    float m = -INFINITY, limit = -INFINITY;
    double sum = 0.0;
    int n = 0;  // candidates of the wave
    if (reads) {
        const T* x = (const T*)a.logits + row * a.row_stride;
        const int end = min((slice + 1) * length, a.vocab);
        constexpr int kAll = kThreads * V * U;
        auto load = [&](int j0, vec* raw) __attribute__((always_inline)) {
            // (no lane has branches of its own: with them the loads in flight cannot be told apart, and each is waited for at once)
            if (j0 + kAll <= end) {
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = *(const vec*)(x + j0 + (u * kThreads + tid) * V);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const int j = j0 + (u * kThreads + tid) * V + e;
                        const T value = x[min(j, end - 1)];
                        raw[u][e] = j < end ? value : (T)(sizeof(T) == 2 ? 0xFF80 : -INFINITY);
                    }
                }
            }
        };
        vec raw[U], next[U];
        load(slice * length, raw);
        for (int j0 = slice * length; j0 < end; j0 += kAll) {
            if (j0 + kAll < end) load(j0 + kAll, next);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float v[V], top;
                auto look = [&](bool clean) __attribute__((always_inline)) {  // clean: NaN and +infinity become -infinity
                    top = -INFINITY;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        v[e] = L::value(raw[u][e]);
                        if (clean) v[e] = v[e] < INFINITY ? v[e] : -INFINITY;
                        top = fmaxf(top, v[e]);
                    }
                };
                auto add = [&]() __attribute__((always_inline)) {
                    float part[2] = {0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < V; ++e) part[e & 1] += __builtin_amdgcn_exp2f((v[e] - m) * kLog2e);
                    return part[0] + part[1];
                };
                look(false);
                bool cleaned = false;
                if (__any(!(top <= m + 1.0f))) {  // the first time, and a few times more (or an infinity, or nothing but NaN)
                    look(true);
                    cleaned = true;
                    const float most = wave_max(top);
                    if (most > m + 1.0f) {
                        if (m > -INFINITY) sum *= exp((double)m - (double)most);
                        m = most;
                    }
                }
                if (m > -INFINITY) {
                    float part = add();
                    if (__any(!(part < INFINITY))) {  // NaN among numbers
                        look(true);
                        cleaned = true;
                        part = add();
                    }
                    sum += part;
                }
                const bool first = limit == -INFINITY;
                if (first && n == 0) {
                    if (!cleaned) look(true);
                    // Lanes in as many groups as are kept, or more: no group's best is below the least of the groups' bests, so that
                    // many logits are not.
                    int group = 64;  // lanes of one
                    while (group > 1 && 64 / group < keep) group >>= 1;
                    limit = least_of_groups(top, group);
                }
                // (in the round that makes the limit what equals it counts)
                if (!__any(first ? top >= limit && top > -INFINITY : top > limit)) continue;
                const int j = j0 + (u * kThreads + tid) * V;
                int mine_counts = 0, at = 0;
                if (!first) {
#pragma unroll
                    for (int e = V - 1; e >= 0; --e) {
                        mine_counts += v[e] > limit;
                        at = v[e] > limit ? e : at;
                    }
                }
                if (!first && !__any(mine_counts > 1)) {  // mostly: one of a lane, its largest
                    const u64 who = __ballot(mine_counts > 0);
                    if (mine_counts) s.best[wave].found[n + lanes_below(who)] = key_of(top, j + at);
                    n += __popcll(who);
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const bool counts = first ? v[e] >= limit && v[e] > -INFINITY : v[e] > limit;
                        const u64 who = __ballot(counts);
                        if (counts) s.best[wave].found[n + lanes_below(who)] = key_of(v[e], j + e);
                        n += __popcll(who);
                    }
                }
                if (n > enough(keep)) n = keep_best(s.best[wave], n, keep, limit);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = next[u];
        }
    }
    if (n > 64) n = keep_best(s.best[wave], n, keep, limit);
    if (lane < 8) s.best[wave].found[n + lane] = 0;
#pragma unroll
    for (int by = 32; by > 0; by >>= 1) sum += __shfl_xor(sum, by, 64);
    if (lane == 0) {
        s.n[wave] = n;
        s.m[wave] = m;
        s.sum[wave] = sum;
    }
    __syncthreads();
    // the workgroup's: a thread has a key and counts those above it
    {
        const u64 key = lane < n ? s.best[wave].found[lane] : 0;
        int rank = 0, all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            rank += above(s.best[w].found, s.n[w], key);
            all += s.n[w];
        }
        if (key && rank < keep) leave(mine + 2 + rank, key);
        if (tid >= all && tid < keep) leave(mine + 2 + tid, 0);
    }
    if (wave == 0) {
        float m_all = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m_all = fmaxf(m_all, s.m[w]);
        double total = lane < kWaves && s.m[lane & (kWaves - 1)] > -INFINITY ? s.sum[lane] * exp((double)s.m[lane] - (double)m_all) : 0.0;
#pragma unroll
        for (int by = kWaves / 2; by > 0; by >>= 1) total += __shfl_xor(total, by, 64);
        if (lane == 0) {
            leave(mine, __float_as_uint(m_all));
            leave(mine + 1, __builtin_bit_cast(u64, total));
        }
    }
    wait_stores_performed();
    __syncthreads();
    if (tid == 0) {
        const int before = arrive_coherent(count + request);
        s.flag = before == a.n_beams * slices - 1;
        if (s.flag) count[request] = 0;  // ready for the next launch
    }
    __syncthreads();
    if (!s.flag) return;
    __syncthreads();  // (the flag's place is the merge's)

    // The last one done.  Its loads come from beyond L2, a microsecond away: as many as there are at once.
    Merge& g = lds.m;
    const int row0 = request * a.n_beams, lists = a.n_beams * slices, candidates = lists * keep;
    const u64* from = scratch + (long long)row0 * slices * kLeft;
    bool few = candidates <= kThreads * kEach;
    u64 my_keys[kEach];
    if (few) {
#pragma unroll
        for (int y = 0; y < kEach; ++y) {
            const int c = y * kThreads + tid;
            my_keys[y] = c < candidates ? left(from + (long long)(c / keep) * kLeft + 2 + c % keep) : 0;
        }
    }
    for (int t = tid; t < lists; t += kThreads) {
        const u64 m_bits = left(from + (long long)t * kLeft), sum_bits = left(from + (long long)t * kLeft + 1);
        g.m[t] = __uint_as_float((unsigned)m_bits);
        g.part[t] = __builtin_bit_cast(double, sum_bits);
    }
    if (tid < a.n_beams) {
        const float score = a.scores[row0 + tid];
        g.score[tid] = score;
        g.ended[tid] = !(fabsf(score) < INFINITY) ? -1 : a.ended && a.ended[row0 + tid] ? 1 : 0;  // -1: no candidates
    }
    __syncthreads();
    // (a list's sum as a multiple of exp of its beam's largest m, then a beam's sum in the order of its slices)
    for (int t = tid; t < lists; t += kThreads) {
        const int first = t / slices * slices;
        float top = -INFINITY;
#pragma unroll 4
        for (int x = 0; x < slices; ++x) top = fmaxf(top, g.m[first + x]);
        if (t == first) g.top[t / slices] = top;
        g.part[t] = g.m[t] > -INFINITY ? g.part[t] * exp((double)g.m[t] - (double)top) : 0.0;
    }
    __syncthreads();
    if (tid < a.n_beams) {
        double total = 0.0;
#pragma unroll 4
        for (int x = 0; x < slices; ++x) total += g.part[tid * slices + x];
        g.log_sum[tid] = (double)g.top[tid] + log(total);
    }
    __syncthreads();
    auto candidate = [&](int at, int k, u64 key) -> Candidate {  // entry k of list `at`
        const int beam = at / slices;
        if (g.ended[beam] != 0) return g.ended[beam] > 0 && at == beam * slices && k == 0 ? candidate_of(g.score[beam], beam, key_of(0.f, a.end_token)) : Candidate{0, 0};
        return key ? candidate_of(g.score[beam] + ((double)value_of(key) - g.log_sum[beam]), beam, key) : Candidate{0, 0};
    };
    Candidate best{0, 0};  // this thread's, and how many are better
    int rank = 0, found = 0;
    // One number for a candidate, in the order of the scores; those that are alike to 2^-44 of them are in the order of the lists.
    auto number = [](const Candidate& c, int place) { return c.score ? (c.score & ~255ull) | (unsigned)(255 - place) : 0ull; };
    if (tid == 0) g.disorder = 0;
    if (candidates <= kThreads) {  // one of a thread
        if (tid < candidates) best = candidate(tid / keep, tid % keep, my_keys[0]);
        const u64 there = __ballot(best.score != 0);
        g.all[tid] = number(best, tid);
        if (lane == 0) g.n[wave] = __popcll(there);
        __syncthreads();
        rank = above(g.all, candidates, g.all[tid]);  // (the places behind the last hold 0)
#pragma unroll
        for (int w = 0; w < kWaves; ++w) found += g.n[w];
    } else if (few) {
        // What may be among the best, n_keep at least: as of logits, none below the least of a wave's groups' bests is.
        Candidate mine[kEach];
        float value[kEach], top = -INFINITY;
#pragma unroll
        for (int y = 0; y < kEach; ++y) {
            const int c = y * kThreads + tid;
            mine[y] = c < candidates ? candidate(c / keep, c % keep, my_keys[y]) : Candidate{0, 0};
            value[y] = mine[y].score ? (float)score_of(mine[y].score) : -INFINITY;
            top = fmaxf(top, value[y]);
        }
        int group = 64;
        while (group > 1 && 64 / group < keep) group >>= 1;
        const float bound = least_of_groups(top, group);
        if (lane == 0) g.bound[wave] = bound;
        __syncthreads();
        top = g.bound[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, g.bound[w]);
        u64 who[kEach];
#pragma unroll
        for (int y = 0; y < kEach; ++y) {
            who[y] = __ballot(mine[y].score != 0 && value[y] >= top);
            if (lane == 0) g.counts[y][wave] = __popcll(who[y]);
        }
        __syncthreads();
        int at[kEach];
#pragma unroll
        for (int y = 0; y < kEach; ++y)
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                if (w == wave) at[y] = found + lanes_below(who[y]);
                found += g.counts[y][w];
            }
        few = found <= kThreads;  // (else as many are alike)
        if (few) {
            g.all[tid] = 0;
            __syncthreads();
#pragma unroll
            for (int y = 0; y < kEach; ++y)
                if ((who[y] >> lane) & 1) {
                    g.all[at[y]] = number(mine[y], at[y]);
                    g.chosen[at[y]] = mine[y];
                }
            __syncthreads();
            if (tid < found) {
                best = g.chosen[tid];
                rank = above(g.all, found, g.all[tid]);
            }
        } else {
            found = 0;
            __syncthreads();
        }
    }
    if (few) {
        // The order of the lists is not that of a beam's logits where it has several: each is compared with the next one, and if any two are the wrong way
        // round, all with all.  (That at once, in place of numbers: one request of 131072 tokens, 16 kept, 24.2 µs in place of 18.6.)
        if (best.score) g.ordered[rank] = best;
        __syncthreads();
        if (__any(tid + 1 < found && g.ordered[tid + 1] > g.ordered[tid]) && lane == 0) g.disorder = 1;
        __syncthreads();
        if (g.disorder && best.score) {
            rank = 0;
#pragma unroll 4
            for (int j = 0; j < found; ++j) rank += g.ordered[j] > best;
        }
    } else {
        // Lists are best first: a wave goes through its lists' first entries, then the second ones, and is done where none of a round is better than
        // the last of what it keeps.
        int held = 0;  // of this wave's list, best first
        Candidate* list = g.best[wave];
        for (int k0 = 0, more = 1; k0 < keep && more; ++k0) {
            more = 0;
            for (int at0 = wave * 64; at0 < lists; at0 += kThreads) {
                const int at = at0 + lane;
                const Candidate c = at < lists ? candidate(at, k0, left(from + (long long)at * kLeft + 2 + k0)) : Candidate{0, 0};
                const bool counts = c.score != 0 && (held < keep || c > list[keep - 1]);
                const u64 who = __ballot(counts);
                if (!who) continue;
                more = 1;
                if (counts) list[held + lanes_below(who)] = c;
                const int n_list = held + __popcll(who);
                in_order();
                // (up to 128: two per lane)
                Candidate x[2];
                int r[2] = {0, 0};
#pragma unroll
                for (int y = 0; y < 2; ++y) x[y] = lane + 64 * y < n_list ? list[lane + 64 * y] : Candidate{0, 0};
                for (int j = 0; j < n_list; ++j) {
                    const Candidate o = list[j];
#pragma unroll
                    for (int y = 0; y < 2; ++y) r[y] += o > x[y];
                }
                in_order();
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    if (lane + 64 * y < n_list && r[y] < keep) list[r[y]] = x[y];
                in_order();
                held = min(n_list, keep);
            }
        }
        if (lane == 0) g.n[wave] = held;
        __syncthreads();
        if (lane < held) best = list[lane];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            found += g.n[w];
            for (int j = 0; j < g.n[w]; ++j) rank += g.best[w][j] > best;
        }
    }
    const long long out0 = (long long)request * keep;
    if (best.score && rank < keep) {
        const int beam = best.beam(), token = best.token();
        a.parents[out0 + rank] = row0 + beam;
        a.tokens[out0 + rank] = token;
        a.new_scores[out0 + rank] = (float)score_of(best.score);
        if (a.new_ended) a.new_ended[out0 + rank] = g.ended[beam] > 0 || (a.end_token >= 0 && token == a.end_token);
    }
    if (tid >= found && tid < keep) {
        a.parents[out0 + tid] = -1;
        a.tokens[out0 + tid] = -1;
        a.new_scores[out0 + tid] = -INFINITY;
        if (a.new_ended) a.new_ended[out0 + tid] = 0;
    }
}

}  // namespace

hipError_t launch_beam_select(const jup_beam_select_t& a, hipStream_t s) {
    const long long rows = (long long)a.n_seqs * a.n_beams;
    auto go = [&](auto kernel, int block) {
        // Slices of whole steps, of 4096 logits at least: as many as give the chip 1024 workgroups (512 rows of 131072 with 512, 1024 and 2048
        // workgroups: 59, 51 and 60 µs), 512 where more than eight are kept, as every wave begins with a list of that many (32 rows of 131072, 16 kept: 25
        // and 33), and no more than the last workgroup can look at at once, where that is four at least (one request of eight beams and 131072 tokens 17 µs
        // in place of 23, of 16 beams and 32000 22 in place of 28).
        const long long wanted = a.n_keep > 8 ? 512 : 1024, fit = kThreads * kEach / (a.n_beams * a.n_keep);
        long long most = rows >= wanted ? 1 : wanted / rows;
        if (fit >= 4 && most > fit) most = fit;
        long long steps = ((a.vocab + block - 1) / block + most - 1) / most;
        const long long least = (4096 + block - 1) / block;
        if (steps < least) steps = least;
        const int length = (int)(steps * block < a.vocab ? steps * block : a.vocab);
        const int slices = (a.vocab + length - 1) / length;
        hipLaunchKernelGGL(kernel, grid_of(rows * slices), dim3(kThreads), 0, s, a, slices, length, (int*)a.workspace,
                           (u64*)((char*)a.workspace + kCountBytes));
    };
    if (a.logits_dtype == JUP_BF16) go(select<u16, 4>, kThreads * 8 * 4);
    else go(select<float, 4>, kThreads * 4 * 4);
    return hipGetLastError();
}

}  // namespace jup
