// The end of a step of a beam search, and tables and pages of requests that go on from others (include/jupiter_paged.h).
//
// Selection.  score(b, j) = scores[b] + x_bj - L_b with L_b = m_b + log sum_j exp(x_bj - m_b).  Within a row the order of the scores is that of
// the logits, so one pass over a row leaves its n_keep largest logits and (m, sum); the workgroup of a request that is done last puts the rows'
// together.  Keys, larger is better: a logit's bits in an order that integers have, then the lower token.
#include "paged.h"

namespace jup {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMost = JUP_BEAM_MOST;
constexpr float kLog2e = 1.4426950408889634f, kLog2eRest = 1.9259629911266175e-08f;  // log2(e) = the sum, to 2^-50

__device__ __forceinline__ u64 key_of(float x, int token) {  // x finite, -0 as 0
    const unsigned bits = __float_as_uint(x + 0.0f);
    return (u64)(bits ^ ((bits >> 31) ? 0xFFFFFFFFu : 0x80000000u)) << 32 | (unsigned)~token;
}
__device__ __forceinline__ float value_of(u64 key) {
    const unsigned bits = (unsigned)(key >> 32);
    return __uint_as_float(bits ^ ((bits >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ int token_of(u64 key) { return (int)~(unsigned)key; }

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
    u64 found[64 + kStep], kept[kMost];
};
__device__ __forceinline__ void in_order() {  // LDS accesses of a wave are in order; so are the compiler's
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ int keep_best(Best& b, int n, int keep, float& limit) {
    const int lane = threadIdx.x & 63;
    in_order();
    if (n <= 64) {  // (a candidate per lane)
        const u64 mine = lane < n ? b.found[lane] : 0;
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += b.found[j] > mine;
        in_order();
        if (lane < n && rank < keep) b.found[rank] = mine;
    } else {
        for (int i = lane; i < n; i += 64) {
            const u64 mine = b.found[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += b.found[j] > mine;
            if (rank < keep) b.kept[rank] = mine;
        }
        in_order();
        if (lane < min(n, keep)) b.found[lane] = b.kept[lane];
    }
    in_order();
    n = min(n, keep);
    if (n == keep) limit = fmaxf(limit, value_of(b.found[n - 1]));
    return n;
}

struct Shared {
    Best best[kWaves];
    int n[kWaves];
    float m[kWaves];
    double sum[kWaves];
    int flag;
};

// The last one done has all rows' statistics and keys.  A candidate, larger is better: its score as an integer of the same order, then the lower beam and
// token.
struct Candidate {
    u64 score, place;
    __device__ __forceinline__ bool operator>(const Candidate& o) const { return score > o.score || (score == o.score && place > o.place); }
};
__device__ __forceinline__ Candidate candidate_of(double score, int beam, int token) {
    const u64 bits = __builtin_bit_cast(u64, score + 0.0);
    return {bits ^ ((bits >> 63) ? ~0ull : 1ull << 63), ~((u64)(unsigned)beam << 32 | (unsigned)token)};
}
__device__ __forceinline__ double score_of(u64 bits) { return __builtin_bit_cast(double, bits ^ ((bits >> 63) ? 1ull << 63 : ~0ull)); }

struct Merge {
    Candidate best[kWaves][kMost + 64];
    double log_sum[kMost], score[kMost];
    int ended[kMost], n[kWaves];
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

// `slices` workgroups per row, each with `length` logits of it.
template <class T, int U>
__global__ __launch_bounds__(kThreads) void select(const jup_beam_select_t a, int slices, int length, int* count, u64* scratch) {
    typedef Logits<T> L;
    constexpr int V = L::V;
    __shared__ Lds lds;
    Shared& s = lds.s;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = (int)(block_number() / (unsigned)slices), slice = (int)(block_number() - (unsigned)row * slices);
    if (row >= a.n_seqs * a.n_beams) return;
    const int request = row / a.n_beams, keep = a.n_keep;
    u64* mine = scratch + ((long long)row * slices + slice) * kLeft;
    const float so_far = a.scores[row];
    const bool reads = fabsf(so_far) < INFINITY && !(a.ended && a.ended[row]);
    // statistics of a thread: the sum of exp(x - m), m one of its first logits
    float m = -INFINITY, limit = -INFINITY;
    double sum = 0.0;
    int n = 0;  // candidates of the wave
    if (reads) {
        const T* x = (const T*)a.logits + row * a.row_stride;
        const int end = min((slice + 1) * length, a.vocab);
        for (int j0 = slice * length; j0 < end; j0 += kThreads * V * U) {
            typename L::vec raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + (u * kThreads + tid) * V;
                if (j + V <= end) {
                    raw[u] = *(const typename L::vec*)(x + j);
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) raw[u][e] = j + e < end ? x[j + e] : (T)(sizeof(T) == 2 ? 0xFF80 : -INFINITY);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float v[V], top = -INFINITY;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    v[e] = L::value(raw[u][e]);
                    v[e] = v[e] < INFINITY ? v[e] : -INFINITY;  // (NaN too)
                    top = fmaxf(top, v[e]);
                }
                // (m need not be the largest: sums have room for 2^86 times as much, and lo keeps far exponentials exact)
                const float m_new = top > m + 60.0f ? top : m;
                if (m_new > -INFINITY) {
                    float part = 0.f;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        // exp(d) = 2^(hi + lo), lo what the product hi loses
                        const float d = v[e] - m_new, hi = d * kLog2e, lo = __builtin_fmaf(d, kLog2eRest, __builtin_fmaf(d, kLog2e, -hi));
                        const float p = __builtin_amdgcn_exp2f(hi);
                        part += d > -104.0f ? __builtin_fmaf(p * lo, 0.69314718f, p) : 0.f;
                    }
                    sum = m_new > m ? (m > -INFINITY ? sum * exp((double)m - (double)m_new) : 0.0) + part : sum + part;
                    m = m_new;
                }
                const bool first = limit == -INFINITY;
                if (first && n == 0) {
                    // Lanes in as many groups as are kept, or more: no group's best is below the least of the groups' bests, so that
                    // many logits are not.
                    float t = top;
                    int group = 64;  // lanes of one
                    while (group > 1 && 64 / group < keep) group >>= 1;
                    for (int x2 = 1; x2 < group; x2 <<= 1) t = fmaxf(t, __shfl_xor(t, x2, 64));
                    for (int x2 = group; x2 < 64; x2 <<= 1) t = fminf(t, __shfl_xor(t, x2, 64));
                    limit = t;
                }
                // (in the round that makes the limit what equals it counts)
                if (!__any(first ? top >= limit && top > -INFINITY : top > limit)) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const bool counts = first ? v[e] >= limit && v[e] > -INFINITY : v[e] > limit;
                    const u64 who = __ballot(counts);
                    if (counts) s.best[wave].found[n + __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0))] =
                        key_of(v[e], j0 + (u * kThreads + tid) * V + e);
                    n += __popcll(who);
                }
                if (n > 64) n = keep_best(s.best[wave], n, keep, limit);
            }
        }
    }
    n = keep_best(s.best[wave], n, keep, limit);
    // the wave's statistics
    float m_wave = m;
#pragma unroll
    for (int by = 32; by > 0; by >>= 1) m_wave = fmaxf(m_wave, __shfl_xor(m_wave, by, 64));
    sum = m > -INFINITY ? sum * exp((double)m - (double)m_wave) : 0.0;
#pragma unroll
    for (int by = 32; by > 0; by >>= 1) sum += __shfl_xor(sum, by, 64);
    if (lane == 0) {
        s.n[wave] = n;
        s.m[wave] = m_wave;
        s.sum[wave] = sum;
    }
    __syncthreads();
    // the workgroup's: a thread has a key and counts those above it
    const int k = tid / kWaves, of = tid % kWaves;
    int all = 0;
    float m_all = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        all += s.n[w];
        m_all = fmaxf(m_all, s.m[w]);
    }
    if (k < s.n[of]) {
        const u64 key = s.best[of].found[k];
        int rank = k;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            if (w != of)
                for (int j = 0; j < s.n[w] && s.best[w].found[j] > key; ++j) ++rank;
        if (rank < keep) leave(mine + 2 + rank, key);
    }
    if (tid >= all && tid < keep) leave(mine + 2 + tid, 0);
    if (tid == 0) {
        double total = 0.0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            if (s.m[w] > -INFINITY) total += s.sum[w] * exp((double)s.m[w] - (double)m_all);
        leave(mine, __float_as_uint(m_all));
        leave(mine + 1, __builtin_bit_cast(u64, total));
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

    Merge& g = lds.m;
    const int row0 = request * a.n_beams;
    const u64* from = scratch + (long long)row0 * slices * kLeft;
    if (tid < a.n_beams) {
        float top = -INFINITY;
        for (int x = 0; x < slices; ++x) top = fmaxf(top, __uint_as_float((unsigned)left(from + (tid * slices + x) * kLeft)));
        double total = 0.0;
        for (int x = 0; x < slices; ++x) {
            const u64* at = from + (tid * slices + x) * kLeft;
            const float part = __uint_as_float((unsigned)left(at));
            if (part > -INFINITY) total += __builtin_bit_cast(double, left(at + 1)) * exp((double)part - (double)top);
        }
        g.log_sum[tid] = (double)top + log(total);
        const float score = a.scores[row0 + tid];
        g.score[tid] = score;
        g.ended[tid] = !(fabsf(score) < INFINITY) ? -1 : a.ended && a.ended[row0 + tid] ? 1 : 0;  // -1: no candidates
    }
    __syncthreads();
    // Lists (a slice of a beam's row each) are best first: a wave goes through its lists' first entries, then the second ones, and is done where
    // none of a round is better than the last of what it keeps.
    const int lists = a.n_beams * slices;
    auto candidate = [&](int at, int k) -> Candidate {
        const int beam = at / slices;
        if (g.ended[beam] != 0) return g.ended[beam] > 0 && at == beam * slices && k == 0 ? candidate_of(g.score[beam], beam, a.end_token) : Candidate{0, 0};
        const u64 key = left(from + (long long)at * kLeft + 2 + k);
        return key ? candidate_of(g.score[beam] + ((double)value_of(key) - g.log_sum[beam]), beam, token_of(key)) : Candidate{0, 0};
    };
    int held = 0;  // of this wave's list, best first
    Candidate* list = g.best[wave];
    for (int k0 = 0, more = 1; k0 < keep && more; ++k0) {
        more = 0;
        for (int at0 = wave * 64; at0 < lists; at0 += kThreads) {
            const Candidate c = at0 + lane < lists ? candidate(at0 + lane, k0) : Candidate{0, 0};
            const bool counts = c.score != 0 && (held < keep || c > list[keep - 1]);
            const u64 who = __ballot(counts);
            if (!who) continue;
            more = 1;
            if (counts) list[held + __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0))] = c;
            const int n_list = held + __popcll(who);
            in_order();
            // (up to 128: two per lane)
            Candidate x[2];
            int rank[2] = {0, 0};
#pragma unroll
            for (int y = 0; y < 2; ++y) x[y] = lane + 64 * y < n_list ? list[lane + 64 * y] : Candidate{0, 0};
            for (int j = 0; j < n_list; ++j) {
                const Candidate o = list[j];
#pragma unroll
                for (int y = 0; y < 2; ++y) rank[y] += o > x[y];
            }
            in_order();
#pragma unroll
            for (int y = 0; y < 2; ++y)
                if (lane + 64 * y < n_list && rank[y] < keep) list[rank[y]] = x[y];
            in_order();
            held = min(n_list, keep);
        }
    }
    if (lane == 0) g.n[wave] = held;
    __syncthreads();
    int found = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) found += g.n[w];
    const long long out0 = (long long)request * keep;
    if (k < g.n[of]) {
        const Candidate c = g.best[of][k];
        int rank = k;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            if (w != of)
                for (int j = 0; j < g.n[w] && g.best[w][j] > c; ++j) ++rank;
        if (rank < keep) {
            const u64 place = ~c.place;
            const int beam = (int)(place >> 32), token = (int)(unsigned)place;
            a.parents[out0 + rank] = row0 + beam;
            a.tokens[out0 + rank] = token;
            a.new_scores[out0 + rank] = (float)score_of(c.score);
            if (a.new_ended) a.new_ended[out0 + rank] = g.ended[beam] > 0 || (a.end_token >= 0 && token == a.end_token);
        }
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
        // slices of whole steps: as many as give the chip 1024 workgroups, of 4096 logits at least
        const long long most = rows >= 1024 ? 1 : 1024 / rows;
        long long steps = ((a.vocab + block - 1) / block + most - 1) / most;
        const long long least = (4096 + block - 1) / block;
        if (steps < least) steps = least;
        const int length = (int)(steps * block < a.vocab ? steps * block : a.vocab);
        const int slices = (a.vocab + length - 1) / length;
        hipLaunchKernelGGL(kernel, grid_of(rows * slices), dim3(kThreads), 0, s, a, slices, length, (int*)a.workspace,
                           (u64*)((char*)a.workspace + kCountBytes));
    };
    if (a.logits_dtype == JUP_BF16) go(select<u16, 2>, kThreads * 8 * 2);
    else go(select<float, 4>, kThreads * 4 * 4);
    return hipGetLastError();
}

}  // namespace jup
