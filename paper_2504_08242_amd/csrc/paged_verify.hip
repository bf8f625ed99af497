// Verification of drafted tokens against the target's probabilities (include/jupiter_paged.h).
//
// With x the token drafted behind row r: accepted while u_r q_r(x) < p_r(x), both sides exact in 64 bits (products of two
// 24-bit numbers).  At the first rejection the next token is drawn from w = max(p - q, 0), behind the last draft from p: the
// lowest j whose running sum exceeds u * sum(w).  Sums are in 64 bits: in any order they are off by at most 2^-53 of the whole for every
// addition on the longest way through them (a thread's tokens, a wave, the workgroup, the slices: below 128 for 131072 tokens, 1.4e-14, and
// 65700 for 2^30, 7e-12), where neighbouring borders are about 1 / vocab apart and 32-bit sums would be 6e-8 off for
// every addition.
#include "paged.h"

namespace jup {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
// E: probabilities of a thread at a time; kThreads * E are a workgroup's, the shortest slice
constexpr int kMostSlices = kVerifySlices;

// What the next token is drawn from: a row of the target's probabilities, less the draft's, or without one token.
template <class T>
struct Weights {
    const T *p, *q;
    int without;  // -1: nothing
    static __device__ __forceinline__ float value(float x) { return x; }
    static __device__ __forceinline__ float value(u16 x) { return bf2f(x); }
    __device__ __forceinline__ double weight(T pj, T qj, int j) const {
        double w = value(pj);
        if (q) w -= (double)value(qj);
        return j != without && w > 0.0 && w < INFINITY ? w : 0.0;
    }
    // f(p_j, q_j, j) for N consecutive j from `first` on, those below `end`.  (Rows of an odd vocabulary begin anywhere: 16-byte loads need
    // no more than a probability's own alignment; one by one, 64 requests and 131073 tokens take 73 µs instead of 33.)
    template <int N, class F>
    __device__ __forceinline__ void run(int first, int end, F f) const {
        if (first + N <= end) {
            constexpr int V = 16 / sizeof(T);
            typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
            vec a[N / V], b[N / V];
#pragma unroll
            for (int k = 0; k < N / V; ++k) a[k] = *(const vec*)(p + first + k * V);
            if (q) {
#pragma unroll
                for (int k = 0; k < N / V; ++k) b[k] = *(const vec*)(q + first + k * V);
            }
#pragma unroll
            for (int k = 0; k < N; ++k) f(a[k / V][k % V], q ? b[k / V][k % V] : T(0), first + k);
        } else {
            for (int k = 0; k < N; ++k)
                if (first + k < end) f(p[first + k], q ? q[first + k] : T(0), first + k);
        }
    }
};

__device__ __forceinline__ double wave_total(double v) {
#pragma unroll
    for (int by = 32; by > 0; by >>= 1) v += __shfl_xor(v, by, 64);
    return v;
}

struct Shared {
    double sum[kMostSlices > kWaves ? kMostSlices : kWaves];
    int first_rejected, found, flag;
};

// Sum of w over [lo, hi), the same in all threads.  64-bit operations are what this costs (half the rate of 32-bit ones, five per
// token): the maximum with 0 takes care of negative differences and of NaN; an infinity shows in the sum, which is then made again
// with every weight looked at.
template <int E, class T>
__device__ double add_up(const Weights<T>& w, int lo, int hi, Shared& s) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int V = 16 / sizeof(T);
    double sum = 0.0;
    for (int careful = 0; careful < 2; ++careful) {
        double mine = 0.0;
        for (int j0 = lo; j0 < hi; j0 += kThreads * E) {
#pragma unroll
            for (int k = 0; k < E / V; ++k)  // neighbouring threads have neighbouring pieces of 16 bytes
                w.template run<V>(j0 + (k * kThreads + tid) * V, hi, [&](T p, T q, int j) {
                    mine += careful ? w.weight(p, q, j) : fmax((double)(j == w.without ? 0.0f : w.value(p)) - (double)w.value(q), 0.0);
                });
        }
        mine = wave_total(mine);
        __syncthreads();
        if (lane == 0) s.sum[wave] = mine;
        __syncthreads();
        sum = 0.0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) sum += s.sum[i];
        if (sum < INFINITY) break;
    }
    return sum;
}

// The last j with w_j > 0, or -1.
template <class T>
__device__ int last_weight(const Weights<T>& w, int vocab, Shared& s) {
    const int tid = threadIdx.x;
    int last = -1;
    for (int j = tid; j < vocab; j += kThreads)
        if (w.weight(w.p[j], w.q ? w.q[j] : T(0), j) > 0.0) last = j;
    __syncthreads();
    if (tid == 0) s.found = -1;
    __syncthreads();
    atomicMax(&s.found, last);
    __syncthreads();
    return s.found;
}

// The lowest j of [lo, hi) with before + w_lo + .. + w_j > border, or -1.  A thread has E neighbours.
template <int E, class T>
__device__ int search(const Weights<T>& w, int lo, int hi, double before, double border, Shared& s) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int j0 = lo; j0 < hi; j0 += kThreads * E) {
        double mine = 0.0;
        w.template run<E>(j0 + tid * E, hi, [&](T p, T q, int j) { mine += w.weight(p, q, j); });
        double upto = mine;
#pragma unroll
        for (int by = 1; by < 64; by *= 2) {
            const double left = __shfl_up(upto, by, 64);
            if (lane >= by) upto += left;
        }
        __syncthreads();
        if (tid == 0) s.found = INT32_MAX;
        if (lane == 63) s.sum[wave] = upto;
        __syncthreads();
        double run = before, all = before;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            if (i == wave) run = all;
            all += s.sum[i];
        }
        run += upto - mine;
        if (mine > 0.0 && run + mine > border) {
            // (threads behind the one that has the border get here too, and find something later)
            int at = INT32_MAX;
            w.template run<E>(j0 + tid * E, hi, [&](T p, T q, int j) {
                const double x = w.weight(p, q, j);
                run += x;
                if (x > 0.0 && run > border) at = min(at, j);
            });
            if (at < INT32_MAX) atomicMin(&s.found, at);
        }
        __syncthreads();
        if (s.found < INT32_MAX) return s.found;
        before = all;
    }
    return -1;
}

// `slices` workgroups per request, each with `length` tokens of the vocabulary.  All of them find the row (a few loads); the one that
// is done last knows where the border is and goes through its slice again.  Bound by trips to memory behind one another (rows, tokens,
// their probabilities, the slice, its sum on the way to memory, the other slices' sums, the slice with the border): 10.0 µs for one request
// and 32000 tokens, 12.4 for 16 requests (one workgroup of 1024 threads per request instead: 22); 64 requests and 131072 tokens, 67 MB, take 27.
template <class T, int E>
__global__ __launch_bounds__(kThreads) void verify(const jup_verify_drafts_t a, int slices, int length, int* count, double* scratch) {
    __shared__ Shared s;
    const int i = blockIdx.x / slices, slice = blockIdx.x - i * slices, tid = threadIdx.x;
    const int begin = a.row_start[i], end = min(a.row_start[i + 1], a.n_rows);
    if (begin < 0 || begin >= end) {
        if (tid == 0 && slice == 0) {
            a.n_accepted[i] = 0;
            a.next_token[i] = -1;
            if (a.new_lengths) a.new_lengths[i] = a.lengths[i];
        }
        return;
    }
    if (tid == 0) s.first_rejected = end - 1;
    __syncthreads();
    for (int row = begin + tid; row < end - 1; row += kThreads) {
        const int x = a.tokens[row + 1];
        bool accepted = false;
        if (x >= 0 && x < a.vocab) {
            const double p = Weights<T>::value(((const T*)a.target_probs)[row * a.target_row_stride + x]);
            const double q = a.draft_probs ? Weights<T>::value(((const T*)a.draft_probs)[row * a.draft_row_stride + x]) : 1.0f;
            accepted = (double)a.u_accept[row] * q < p;
        }
        if (!accepted) atomicMin(&s.first_rejected, row);
    }
    __syncthreads();
    const int row = s.first_rejected, n = row - begin;
    Weights<T> w{(const T*)a.target_probs + row * a.target_row_stride, nullptr, -1};
    if (row < end - 1) {
        if (a.draft_probs) w.q = (const T*)a.draft_probs + row * a.draft_row_stride;
        else w.without = a.tokens[row + 1];
    }
    const double sum = add_up<E>(w, min(slice * length, a.vocab), min((slice + 1) * length, a.vocab), s);
    if (slices > 1) {
        float* mine = (float*)(scratch + (long long)i * slices + slice);
        if (tid == 0) {
            const unsigned long long bits = __builtin_bit_cast(unsigned long long, sum);
            store_coherent2(mine, __uint_as_float((unsigned)bits), __uint_as_float((unsigned)(bits >> 32)));
            wait_stores_performed();
            const int before = arrive_coherent(count + i);
            s.flag = before == slices - 1;
            if (before == slices - 1) count[i] = 0;  // ready for the next launch
        }
        __syncthreads();
        if (!s.flag) return;
        if (tid < slices) {
            const float2 x = load_coherent2((const float*)(scratch + (long long)i * slices + tid));
            s.sum[tid] = __builtin_bit_cast(double, (unsigned long long)__float_as_uint(x.x) | ((unsigned long long)__float_as_uint(x.y) << 32));
        }
        __syncthreads();
    } else {
        __syncthreads();
        if (tid == 0) s.sum[0] = sum;
        __syncthreads();
    }
    const float u = a.u_sample[i];
    int next = -1, at = -1;  // at: the slice with the border
    double all = 0.0, before = 0.0, run = 0.0;
    for (int k = 0; k < slices; ++k) all += s.sum[k];
    const double border = u < 0.0f ? 0.0 : (double)u * all;
    for (int k = 0; k < slices; ++k) {
        if (at < 0 && run + s.sum[k] > border) {
            at = k;
            before = run;
        }
        run += s.sum[k];
    }
    // (beyond the slice, should its sum in this order fall short of the border by a rounding)
    if (at >= 0) next = search<E>(w, min(at * length, a.vocab), a.vocab, before, border, s);
    if (next < 0) {  // hardly ever, and this workgroup alone: u leaves no token (or rounding does), or there is none
        next = last_weight(w, a.vocab, s);
        if (next < 0 && row < end - 1) {  // a rejected row whose weights are all 0: the target itself
            w.q = nullptr;
            w.without = -1;
            const double whole = add_up<E>(w, 0, a.vocab, s);
            next = search<E>(w, 0, a.vocab, 0.0, u < 0.0f ? 0.0 : (double)u * whole, s);
            if (next < 0) next = last_weight(w, a.vocab, s);
        }
    }
    if (a.emitted)
        for (int r = begin + tid; r < end; r += kThreads) a.emitted[r] = r < row ? a.tokens[r + 1] : r == row ? next : -1;
    if (tid == 0) {
        a.n_accepted[i] = n;
        a.next_token[i] = next;
        if (a.new_lengths) a.new_lengths[i] = a.lengths[i] + 1 + n;
    }
}

}  // namespace

hipError_t launch_verify_drafts(const jup_verify_drafts_t& a, hipStream_t s) {
    auto go = [&](auto kernel, int each) {
        const int block = kThreads * each;
        const int length = (int)(((long long)a.vocab + (long long)kMostSlices * block - 1) / ((long long)kMostSlices * block)) * block;
        const int slices = (a.vocab + length - 1) / length;
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.n_seqs * (unsigned)slices), dim3(kThreads), 0, s, a, slices, length, (int*)a.workspace,
                           (double*)((char*)a.workspace + kCountBytes));
    };
    // Slices of 4096 tokens, or of 8192 where the short ones would be more workgroups than four per CU.  16 requests and 32000 tokens 11.5 and
    // 15.6 µs, 32 and 131072 (1024 short slices) 19.8 and 20.4; 64 and 131072 27.8 and 27.0, 256 and 32000 21.5 and 19.5.
    const bool shorter = (long long)a.n_seqs * ((a.vocab + 4095) / 4096) <= 1024;
    if (a.probs_dtype == JUP_BF16) shorter ? go(verify<u16, 16>, 16) : go(verify<u16, 32>, 32);
    else shorter ? go(verify<float, 16>, 16) : go(verify<float, 32>, 32);
    return hipGetLastError();
}

}  // namespace jup
