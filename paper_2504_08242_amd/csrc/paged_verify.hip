// Verification of drafted tokens against the target's probabilities (include/jupiter_paged.h).
//
// With x the token drafted behind row r: accepted while u_r q_r(x) < p_r(x), both sides exact in 64 bits (products of two
// 24-bit numbers).  At the first rejection the next token is drawn from w = max(p - q, 0), behind the last draft from p: the
// lowest j whose running sum exceeds u * sum(w).  Sums are in 64 bits: with up to 2^17 addends of 24 bits in different orders
// they differ by 1e-16 of the whole, where neighbouring borders are 1e-5 apart and 32-bit sums would be 1e-7 off.
#include "paged.h"

namespace jup {
namespace {

constexpr int kVerifyThreads = 1024;
constexpr int kVerifyWaves = kVerifyThreads / 64;

__device__ __forceinline__ float prob(const float* p, long long i) { return p[i]; }
__device__ __forceinline__ float prob(const u16* p, long long i) { return bf2f(p[i]); }

// What the next token is drawn from: a row of the target's probabilities, less the draft's, or without one token.
template <class T>
struct Weights {
    const T *p, *q;
    int without;  // -1: nothing
    __device__ __forceinline__ double at(int j) const {
        double w = prob(p, j);
        if (q) w -= (double)prob(q, j);
        return j != without && w > 0.0 && w < INFINITY ? w : 0.0;
    }
};

__device__ __forceinline__ double wave_total(double v) {
#pragma unroll
    for (int by = 32; by > 0; by >>= 1) v += __shfl_xor(v, by, 64);
    return v;
}

// The lowest j with w_0 + .. + w_j > u * sum(w) (the last j with w_j > 0 where rounding or u leaves none); -1 if all w are 0.
// A wave owns a contiguous range, kRun columns at a time; its runs' sums say which one holds the border, and that one is
// gone through again.
template <class T>
__device__ int draw(const Weights<T>& w, int vocab, float u, double* wave_sum_lds, int* found, int* last) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = ((vocab + kVerifyWaves - 1) / kVerifyWaves + 63) / 64 * 64;
    const int lo = min(wave * each, vocab), hi = min(lo + each, vocab);
    double sum = 0.0;
    int top = -1;
    for (int j = lo + lane; j < hi; j += 64) {
        const double x = w.at(j);
        sum += x;
        if (x > 0.0) top = j;
    }
    sum = wave_total(sum);
    for (int by = 32; by > 0; by >>= 1) top = max(top, __shfl_xor(top, by, 64));
    __syncthreads();
    if (tid == 0) {
        *found = INT32_MAX;
        *last = -1;
    }
    __syncthreads();
    if (lane == 0) {
        wave_sum_lds[wave] = sum;
        atomicMax(last, top);
    }
    __syncthreads();
    double all = 0.0, before = 0.0;
    for (int i = 0; i < kVerifyWaves; ++i) {
        if (i == wave) before = all;
        all += wave_sum_lds[i];
    }
    if (*last < 0) return -1;
    const double border = u < 0.0f ? 0.0 : (double)u * all;
    if (before <= border && before + sum > border) {
        double run = before;
        bool none = true;
        for (int j0 = lo; j0 < hi; j0 += 64) {
            const int j = j0 + lane;
            double x = j < hi ? w.at(j) : 0.0;
            const bool some = x > 0.0;
            for (int by = 1; by < 64; by *= 2) {
                const double left = __shfl_up(x, by, 64);
                if (lane >= by) x += left;
            }
            const unsigned long long over = __ballot(some && run + x > border);
            if (over) {
                if (lane == 0) *found = j0 + __builtin_ctzll(over);
                none = false;
                break;
            }
            run += __shfl(x, 63, 64);
        }
        if (none && lane == 0) *found = top;  // (added up in this order the wave ends on the border)
    }
    __syncthreads();
    return *found == INT32_MAX ? *last : *found;
}

// One workgroup per request.
template <class T>
__global__ __launch_bounds__(kVerifyThreads) void verify(const jup_verify_drafts_t a) {
    __shared__ double sums[kVerifyWaves];
    __shared__ int first_rejected, found, last;
    const int i = blockIdx.x, tid = threadIdx.x;
    const int begin = a.row_start[i], end = min(a.row_start[i + 1], a.n_rows);
    if (begin < 0 || begin >= end) {
        if (tid == 0) {
            a.n_accepted[i] = 0;
            a.next_token[i] = -1;
            if (a.new_lengths) a.new_lengths[i] = a.lengths[i];
        }
        return;
    }
    if (tid == 0) first_rejected = end - 1;
    __syncthreads();
    for (int row = begin + tid; row < end - 1; row += kVerifyThreads) {
        const int x = a.tokens[row + 1];
        bool accepted = false;
        if (x >= 0 && x < a.vocab) {
            const double p = prob((const T*)a.target_probs + row * a.target_row_stride, x);
            const double q = a.draft_probs ? prob((const T*)a.draft_probs + row * a.draft_row_stride, x) : 1.0f;
            accepted = (double)a.u_accept[row] * q < p;
        }
        if (!accepted) atomicMin(&first_rejected, row);
    }
    __syncthreads();
    const int row = first_rejected, n = row - begin;
    Weights<T> w{(const T*)a.target_probs + row * a.target_row_stride, nullptr, -1};
    if (row < end - 1) {
        if (a.draft_probs) w.q = (const T*)a.draft_probs + row * a.draft_row_stride;
        else w.without = a.tokens[row + 1];
    }
    int next = draw(w, a.vocab, a.u_sample[i], sums, &found, &last);
    if (next < 0 && row < end - 1) {
        w.q = nullptr;
        w.without = -1;
        next = draw(w, a.vocab, a.u_sample[i], sums, &found, &last);
    }
    if (a.emitted)
        for (int r = begin + tid; r < end; r += kVerifyThreads) a.emitted[r] = r < row ? a.tokens[r + 1] : r == row ? next : -1;
    if (tid == 0) {
        a.n_accepted[i] = n;
        a.next_token[i] = next;
        if (a.new_lengths) a.new_lengths[i] = a.lengths[i] + 1 + n;
    }
}

}  // namespace

hipError_t launch_verify_drafts(const jup_verify_drafts_t& a, hipStream_t s) {
    if (a.probs_dtype == JUP_BF16) hipLaunchKernelGGL(verify<u16>, dim3(a.n_seqs), dim3(kVerifyThreads), 0, s, a);
    else hipLaunchKernelGGL(verify<float>, dim3(a.n_seqs), dim3(kVerifyThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace jup
