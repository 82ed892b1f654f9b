// Verification of drafted tokens against the target's probabilities with the caller's random numbers.
#pragma once

#include "common.h"

namespace msd {

constexpr int AP_NT = 1024, AP_SEG = 4 * AP_NT;      // threads of a workgroup, tokens of a segment of the vocabulary

struct AcceptProbs {
    const float *P, *Q;
    size_t p_row, p_pos, q_row, q_pos;      // elements between requests and between positions
    const int *d, *n;
    const float *u, *w;
    int rows, gamma, V, vec;                // vec: rows of P and Q start on 16 bytes
    double2* seg;                           // [rows][segments] sums of a segment: (what is drawn from, the target's law)
    int *n_acc, *tokens;
};

// The first draft of row b that fails its test u q < p (n: none does).  Every thread gets it.
__device__ __forceinline__ int first_failure(const AcceptProbs& a, int b, int n, int* sh) {
    if (threadIdx.x == 0) *sh = n;
    __syncthreads();
    for (int j = threadIdx.x; j < n; j += AP_NT) {
        const int t = a.d[(size_t)b * a.gamma + j];
        bool ok = false;
        if (t >= 0 && t < a.V) {
            const double p = a.P[(size_t)b * a.p_row + (size_t)j * a.p_pos + t], q = a.Q ? (double)a.Q[(size_t)b * a.q_row + (size_t)j * a.q_pos + t] : 1.0;
            ok = (double)a.u[(size_t)b * a.gamma + j] * q < p;        // exact: two 24-bit factors
        }
        if (!ok) atomicMin(sh, j);
    }
    __syncthreads();
    return *sh;
}
__device__ __forceinline__ int drafts_of(const AcceptProbs& a, int b) { return a.n ? min(max(a.n[b], 0), a.gamma) : a.gamma; }

// Weights of four tokens from v on: p (what the target gives) and r (what is drawn from: the bonus token from p, else from max(0, p - q)).
__device__ __forceinline__ void weights4(const AcceptProbs& a, const float* p, const float* q, int out, int v, double* pw, double* rw) {
    float x[4] = {}, y[4] = {};
    if (a.vec && v + 3 < a.V) {
        const float4 f = *reinterpret_cast<const float4*>(p + v);
        x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
        if (q) { const float4 h = *reinterpret_cast<const float4*>(q + v); y[0] = h.x; y[1] = h.y; y[2] = h.z; y[3] = h.w; }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (v + i < a.V) { x[i] = p[v + i]; if (q) y[i] = q[v + i]; }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        pw[i] = x[i] > 0.f ? (double)x[i] : 0.0;
        const double r = (double)x[i] - (double)y[i];
        rw[i] = v + i == out ? 0.0 : r > 0.0 ? r : 0.0;               // out: the rejected token of a drafter without a law of its own
    }
}

// grid (segments, rows), block AP_NT
__global__ __launch_bounds__(AP_NT) void accept_probs_sum_kernel(AcceptProbs a) {
    __shared__ int fail;
    __shared__ double2 red[AP_NT / 64];
    const int b = blockIdx.y, n = drafts_of(a, b), k = first_failure(a, b, n, &fail);
    const bool rejected = k < n;
    const float* p = a.P + (size_t)b * a.p_row + (size_t)k * a.p_pos;
    const float* q = rejected && a.Q ? a.Q + (size_t)b * a.q_row + (size_t)k * a.q_pos : nullptr;
    const int out = rejected && !a.Q ? a.d[(size_t)b * a.gamma + k] : -1;
    double pw[4], rw[4];
    weights4(a, p, q, out, blockIdx.x * AP_SEG + threadIdx.x * 4, pw, rw);
    const double ps = dpp_sum((pw[0] + pw[1]) + (pw[2] + pw[3])), rs = dpp_sum((rw[0] + rw[1]) + (rw[2] + rw[3]));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = make_double2(rs, ps);
    __syncthreads();
    if (threadIdx.x == 0) {
        double2 t = make_double2(0.0, 0.0);
        for (int i = 0; i < AP_NT / 64; ++i) { t.x += red[i].x; t.y += red[i].y; }
        a.seg[(size_t)b * gridDim.x + blockIdx.x] = t;
    }
}

// grid (rows), block AP_NT
__global__ __launch_bounds__(AP_NT) void accept_probs_draw_kernel(AcceptProbs a, int nseg) {
    __shared__ int fail, token, first[AP_NT / 64], final_[AP_NT / 64];
    __shared__ double red[AP_NT / 64];
    const int tid = threadIdx.x, b = blockIdx.x, n = drafts_of(a, b), k = first_failure(a, b, n, &fail);
    const bool rejected = k < n;
    const float* p = a.P + (size_t)b * a.p_row + (size_t)k * a.p_pos;
    const float* q = rejected && a.Q ? a.Q + (size_t)b * a.q_row + (size_t)k * a.q_pos : nullptr;
    const int out = rejected && !a.Q ? a.d[(size_t)b * a.gamma + k] : -1;
    double Z = 0.0, Zp = 0.0;
    for (int i = 0; i < nseg; ++i) { const double2 t = a.seg[(size_t)b * nseg + i]; Z += t.x; Zp += t.y; }
    const bool from_p = !(Z > 0.0);                    // nothing is left of the residual: the target's law itself
    const double target = (double)a.w[b] * (from_p ? Zp : Z);
    double before = 0.0;
    int s = -1, s_pos = -1;                            // the segment in which the sum passes the target; the last that adds anything
    double at = 0.0, at_pos = 0.0;
    for (int i = 0; i < nseg && s < 0; ++i) {
        const double2 t = a.seg[(size_t)b * nseg + i];
        const double x = from_p ? t.y : t.x;
        if (x > 0.0) { s_pos = i; at_pos = before; }
        if (before + x > target) { s = i; at = before; }
        before += x;
    }
    if (s < 0) { s = s_pos; at = at_pos; }
    if (tid == 0) token = -1;
    if (s >= 0) {
        const int v = s * AP_SEG + tid * 4;
        double pw[4], rw[4];
        weights4(a, p, q, out, v, pw, rw);
        double* x = from_p ? pw : rw;
        const double mine = (x[0] + x[1]) + (x[2] + x[3]), scan = dpp_scan(mine);
        if ((tid & 63) == 63) red[tid >> 6] = scan;
        __syncthreads();
        double base = at;
        for (int i = 0; i < tid >> 6; ++i) base += red[i];
        // the first token that passes the target; if rounding leaves none, the last one with a weight
        const unsigned long long some = __ballot(mine > 0.0), pass = __ballot(mine > 0.0 && base + scan > target);
        const int lane = tid & 63;
        if (lane == 0) { first[tid >> 6] = -1; final_[tid >> 6] = -1; }
        if (pass && lane == __ffsll(pass) - 1) {
            double run = base + (scan - mine);
            int pick = -1;
            bool done = false;
            for (int i = 0; i < 4; ++i) {
                run += x[i];
                if (x[i] > 0.0 && !done) { pick = v + i; done = run > target; }
            }
            first[tid >> 6] = pick;
        }
        if (some && lane == 63 - __clzll(some)) final_[tid >> 6] = v + (x[3] > 0.0 ? 3 : x[2] > 0.0 ? 2 : x[1] > 0.0 ? 1 : 0);
        __syncthreads();
        if (tid == 0) {
            int t = -1;
            for (int i = 0; i < AP_NT / 64 && t < 0; ++i) t = first[i];
            for (int i = AP_NT / 64 - 1; i >= 0 && t < 0; --i) t = final_[i];
            token = t;
        }
    }
    __syncthreads();
    if (tid == 0) a.n_acc[b] = k;
    for (int j = tid; j <= a.gamma; j += AP_NT)
        a.tokens[(size_t)b * (a.gamma + 1) + j] = j < k ? a.d[(size_t)b * a.gamma + j] : j == k ? token : -1;
}

}  // namespace msd
