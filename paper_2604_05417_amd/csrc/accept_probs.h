// Verification of drafted tokens against the target's probabilities with the caller's random numbers.
#pragma once

#include "common.h"

namespace msd {

constexpr int AP_NT = 1024, AP_NW = AP_NT / 64, AP_U = 4;      // threads and wavefronts of a workgroup; requests in flight per lane and law

struct AcceptProbs {
    const float *P, *Q;
    size_t p_row, p_pos, q_row, q_pos;      // elements between requests and between positions
    const int *d, *n;
    const float *u, *w;
    int gamma, V, vec;                      // vec: rows of P and Q start on 16 bytes
    int *n_acc, *tokens;
};

// Four tokens of a law from v on, zeros past the end.
__device__ __forceinline__ f32x4 law4(const float* p, int v, int V, int vec) {
    if (vec && v + 3 < V) return *reinterpret_cast<const f32x4*>(p + v);
    f32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v + i < V ? p[v + i] : 0.f;
    return x;
}
// What four tokens add to what is drawn from: max(0, p - q) in 64 bits, a NaN nothing; not the token `out`.
__device__ __forceinline__ void rest4(const f32x4& p, const f32x4& q, int v, int out, double* r) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bool on = p[e] > q[e] && v + e != out;
        r[e] = (double)(on ? p[e] : 0.f) - (double)(on ? q[e] : 0.f);
    }
}
// Sum of the weights of the tokens v0 .. v1 - 1 over the wavefront; q == nullptr: zeros.
__device__ __forceinline__ double span_sum(const float* p, const float* q, int v0, int v1, int V, int vec, int out) {
    const int lane4 = (threadIdx.x & 63) * 4;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    double sum = 0.0, r[4];
    int c = v0;
    if (vec)
        for (; c + AP_U * 256 <= v1; c += AP_U * 256) {               // requests without a condition: all in flight together
            f32x4 x[AP_U], y[AP_U];
#pragma unroll
            for (int i = 0; i < AP_U; ++i) x[i] = *reinterpret_cast<const f32x4*>(p + c + i * 256 + lane4);
#pragma unroll
            for (int i = 0; i < AP_U; ++i) y[i] = q ? *reinterpret_cast<const f32x4*>(q + c + i * 256 + lane4) : zero;
#pragma unroll
            for (int i = 0; i < AP_U; ++i) {
                rest4(x[i], y[i], c + i * 256 + lane4, out, r);
                sum += (r[0] + r[1]) + (r[2] + r[3]);
            }
        }
    for (; c < v1; c += 256) {
        const int v = c + lane4;
        if (v >= v1) break;
        rest4(law4(p, v, V, vec), q ? law4(q, v, V, vec) : zero, v, out, r);
        sum += (r[0] + r[1]) + (r[2] + r[3]);
    }
    return dpp_sum(sum);
}

// One workgroup per request.  The tests are exact: u q and p are products and numbers of 24 bits, compared in 64.  Then one row of P - and,
// behind a rejection, one of Q - is all that is read, once: wavefront i sums the weights of its span of the vocabulary (256 tokens at a time,
// both in their ascending order), and all of them read the span that the drawn sum falls into again, from L2, to find the token (the
// span's wavefront alone, 256 tokens after the other: 32 requests 11.0 us instead of 9.0, of 128 256 tokens 28 instead of 17.4).
// What bounds it: up to hundreds of requests the chain n - d - p, q - row - sums - token, 8.0 us for one at 32000 tokens (no faster with twice the
// requests in flight); for hundreds HBM: 511 of 6 drafts at 32000 tokens, 103 MB in 22.7 us, 4.5 TB/s.
// grid (requests), block AP_NT
__global__ __launch_bounds__(AP_NT, 8) void accept_probs_kernel(AcceptProbs a) {
    __shared__ int fail, token;
    __shared__ double rest[AP_NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x;
    const int* db = a.d + (size_t)b * a.gamma;
    const float *pb = a.P + (size_t)b * a.p_row, *qb = a.Q ? a.Q + (size_t)b * a.q_row : nullptr;
    // ---- the first draft that fails its test
    const int n = a.n ? min(max(a.n[b], 0), a.gamma) : a.gamma;
    const float w = a.w[b];
    if (tid == 0) { fail = n; token = -1; }
    __syncthreads();
    for (int j = tid; j < a.gamma; j += AP_NT) {
        const int t = db[j];
        const float u = a.u[(size_t)b * a.gamma + j];
        if (j >= n) continue;
        bool ok = false;
        if (t >= 0 && t < a.V) {
            const float p = pb[(size_t)j * a.p_pos + t], q = qb ? qb[(size_t)j * a.q_pos + t] : 1.f;
            ok = (double)u * (double)q < (double)p;
        }
        if (!ok) atomicMin(&fail, j);
    }
    __syncthreads();
    const int k = fail;
    const bool rejected = k < n;
    const float* p = pb + (size_t)k * a.p_pos;
    const float* q = rejected && qb ? qb + (size_t)k * a.q_pos : nullptr;
    int out = rejected && !qb ? db[k] : -1;            // the rejected draft of a drafter without a law of its own
    // ---- sums of the wavefronts' spans
    const int span = (a.V + AP_NW * 256 - 1) / (AP_NW * 256) * 256, v0 = min(wave * span, a.V), v1 = min(v0 + span, a.V);
    auto total = [&]() {
        const double s = span_sum(p, q, v0, v1, a.V, a.vec, out);
        if (lane == 0) rest[wave] = s;
        __syncthreads();
        double Z = 0.0;
        for (int i = 0; i < AP_NW; ++i) Z += rest[i];
        return Z;
    };
    double Z = total();
    if (rejected && !(Z > 0.0)) {                      // nothing is left of the residual: the target's law itself
        q = nullptr;
        out = -1;
        __syncthreads();
        Z = total();
    }
    // ---- the span that the drawn sum falls into
    const double target = (double)w * Z;
    double before = 0.0, base = 0.0;
    int mine = -1, last = -1;                          // .. or, should rounding leave none, the last with a weight
    for (int i = 0; i < AP_NW; ++i) {
        const double x = rest[i];
        if (x > 0.0) last = i;
        if (mine < 0 && before + x > target) { mine = i; base = before; }
        before += x;
    }
    if (mine < 0) mine = last;
    if (mine >= 0) {                                   // workgroup-uniform, as is all that decides below
        // .. read again, 256 tokens a wavefront: the first of them at whose end the sum passes the target has the token
        const int m0 = mine * span, m1 = min(m0 + span, a.V);
        bool found = false;
        for (int c = m0; c < m1 && !found; c += AP_NW * 256) {
            const int v = c + (wave * 64 + lane) * 4;
            f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
            if (v < m1) {
                x = law4(p, v, a.V, a.vec);
                if (q) y = law4(q, v, a.V, a.vec);
            }
            double r[4];
            rest4(x, y, v, out, r);
            const double sum = (r[0] + r[1]) + (r[2] + r[3]), scan = dpp_scan(sum);
            __syncthreads();                           // the sums there have been read
            if (lane == 63) rest[wave] = scan;
            __syncthreads();
            int at = -1;
            last = -1;
            before = base;
            for (int i = 0; i < AP_NW; ++i) {
                const double t = rest[i];
                if (t > 0.0) last = i;
                if (at < 0 && t > 0.0 && before + t > target) { at = i; base = before; }
                before += t;
            }
            found = at >= 0;
            if (wave == (found ? at : last)) {         // wavefront-uniform; should rounding leave none: the last token with a weight so far
                const unsigned long long some = __ballot(sum > 0.0), pass = __ballot(sum > 0.0 && base + scan > target);
                const int l = found && pass ? __ffsll(pass) - 1 : 63 - __clzll(some);
                double run = base + (scan - sum);
                int pick = -1;
                bool done = false;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    run += r[e];
                    if (r[e] > 0.0 && !done) { pick = v + e; done = found && run > target; }
                }
                if (lane == l) token = pick;
            }
            base = before;
        }
    }
    __syncthreads();
    if (tid == 0) a.n_acc[b] = k;
    for (int j = tid; j <= a.gamma; j += AP_NT) a.tokens[(size_t)b * (a.gamma + 1) + j] = j < k ? db[j] : j == k ? token : -1;
}

}  // namespace msd
