// Attention of ragged blocks over 4-bit pages.
#pragma once

#include "common.h"
#include "pages.h"
#include "pages_plan.h"

namespace msd {

struct PagesAttn {
    const void* q;           // [rows][H][hd], rows ldq elements apart: bf16 (one term) or fp32 (two)
    void* out;               // the same, ldo apart; split != 0: two bf16 terms (store_terms4, lo_off)
    size_t ldq, ldo, lo_off;
    const int *table, *start, *lens;
    float* rec;
    float scale2;            // scale * log2(e)
    int split, B, width, rows, H, G, max_new, spw, nsp, ncg;
};

// What request b is, bounded by what the arrays hold: rows row0 .. row0 + n - 1, L positions.
struct PagesReq { int row0, n, L; };
__device__ __forceinline__ PagesReq pages_req(const PagesAttn& a, int b, int shift) {
    PagesReq r;
    r.row0 = max(a.start[b], 0);
    r.n = max(min(a.start[b + 1], a.rows) - r.row0, 0);
    r.L = (int)min((long long)max(a.lens[b], 0), (long long)a.width << shift);
    return r;
}
// Positions that the columns c0 .. c0 + cols - 1 of a request see together, sub-blocks of 32 of them, and records that they leave.
__device__ __forceinline__ int pages_seen(const PagesReq& r, int G, int c0, int cols) {
    const int last = (min(c0 + cols, r.n * G) - 1) / G;
    return max(min(r.L, r.L - r.n + last + 1), 0);
}
__device__ __forceinline__ int pages_records_of(const PagesAttn& a, int seen) { return max(1, min(((seen + 31) / 32 + a.spw - 1) / a.spw, a.nsp)); }

// Byte i of w as the scale of a conversion, which goes by the exponent of its operand alone: the bits of the other bytes that this leaves in sign
// and mantissa do not matter (one instruction instead of two; a layout test and the tests of the values would notice).
template <int I>
__device__ __forceinline__ float scale_of(uint32_t w) { return __uint_as_float(I < 3 ? w << (23 - 8 * I) : w >> 1); }
#define PAGES_CVT(W, S, B) __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(W, S, B))

// max over the four lanes of a column
__device__ __forceinline__ float column_max(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// the value of the lane N places on in its row of 16
template <int N>
__device__ __forceinline__ float rotated(float v) { return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + N, 0xf, 0xf, false)); }
// x = its bf16 terms, largest first
template <int TERMS>
__device__ __forceinline__ void terms_of(float a, float b, uint32_t* t) {
#pragma unroll
    for (int u = 0; u < TERMS; ++u) {
        t[u] = f2bf2(a, b);
        a -= __uint_as_float(t[u] << 16);
        b -= __uint_as_float(t[u] & 0xffff0000u);
    }
}

template <int N> struct Words { uint32_t w[N]; };
template <int N>
__device__ __forceinline__ Words<N> load_words(const unsigned char* p) {
    Words<N> r;
    if constexpr (N == 4) { const uint4 x = *reinterpret_cast<const uint4*>(p); r.w[0] = x.x; r.w[1] = x.y; r.w[2] = x.z; r.w[3] = x.w; }
    else if constexpr (N == 2) { const uint2 x = *reinterpret_cast<const uint2*>(p); r.w[0] = x.x; r.w[1] = x.y; }
    else r.w[0] = *reinterpret_cast<const uint32_t*>(p);
    return r;
}

// A row of four outputs.
template <int TERMS>
__device__ __forceinline__ void pages_store4(const PagesAttn& a, int row, int h, int hd, int d, const f32x4& y) {
    if (TERMS >= 2 && a.split) store_terms4(reinterpret_cast<float*>(a.out), a.split, a.lo_off, (size_t)row * a.ldo + (size_t)h * hd + d, make_float4(y[0], y[1], y[2], y[3]));
    else if (TERMS >= 2) *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + (size_t)row * a.ldo + (size_t)h * hd + d) = y;
    else *reinterpret_cast<uint2*>(reinterpret_cast<bf16_t*>(a.out) + (size_t)row * a.ldo + (size_t)h * hd + d) = make_uint2(f2bf2(y[0], y[1]), f2bf2(y[2], y[3]));
}

// One workgroup of 4 wavefronts per (request, K/V head, group of 16 CT columns, span of positions).  A column is a (row, query head) pair of
// the K/V head, so K and V are read and widened once for all of them.  A wavefront walks every fourth sub-block of 32 positions of the
// span with a running (maximum, sum, O) per column and no barrier:
//   S^T[pos][col] = K . q^T    A = K codes straight from the page, widened to bf16 (exact: 2 significant bits times a power of two)
//   O^T[d][col]  += V^T . P^T  A = V widened and transposed pairwise in registers, B = P straight from the registers that held S^T (slot 8 g
//                              + i of the 32 positions stands for 4 g + i or 16 + 4 g + i - 4)
// TERMS = 2: q and P as two bf16 terms each.  The maximum is only raised, and O rescaled, when a score exceeds it by more than 2^8; sums are in
// 32 bits.  The next sub-block is requested while the present one is multiplied.  The wavefronts merge through LDS; a context of one
// record is written as it is, several are merged by pages_merge_kernel.
template <int HD, int CT, int TERMS, int PACK>
struct PagesForm {
    static constexpr int W = 16 / PACK;                               // (row, head) pairs of a column tile
    static constexpr int NQ = PACK == 1 ? TERMS : PACK == 2 ? 2 : 1;  // products per operand of K or V
    static constexpr int Q = CT * (HD / 32) * NQ;                     // operands of q, four registers each
    static constexpr bool QL = Q > 8 || (PACK == 2 && HD == 128);     // more than 32 registers (or what would spill): they stay in LDS
    static constexpr int OS = HD + 4, LDS = QL && Q * 1024 > PA_NW * 16 * OS * 4 ? Q * 1024 : PA_NW * 16 * OS * 4;
    static constexpr int WAVES = HD == 128 ? (CT == 1 ? 4 : 2) : HD == 64 ? (CT == 1 ? 4 : 3) : CT == 1 ? 6 : 4;      // per SIMD, without spills
};
template <int HD, int CT, int TERMS, int PACK>
__global__ __launch_bounds__(64 * PA_NW, (PagesForm<HD, CT, TERMS, PACK>::WAVES)) void attn_pages_kernel(PagesAttn a, Pool pl) {
    typedef PagesForm<HD, CT, TERMS, PACK> F;
    constexpr int KC = HD / 32, OS = F::OS, W = F::W, NQ = F::NQ;
    __shared__ __align__(16) unsigned char lds[F::LDS];
    float* o_sh = reinterpret_cast<float*>(lds);
    u32x4* q_sh = reinterpret_cast<u32x4*>(lds);                      // [column tile][k][term][lane]
    __shared__ float mx_sh[PA_NW][CT * W], sum_sh[PA_NW][CT * W];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g = lane >> 4;
    int id = blockIdx.x;
    const int cg = id % a.ncg; id /= a.ncg;
    const int sp = id % a.nsp; id /= a.nsp;
    const int kh = id % pl.KH, b = id / pl.KH;
    const PagesReq rq = pages_req(a, b, pl.shift);
    const int ncol = rq.n * a.G, c0 = cg * W * CT, group = col / W;      // group: which terms of a row this lane's column carries
    if (c0 >= ncol) return;                            // workgroup-uniform, as is the next
    const int seen = pages_seen(rq, a.G, c0, W * CT), nsub = (seen + 31) / 32, nrec = pages_records_of(a, seen);
    if (sp >= nrec) return;
    const int s1 = sp == nrec - 1 ? nsub : min(nsub, (sp + 1) * a.spw);
    const int all_see = rq.L - rq.n + c0 / a.G;        // every column sees the positions up to here
    int lim[CT];
    u32x4 qf[F::QL ? 1 : CT][KC][NQ];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int c = c0 + ct * W + col % W, cc = min(c, ncol - 1), r = cc / a.G, h = kh * a.G + (cc - r * a.G);
        lim[ct] = c < ncol ? min(rq.L - rq.n + r, rq.L - 1) : -1;
        const size_t at = (size_t)(rq.row0 + r) * a.ldq + (size_t)h * HD + g * 8;
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            if (F::QL && ((ct * KC + k) & (PA_NW - 1)) != wave) continue;          // each wavefront brings a part
            u32x4 x[NQ];
            if constexpr (TERMS == 1) x[0] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const bf16_t*>(a.q) + at + k * 32);
            else {
                float f[8];
                load8(reinterpret_cast<const float*>(a.q) + at + k * 32, f);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t t[TERMS];
                    terms_of<TERMS>(f[2 * i], f[2 * i + 1], t);
                    if constexpr (PACK == 1) {
#pragma unroll
                        for (int u = 0; u < TERMS; ++u) x[u][i] = t[u];
                    } else if constexpr (PACK == 2) {
                        x[0][i] = group ? t[1] : t[0];
                        x[1][i] = group ? 0u : t[2];
                    } else x[0][i] = group == 0 ? t[0] : group == 1 ? t[1] : group == 2 ? t[2] : 0u;
                }
            }
#pragma unroll
            for (int u = 0; u < NQ; ++u) {
                if constexpr (F::QL) q_sh[((ct * KC + k) * NQ + u) * 64 + lane] = x[u];
                else qf[ct][k][u] = x[u];
            }
        }
    }
    if constexpr (F::QL) __syncthreads();
    f32x4 o[CT][KC][2];
    float mx[CT], sum[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        mx[ct] = -INFINITY;
        sum[ct] = 0.f;
#pragma unroll
        for (int j = 0; j < KC; ++j) o[ct][j][0] = o[ct][j][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    Words<KC> kd[2], vd[2], vs[2];
    uint32_t ks[2];
    const int tshift = pl.shift - 4, tlast = max(seen - 1, 0) >> 4;
    const int* tab = a.table + (size_t)b * a.width;
    const int first = sp * a.spw + wave;               // this wavefront's sub-blocks: first, first + PA_NW, ..
    // page numbers of the next 32 sub-blocks, two tiles each, one a lane: a request finds them in a register
    int ids = 0;
    auto look_up = [&](int k) {
        const int tile = min(2 * (first + (k + (lane >> 1)) * PA_NW) + (lane & 1), tlast);       // past the end: the last tile again, whose weights are zero there
        ids = (int)min((unsigned)tab[tile >> tshift], (unsigned)(pl.n_pages - 1));
    };
    auto place = [&](int k, int t) {
        const int tile = min(2 * (first + k * PA_NW) + t, tlast);
        return tile_at<HD>(pl, __builtin_amdgcn_readlane(ids, (k & 31) * 2 + t), kh, tile & ((1 << tshift) - 1));
    };
    const unsigned char *at0, *at1;                    // the tiles of the sub-block whose V is still to be requested
    auto request_k = [&](int k) {
        at0 = place(k, 0);
        at1 = place(k, 1);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const unsigned char* p = t ? at1 : at0;
            kd[t] = load_words<KC>(p + lane * Tile<HD>::LB);
            if constexpr (HD == 128) ks[t] = *reinterpret_cast<const uint32_t*>(p + Tile<HD>::KS + col * 4);
            else if constexpr (HD == 64) ks[t] = *reinterpret_cast<const uint16_t*>(p + Tile<HD>::KS + col * 2);
            else ks[t] = p[Tile<HD>::KS + col];
        }
    };
    auto request_v = [&]() {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const unsigned char* p = t ? at1 : at0;
            vd[t] = load_words<KC>(p + Tile<HD>::V + lane * Tile<HD>::LB);
            vs[t] = load_words<KC>(p + Tile<HD>::VS + g * Tile<HD>::LB);
        }
    };
    if (first < s1) {
        look_up(0);
        request_k(0);
        request_v();
    }
    for (int s = first, k = 0; s < s1; s += PA_NW, ++k) {
        const int p0 = s * 32;
        const bool more = s + PA_NW < s1;
        if (more && ((k + 1) & 31) == 0) look_up(k + 1);
        // ---- scores
        __builtin_amdgcn_s_setprio(1);
        f32x4 sc[CT][2];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) sc[ct][0] = sc[ct][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            // q stays in LDS: no more than two chunks of it are moved into registers ahead of their use
            if constexpr (F::QL) { if ((c & 1) == 0) asm volatile("" ::: "memory"); }
            u32x4 kf[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float f = c == 0 ? scale_of<0>(ks[t]) : c == 1 ? scale_of<1>(ks[t]) : c == 2 ? scale_of<2>(ks[t]) : scale_of<3>(ks[t]);
                kf[t] = u32x4{PAGES_CVT(kd[t].w[c], f, 0), PAGES_CVT(kd[t].w[c], f, 1), PAGES_CVT(kd[t].w[c], f, 2), PAGES_CVT(kd[t].w[c], f, 3)};
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int u = NQ - 1; u >= 0; --u) {
                    const bf16x8 qv = __builtin_bit_cast(bf16x8, F::QL ? q_sh[((ct * KC + c) * NQ + u) * 64 + lane] : qf[F::QL ? 0 : ct][c][u]);
#pragma unroll
                    for (int t = 0; t < 2; ++t) sc[ct][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[t]), qv, sc[ct][t], 0, 0, 0);
                }
        }
        __builtin_amdgcn_s_setprio(0);
        if constexpr (PACK > 1)                        // a score is the sum over the columns that carry its row's terms
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    sc[0][t][v] += rotated<8>(sc[0][t][v]);
                    if constexpr (PACK == 4) sc[0][t][v] += rotated<4>(sc[0][t][v]);
                }
        if (more) request_k(k + 1);
        if (p0 + 31 > all_see) {                       // some column does not see all 32 positions
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int q0 = p0 + t * 16 + g * 4;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int v = 0; v < 4; ++v) sc[ct][t][v] = q0 + v <= lim[ct] ? sc[ct][t][v] : -INFINITY;
                // positions past the end: whatever lies there, V's scale must not make it infinite
                const int ok = min(max(rq.L - q0, 0), 4);
                const uint32_t keep = ok == 4 ? 0xffffffffu : (1u << (8 * ok)) - 1;
#pragma unroll
                for (int j = 0; j < KC; ++j) vs[t].w[j] &= keep;
            }
        }
        // ---- running maximum
        float tm[CT];
        bool raise = false;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            float m = fmaxf(fmaxf(fmaxf(sc[ct][0][0], sc[ct][0][1]), fmaxf(sc[ct][0][2], sc[ct][0][3])),
                            fmaxf(fmaxf(sc[ct][1][0], sc[ct][1][1]), fmaxf(sc[ct][1][2], sc[ct][1][3])));
            tm[ct] = column_max(m) * a.scale2;
            raise = raise || tm[ct] > mx[ct] + 8.f;
        }
        if (__any(raise)) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const float nm = fmaxf(mx[ct], tm[ct]), alpha = nm == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mx[ct] - nm);
                mx[ct] = nm;
                sum[ct] *= alpha;
#pragma unroll
                for (int j = 0; j < KC; ++j) { o[ct][j][0] *= alpha; o[ct][j][1] *= alpha; }
            }
        }
        // ---- weights
        u32x4 pf[CT][NQ];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const float base = mx[ct] == -INFINITY ? 0.f : mx[ct];
            float part = 0.f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[ct][t][v], a.scale2, -base));
                    sc[ct][t][v] = e;
                    part += e;
                }
            sum[ct] += part;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    float x = sc[ct][t][2 * v], y = sc[ct][t][2 * v + 1];
                    const int at = 2 * t + v;
                    if constexpr (PACK == 4) {         // every lane its own term: what the terms before it leave
#pragma unroll
                        for (int u = 1; u < TERMS; ++u) {
                            const uint32_t h = f2bf2(x, y);
                            x = __builtin_fmaf(group >= u ? -1.f : 0.f, __uint_as_float(h << 16), x);
                            y = __builtin_fmaf(group >= u ? -1.f : 0.f, __uint_as_float(h & 0xffff0000u), y);
                        }
                        pf[ct][0][at] = f2bf2(x, y);
                    } else {
                        uint32_t w[TERMS];
                        terms_of<TERMS>(x, y, w);
                        if constexpr (PACK == 2) {
                            pf[ct][0][at] = group ? w[1] : w[0];
                            pf[ct][1][at] = group ? 0u : w[2];
                        } else
#pragma unroll
                            for (int u = 0; u < TERMS; ++u) pf[ct][u][at] = w[u];
                    }
                }
        }
        // ---- products with V
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int j = 0; j < KC; ++j) {
            u32x4 even, odd;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint32_t w = vd[t].w[j], f = vs[t].w[j];
                const uint32_t x0 = PAGES_CVT(w, scale_of<0>(f), 0), x1 = PAGES_CVT(w, scale_of<1>(f), 1), x2 = PAGES_CVT(w, scale_of<2>(f), 2), x3 = PAGES_CVT(w, scale_of<3>(f), 3);
                even[2 * t] = __builtin_amdgcn_perm(x1, x0, 0x05040100u);
                even[2 * t + 1] = __builtin_amdgcn_perm(x3, x2, 0x05040100u);
                odd[2 * t] = __builtin_amdgcn_perm(x1, x0, 0x07060302u);
                odd[2 * t + 1] = __builtin_amdgcn_perm(x3, x2, 0x07060302u);
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int u = NQ - 1; u >= 0; --u) {
                    o[ct][j][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), __builtin_bit_cast(bf16x8, pf[ct][u]), o[ct][j][0], 0, 0, 0);
                    o[ct][j][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), __builtin_bit_cast(bf16x8, pf[ct][u]), o[ct][j][1], 0, 0, 0);
                }
        }
        __builtin_amdgcn_s_setprio(0);
        if (more) request_v();
    }
    // ---- merge the wavefronts
    if constexpr (F::QL) __syncthreads();              // q has been read
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        float t = sum[ct];
        t += __shfl_xor(t, 16, 64);
        t += __shfl_xor(t, 32, 64);
        if (g == 0 && group == 0) { mx_sh[wave][ct * W + col] = mx[ct]; sum_sh[wave][ct * W + col] = t; }
    }
    float* rec = nrec == 1 ? nullptr : a.rec + ((((size_t)b * pl.KH + kh) * a.ncg + cg) * a.nsp + sp) * (W * CT) * OS;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        if (ct) __syncthreads();                       // the tile before has been read
#pragma unroll
        for (int j = 0; j < KC; ++j) {                 // element v of o[ct][j][u]: dimension 32 j + 2 (4 g + v) + u
            float* dst = o_sh + (wave * 16 + col) * OS + 32 * j + 8 * g;
            *reinterpret_cast<f32x4*>(dst) = f32x4{o[ct][j][0][0], o[ct][j][1][0], o[ct][j][0][1], o[ct][j][1][1]};
            *reinterpret_cast<f32x4*>(dst + 4) = f32x4{o[ct][j][0][2], o[ct][j][1][2], o[ct][j][0][3], o[ct][j][1][3]};
        }
        __syncthreads();
        for (int i = tid; i < W * (HD / 4); i += 64 * PA_NW) {
            const int k = i / (HD / 4), d = (i - k * (HD / 4)) * 4, cc = ct * W + k, c = c0 + cc;
            if (c >= ncol) break;                      // columns ascend
            float M = mx_sh[0][cc];
#pragma unroll
            for (int w = 1; w < PA_NW; ++w) M = fmaxf(M, mx_sh[w][cc]);
            f32x4 y = {0.f, 0.f, 0.f, 0.f};
            float tot = 0.f;
#pragma unroll
            for (int w = 0; w < PA_NW; ++w) {
                const float f = mx_sh[w][cc] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx_sh[w][cc] - M);
                f32x4 x = *reinterpret_cast<const f32x4*>(o_sh + (w * 16 + k) * OS + d);
#pragma unroll
                for (int u = 1; u < (PACK == 4 ? 3 : PACK); ++u) x += *reinterpret_cast<const f32x4*>(o_sh + (w * 16 + u * W + k) * OS + d);
                y += x * f;
                tot += sum_sh[w][cc] * f;
            }
            if (rec) {
                *reinterpret_cast<f32x4*>(rec + (size_t)cc * OS + d) = y;
                if (d == 0) *reinterpret_cast<float2*>(rec + (size_t)cc * OS + HD) = make_float2(M, tot);
            } else {
                const int r = c / a.G, h = kh * a.G + (c - r * a.G);
                pages_store4<TERMS>(a, rq.row0 + r, h, HD, d, y * (tot == 0.f ? 0.f : 1.0f / tot));     // a row that sees nothing: zeros
            }
        }
    }
}

// Records of a column merged in their order.  HD / 4 lanes per (request, row, head).   grid ceil(B max_new H / units), block 256
template <int HD, int TERMS>
__global__ __launch_bounds__(256) void pages_merge_kernel(PagesAttn a, Pool pl, int cols) {
    constexpr int LN = HD / 4, OS = HD + 4;
    const long u = (long)blockIdx.x * (256 / LN) + threadIdx.x / LN;
    const int d = threadIdx.x % LN * 4;
    const int b = (int)(u / ((long)a.max_new * a.H)), x = (int)(u - (long)b * a.max_new * a.H), r = x / a.H, h = x - r * a.H;
    if (b >= a.B) return;
    const PagesReq rq = pages_req(a, b, pl.shift);
    if (r >= rq.n) return;
    const int kh = h / a.G, c = r * a.G + (h - kh * a.G), cg = c / cols, cc = c - cg * cols;
    const int nrec = pages_records_of(a, pages_seen(rq, a.G, cg * cols, cols));
    if (nrec == 1) return;                             // written already
    const float* rec = a.rec + (((size_t)b * pl.KH + kh) * a.ncg + cg) * a.nsp * cols * OS + (size_t)cc * OS;
    const size_t step = (size_t)cols * OS;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    float M = -INFINITY, tot = 0.f;
    for (int i0 = 0; i0 < nrec; i0 += 8) {             // eight records in flight; past the last one that again, with no weight
        f32x4 x[8];
        float2 ms[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float* p = rec + min(i0 + i, nrec - 1) * step;
            x[i] = *reinterpret_cast<const f32x4*>(p + d);
            ms[i] = *reinterpret_cast<const float2*>(p + HD);
        }
        float m = M;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, ms[i].x);
        const float base = m == -INFINITY ? 0.f : m, f = __builtin_amdgcn_exp2f(M - base);
        y *= f;
        tot *= f;
        M = m;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float w = __builtin_amdgcn_exp2f(ms[i].x - base);
            if (i0 + i < nrec) { y += x[i] * w; tot += ms[i].y * w; }
        }
    }
    pages_store4<TERMS>(a, rq.row0 + r, h, HD, d, y * (tot == 0.f ? 0.f : 1.0f / tot));
}

}  // namespace msd
