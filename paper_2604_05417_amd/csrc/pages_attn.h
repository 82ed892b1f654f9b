// Attention of ragged blocks over 4-bit pages.
#pragma once

#include "common.h"
#include "pages.h"
#include "pages_plan.h"

namespace msd {

struct PagesAttn {
    const void* q;           // [rows][H][hd], rows ldq elements apart: bf16 (one term) or fp32 (three)
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
__device__ __forceinline__ int sub_blocks(int seen) { return (int)(((unsigned)seen + 31) / 32); }
__device__ __forceinline__ int pages_records_of(const PagesAttn& a, int seen) { return max(1, min((sub_blocks(seen) + a.spw - 1) / a.spw, a.nsp)); }

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

constexpr u32x4 ONES = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};       // bf16

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
// TERMS = 1 (bf16 rows): P rounded to bf16, and the sum of a column that of the rounded weights, a product with ones: what a weight is off by
// cancels where it is the row's only large one, and no lane adds (24 single tokens behind 5000 17.6 / 17.1 us).
// TERMS = 3 (fp32 rows): q and P as three bf16 terms each, 24 bits; with PACK 2 or 4 the terms of a pair lie in different columns of one
// product.  The maximum is only raised, and O rescaled, when a score exceeds it by more than 2^8; sums are in 32 bits.  The next sub-block is
// requested while the present one is multiplied.  The wavefronts merge through LDS; a context of one record is written as it is, several are
// merged by pages_merge_kernel.
// What bounds it: HBM for many long contexts - 32 requests of 8 rows behind 4104 positions, 32 heads of 128, fp32 rows: 578 MB in 104 - 119 us, 4.9 - 5.5 TB/s,
// where the same requests without any arithmetic take 100 and bf16 rows 102 - with 305 vector instructions per 32 positions, two thirds of the
// cycles, and the matrix unit a quarter.  One request of 6 rows behind 2053: 7.8 us and the merge's 4, a chain of q, page number, tile and
// products per wavefront.  A deeper prefetch, non-temporal loads and eight or sixteen spans per CU change nothing.
template <int HD, int CT, int TERMS, int PACK, int NW>
struct PagesForm {
    static constexpr int W = 16 / PACK;                               // (row, head) pairs of a column tile
    static constexpr int NQ = PACK == 1 ? TERMS : PACK == 2 ? 2 : 1;  // products per operand of K or V
    static constexpr int Q = CT * (HD / 32) * NQ;                     // operands of q, four registers each
    static constexpr bool QL = Q > 8 || (PACK == 2 && HD == 128);     // more than 32 registers (or what would spill): they stay in LDS
    static constexpr int OS = HD + 4, LDS = QL && Q * 1024 > NW * 16 * OS * 4 ? Q * 1024 : NW * 16 * OS * 4;
    static constexpr int WAVES = NW > 4 ? 4 : HD == 128 ? (CT == 1 ? 4 : 2) : HD == 64 ? (CT == 1 ? 4 : 3) : CT == 1 ? 6 : 4;      // per SIMD, without spills
};
template <int HD, int CT, int TERMS, int PACK, int NW>
__global__ __launch_bounds__(64 * NW, (PagesForm<HD, CT, TERMS, PACK, NW>::WAVES)) void attn_pages_kernel(PagesAttn a, Pool pl) {
    typedef PagesForm<HD, CT, TERMS, PACK, NW> F;
    constexpr int KC = HD / 32, OS = F::OS, W = F::W, NQ = F::NQ;
    __shared__ __align__(16) unsigned char lds[F::LDS];
    float* o_sh = reinterpret_cast<float*>(lds);
    u32x4* q_sh = reinterpret_cast<u32x4*>(lds);                      // [column tile][k][term][lane]
    __shared__ float mx_sh[NW][CT * W], sum_sh[NW][CT * W];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g = lane >> 4;
    int id = blockIdx.x;
    const int cg = id % a.ncg; id /= a.ncg;
    const int sp = id % a.nsp; id /= a.nsp;
    const int kh = id % pl.KH, b = id / pl.KH;
    const PagesReq rq = pages_req(a, b, pl.shift);
    const int ncol = rq.n * a.G, c0 = cg * W * CT, group = col / W;      // group: which terms of a row this lane's column carries
    if (c0 >= ncol) return;                            // workgroup-uniform, as is the next
    const int seen = pages_seen(rq, a.G, c0, W * CT), nsub = sub_blocks(seen), nrec = pages_records_of(a, seen);
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
            if (F::QL && ((ct * KC + k) & (NW - 1)) != wave) continue;          // each wavefront brings a part
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
    f32x4 total[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        mx[ct] = -INFINITY;
        sum[ct] = 0.f;
        total[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < KC; ++j) o[ct][j][0] = o[ct][j][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    Words<KC> kd[2], vd[2], vs[2];
    uint32_t ks[2];
    const int tshift = pl.shift - 4, tlast = min(max(seen - 1, 0) >> 4, 2 * s1 - 1);
    const int* tab = a.table + (size_t)b * a.width;
    const int first = sp * a.spw + wave;               // this wavefront's sub-blocks: first, first + NW, ..
    // page numbers of the next 32 sub-blocks, two tiles each, one a lane: a request finds them in a register
    int ids = 0;
    auto look_up = [&](int k) {
        const int tile = min(2 * (first + (k + (lane >> 1)) * NW) + (lane & 1), tlast);       // past the end: the last tile again, whose weights are zero there
        ids = (int)min((unsigned)tab[tile >> tshift], (unsigned)(pl.n_pages - 1));
    };
    auto place = [&](int k, int t) {
        const int tile = min(2 * (first + k * NW) + t, tlast);
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
    for (int s = first, k = 0; s < s1; s += NW, ++k) {
        const int p0 = s * 32;
        if (((k + 1) & 31) == 0) look_up(k + 1);
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
        request_k(k + 1);                              // also behind the last: what is requested on one of two paths is waited for on both
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
                if constexpr (TERMS == 1) total[ct][0] *= alpha; else sum[ct] *= alpha;
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
                    if constexpr (TERMS > 1) part += e;
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
        if constexpr (TERMS == 1)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
                total[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ONES), __builtin_bit_cast(bf16x8, pf[ct][0]), total[ct], 0, 0, 0);
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
        request_v();
    }
    // ---- merge the wavefronts
    if constexpr (F::QL) __syncthreads();              // q has been read
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        float t = sum[ct];
        t += __shfl_xor(t, 16, 64);
        t += __shfl_xor(t, 32, 64);
        if constexpr (TERMS == 1) t = total[ct][0];
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
        for (int i = tid; i < W * (HD / 4); i += 64 * NW) {
            const int k = i / (HD / 4), d = (i - k * (HD / 4)) * 4, cc = ct * W + k, c = c0 + cc;
            if (c >= ncol) break;                      // columns ascend
            float M = mx_sh[0][cc];
#pragma unroll
            for (int w = 1; w < NW; ++w) M = fmaxf(M, mx_sh[w][cc]);
            f32x4 y = {0.f, 0.f, 0.f, 0.f};
            float tot = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
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

// The same for long blocks (prompts): every one of the four wavefronts has 16 columns of its own and all walk the same positions, 64 at a time.
// Each widens one tile of 16 positions into LDS as the operands that all of them multiply with, so that a position is widened once for 64
// columns; while they multiply, the codes of the next 64 are on their way.  One buffer, so that four workgroups share a CU: with two
// buffers and half as many 56 instead of 44 us (in the order of pairs; 1500 rows, 32 heads of 128, bf16), with 32 columns a wavefront 55, with a second team of four for
// every other step 46; the kernel above, which widens for 32 columns, 51.  What bounds it: nearly as many cycles in LDS (32 KiB read per
// wavefront and step, 1024) as in the exponentials and the widening (800) and in the products (512).
// LDS layout: [K: tile][chunk][lane] and [V: pair of tiles][chunk][even, odd][lane], 16 bytes a lane.
// Workgroup ids deal the (request, K/V head) pairs out over the 8 XCDs, so that the column groups of one share an L2.  Within a bundle of pairs
// (512 workgroups or more) the longest groups come first, and every other round over the XCD's 32 CUs goes backwards: a CU that got the
// longest group of one round gets the shortest of the next.  Pair after pair / so: prompts of 1500 rows 45.6 / 39.4 us, 4000 193 / 174, 8000 630 / 580, eight
// requests of up to 500 rows behind up to 3000 positions 89 / 64 (bf16, 32 heads of 128); bundles of 128 workgroups lose 4 - 15 % of it.
template <int HD, int TERMS>
__global__ __launch_bounds__(256, TERMS == 1 ? 4 : 3) void attn_pages_long_kernel(PagesAttn a, Pool pl) {
    constexpr int KC = HD / 32, OS = HD + 4, GC = 64;  // columns of the workgroup
    __shared__ u32x4 k_sh[4][KC][64];
    __shared__ u32x4 v_sh[2][KC][2][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int per = a.ncg * a.nsp, units = (int)(gridDim.x >> 3) / per, most = min(units, (511 + per) / per), y = blockIdx.x >> 3, bundle = y / (most * per);
    const int n_units = min(most, units - bundle * most), z = y - bundle * most * per, round = z >> 5;
    const int place = round & 1 ? min(32 * round + 31, n_units * per - 1) - (z & 31) : z, unit = (blockIdx.x & 7) + 8 * (bundle * most + place / a.nsp % n_units);
    if (unit >= a.B * pl.KH) return;                   // workgroup-uniform, as are the next two
    const int cg = a.ncg - 1 - place / (a.nsp * n_units), sp = place % a.nsp, b = unit / pl.KH, kh = unit - b * pl.KH;
    const PagesReq rq = pages_req(a, b, pl.shift);
    const int ncol = rq.n * a.G;
    if (cg * GC >= ncol) return;
    const int seen = pages_seen(rq, a.G, cg * GC, GC), nsub = sub_blocks(seen), nrec = pages_records_of(a, seen);
    if (sp >= nrec) return;
    const int it0 = sp * a.spw / 2, it1 = ((sp == nrec - 1 ? nsub : min(nsub, (sp + 1) * a.spw)) + 1) / 2;      // steps of 64 positions
    const int c0 = cg * GC + wave * 16;
    const int mine = c0 < ncol ? pages_seen(rq, a.G, c0, 16) : 0, all_see = rq.L - rq.n + c0 / a.G;       // positions that some (every) column of the wavefront sees
    const int c = c0 + col, rc = min(c, ncol - 1) / a.G, h = kh * a.G + (min(c, ncol - 1) - rc * a.G);
    const int lim = c < ncol ? min(rq.L - rq.n + rc, rq.L - 1) : -1;
    u32x4 qf[KC][TERMS];
#pragma unroll
    for (int k = 0; k < KC; ++k) {
        const size_t at = (size_t)(rq.row0 + rc) * a.ldq + (size_t)h * HD + g * 8 + k * 32;
        if constexpr (TERMS == 1) qf[k][0] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const bf16_t*>(a.q) + at);
        else {
            float f[8];
            load8(reinterpret_cast<const float*>(a.q) + at, f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t t[TERMS];
                terms_of<TERMS>(f[2 * i], f[2 * i + 1], t);
#pragma unroll
                for (int u = 0; u < TERMS; ++u) qf[k][u][i] = t[u];
            }
        }
    }
    f32x4 o[KC][2];
    float mx = -INFINITY, sum = 0.f;
    f32x4 total = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < KC; ++j) o[j][0] = o[j][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int tshift = pl.shift - 4, tlast = max(seen - 1, 0) >> 4;
    const int* tab = a.table + (size_t)b * a.width;
    Words<KC> kd, vd, vs;
    uint32_t ks;
    int ids = 0;
    auto look_up = [&](int it) {                       // page numbers of this wavefront's tiles in its next 64 steps, one a lane
        const int tile = min(4 * (it + lane) + wave, tlast);
        ids = (int)min((unsigned)tab[tile >> tshift], (unsigned)(pl.n_pages - 1));
    };
    auto request = [&](int it) {                       // past the end: the last tile again, whose weights are zero there
        const int tile = min(4 * it + wave, tlast);
        const unsigned char* p = tile_at<HD>(pl, __builtin_amdgcn_readlane(ids, (it - it0) & 63), kh, tile & ((1 << tshift) - 1));
        kd = load_words<KC>(p + lane * Tile<HD>::LB);
        vd = load_words<KC>(p + Tile<HD>::V + lane * Tile<HD>::LB);
        if constexpr (HD == 128) ks = *reinterpret_cast<const uint32_t*>(p + Tile<HD>::KS + col * 4);
        else if constexpr (HD == 64) ks = *reinterpret_cast<const uint16_t*>(p + Tile<HD>::KS + col * 2);
        else ks = p[Tile<HD>::KS + col];
        vs = load_words<KC>(p + Tile<HD>::VS + g * Tile<HD>::LB);
    };
    // Operands are read from LDS four ahead of their products, in this order; left to itself the compiler reads two of V's, and waits: 1500 rows
    // 38.7 us instead of 35.7, 700 16.9 / 15.1 (32 heads of 128, bf16; of 64 on 8 24.2 / 22.6).  Six ahead: the same; eight do not fit.
    constexpr int AHEAD = 4, NF = 4 * KC;
    auto in_turn = [&]() {
#pragma unroll
        for (int f = AHEAD; f < NF; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x008, TERMS, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, TERMS * AHEAD, 0);
    };
    auto k_at = [&](int f) { return k_sh[f & 3][f >> 2][lane]; };
    auto v_at = [&](int f) { return v_sh[f / (2 * KC)][f / 2 % KC][f & 1][lane]; };
    auto stage = [&](int it) {
        // positions past the end: whatever lies there, V's scale must not make it infinite
        const int ok = min(max(rq.L - ((4 * it + wave) * 16 + 4 * g), 0), 4);
        const uint32_t keep = ok == 4 ? 0xffffffffu : (1u << (8 * ok)) - 1;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            const float f = c == 0 ? scale_of<0>(ks) : c == 1 ? scale_of<1>(ks) : c == 2 ? scale_of<2>(ks) : scale_of<3>(ks);
            k_sh[wave][c][lane] = u32x4{PAGES_CVT(kd.w[c], f, 0), PAGES_CVT(kd.w[c], f, 1), PAGES_CVT(kd.w[c], f, 2), PAGES_CVT(kd.w[c], f, 3)};
        }
#pragma unroll
        for (int j = 0; j < KC; ++j) {
            const uint32_t w = vd.w[j], f = vs.w[j] & keep;
            const uint32_t x0 = PAGES_CVT(w, scale_of<0>(f), 0), x1 = PAGES_CVT(w, scale_of<1>(f), 1), x2 = PAGES_CVT(w, scale_of<2>(f), 2), x3 = PAGES_CVT(w, scale_of<3>(f), 3);
            uint2* even = reinterpret_cast<uint2*>(&v_sh[wave >> 1][j][0][lane]) + (wave & 1);
            uint2* odd = reinterpret_cast<uint2*>(&v_sh[wave >> 1][j][1][lane]) + (wave & 1);
            *even = make_uint2(__builtin_amdgcn_perm(x1, x0, 0x05040100u), __builtin_amdgcn_perm(x3, x2, 0x05040100u));
            *odd = make_uint2(__builtin_amdgcn_perm(x1, x0, 0x07060302u), __builtin_amdgcn_perm(x3, x2, 0x07060302u));
        }
    };
    if (it0 < it1) {
        look_up(it0);
        request(it0);
    }
    for (int it = it0; it < it1; ++it) {
        const int p0 = it * 64;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");            // the readers of the step before are done
        stage(it);
        if (it + 1 < it1) {
            if (((it + 1 - it0) & 63) == 0) look_up(it + 1);
            request(it + 1);
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");            // this step is staged
        if (p0 >= mine) continue;                      // wavefront-uniform: none of its columns sees these
        __builtin_amdgcn_s_setprio(1);
        f32x4 sc[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        u32x4 fr[AHEAD];
#pragma unroll
        for (int f = 0; f < AHEAD; ++f) fr[f] = k_at(f);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const bf16x8 kf = __builtin_bit_cast(bf16x8, fr[f % AHEAD]);
#pragma unroll
            for (int u = TERMS - 1; u >= 0; --u) sc[f & 3] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, __builtin_bit_cast(bf16x8, qf[f >> 2][u]), sc[f & 3], 0, 0, 0);
            if (f + AHEAD < NF) fr[f % AHEAD] = k_at(f + AHEAD);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
        in_turn();
        __builtin_amdgcn_s_setprio(0);
        if (p0 + 63 > all_see) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) sc[t][v] = p0 + t * 16 + g * 4 + v <= lim ? sc[t][v] : -INFINITY;
        }
        float m = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t) m = fmaxf(m, fmaxf(fmaxf(sc[t][0], sc[t][1]), fmaxf(sc[t][2], sc[t][3])));
        m = column_max(m) * a.scale2;
        if (__any(m > mx + 8.f)) {
            const float nm = fmaxf(mx, m), alpha = nm == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mx - nm);
            mx = nm;
            if constexpr (TERMS == 1) total[0] *= alpha; else sum *= alpha;
#pragma unroll
            for (int j = 0; j < KC; ++j) { o[j][0] *= alpha; o[j][1] *= alpha; }
        }
        // V's first operands are on their way while the weights are formed
#pragma unroll
        for (int f = 0; f < AHEAD; ++f) fr[f] = v_at(f);
        __builtin_amdgcn_sched_barrier(0);
        u32x4 pf[2][TERMS];
        const float base = mx == -INFINITY ? 0.f : mx;
        float part = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][v], a.scale2, -base));
                sc[t][v] = e;
                if constexpr (TERMS > 1) part += e;
            }
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                uint32_t w[TERMS];
                terms_of<TERMS>(sc[t][2 * v], sc[t][2 * v + 1], w);
#pragma unroll
                for (int u = 0; u < TERMS; ++u) pf[t >> 1][u][2 * (t & 1) + v] = w[u];
            }
        }
        sum += part;
        __builtin_amdgcn_s_setprio(1);
        if constexpr (TERMS == 1)
#pragma unroll
            for (int s = 0; s < 2; ++s) total = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ONES), __builtin_bit_cast(bf16x8, pf[s][0]), total, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const bf16x8 vf = __builtin_bit_cast(bf16x8, fr[f % AHEAD]);
#pragma unroll
            for (int u = TERMS - 1; u >= 0; --u) o[f / 2 % KC][f & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, pf[f / (2 * KC)][u]), o[f / 2 % KC][f & 1], 0, 0, 0);
            if (f + AHEAD < NF) fr[f % AHEAD] = v_at(f + AHEAD);
        }
        in_turn();
        __builtin_amdgcn_s_setprio(0);
    }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if constexpr (TERMS == 1) sum = total[0];
    if (c >= ncol) return;
    // every lane has eight neighbouring dimensions of its column per chunk: 32 j + 8 g .. + 7
    const int cc = wave * 16 + col;
    float* rec = nrec == 1 ? nullptr : a.rec + (((((size_t)b * pl.KH + kh) * a.ncg + cg) * a.nsp + sp) * GC + cc) * OS;
    const float inv = rec ? 1.f : sum == 0.f ? 0.f : 1.0f / sum;          // a row that sees nothing: zeros
#pragma unroll
    for (int j = 0; j < KC; ++j) {
        const f32x4 x = o[j][0] * inv, y = o[j][1] * inv;
        const f32x4 lo = f32x4{x[0], y[0], x[1], y[1]}, hi = f32x4{x[2], y[2], x[3], y[3]};
        const int d = 32 * j + 8 * g;
        if (rec) {
            *reinterpret_cast<f32x4*>(rec + d) = lo;
            *reinterpret_cast<f32x4*>(rec + d + 4) = hi;
        } else {
            pages_store4<TERMS>(a, rq.row0 + rc, h, HD, d, lo);
            pages_store4<TERMS>(a, rq.row0 + rc, h, HD, d + 4, hi);
        }
    }
    if (rec && g == 0) *reinterpret_cast<float2*>(rec + HD) = make_float2(mx, sum);
}

// Records of a column merged in their order.  HD / 4 lanes per (request, row, head).  Bound by its launch and one round of requests: 3.9 us for 192
// columns of 6 records.   grid ceil(B max_new H / units), block 256
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
