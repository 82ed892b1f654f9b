// How the attention over 4-bit pages (pages_attn.h) is split over workgroups.  Host code that needs nothing of HIP.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace msd {

// Columns from which on a block takes the long form.  Without / with it, bf16 (fp32) rows: 1500 rows of 32 heads of 128 50.9 / 39 us (78.1 / 60), 700 29.1
// / 17.4 (36.3 / 27.6), of 32 heads of 64 on 8 30.7 / 24.4 (48.6 / 41); 200 rows 10.8 / 11.8 (10.9 / 12.0); 128 behind 1872 positions 24.5 / 25.3 (27 / 31.8).
constexpr int PAGES_WIDE = 256;

struct PagesPlan {
    bool wide;     // long blocks: the wavefronts of a workgroup have columns of their own and share the positions (attn_pages_long_kernel)
    int ct, pack;  // tiles of 16 columns that a workgroup carries through its span, and columns that a (row, query head) pair takes in a tile
    int cols;      // .. so many pairs in all
    int nw;        // wavefronts of a workgroup, 4 or 16; each takes every nw-th sub-block of 32 positions of its span
    int ncg;       // groups of `cols` pairs that a request can have
    int spw, nsp;  // sub-blocks of a span, spans of the longest context
};

// B requests of at most max_new rows and max_len positions, G query heads per K/V head.
//   pack: fp32 rows, whose q and weights are three bf16 terms, take three products per operand of K and V; where at most 4 (8) pairs
// share them, the terms of a pair lie in different columns of the same product instead, which leaves one (two).
//   nw: one workgroup of 16 wavefronts per (request, K/V head) needs no records and no second launch, but leaves the other CUs idle.  An
// iteration of its 512 positions takes 1.75 (head_dim 128; 64: 1.15) us with bf16 rows and 2.4 (1.7) with fp32 ones; the records, their merge
// and its launch cost some 6.5.  Measured, alone / split: 32 heads of 128, 6 rows behind 1000 positions, fp32 11.6 / 15.0 us, 2000 16.9 / 14.8, bf16
// 12.7 / 15.1, 4000 20.5 / 14.9; 192 heads of 64, bf16 rows behind 4000 16.5 / 20.0, fp32 behind 16000 66.5 / 61.2.
// limit: floats of records that there is room for.
inline size_t pages_records(const PagesPlan& p, int B, int KH, int hd);
inline PagesPlan plan_pages(int B, int KH, int G, int hd, int max_new, int max_len, int terms, int n_cu, size_t limit = SIZE_MAX) {
    PagesPlan p{};
    const long cols = (long)max_new * G;
    p.ct = cols <= 16 ? 1 : 2;
    p.pack = terms == 1 || cols > 8 ? 1 : cols > 4 ? 2 : 4;
    p.cols = 16 * p.ct / p.pack;
    p.ncg = (int)((cols + p.cols - 1) / p.cols);
    const int nsub = (std::max(1, max_len) - 1) / 32 + 1;
    p.wide = cols >= PAGES_WIDE;
    if (p.wide) {
        p.ct = 1;
        p.cols = 64;
        p.nw = 4;
        p.ncg = (int)((cols + p.cols - 1) / p.cols);
        const long wgs = (long)B * KH * p.ncg;
        int want = (int)std::max(1L, std::min(16L, 2L * n_cu / wgs));
        want = std::min(want, std::max(1, nsub / 8));
        for (;; want /= 2) {
            p.spw = 2 * ((nsub + 2 * want - 1) / (2 * want));
            p.nsp = (nsub + p.spw - 1) / p.spw;
            if (want == 1 || pages_records(p, B, KH, hd) <= limit) return p;
        }
    }
    const long wgs = (long)B * KH * p.ncg;
    const double alone = (nsub + 15) / 16 * (hd == 128 ? (terms == 1 ? 1.75 : 2.4) : (terms == 1 ? 1.15 : 1.7));
    p.nw = p.ct == 1 && wgs <= n_cu && alone * (1.0 - (double)wgs / n_cu) <= 6.5 ? 16 : 4;
    int want = p.nw == 16 ? 1 : (int)std::max(1L, std::min(32L, (4L * n_cu + wgs - 1) / wgs));     // spans per context that fill the chip
    want = std::min(want, std::max(1, nsub / (2 * p.nw)));
    for (;; want /= 2) {
        p.spw = p.nw * ((nsub + p.nw * want - 1) / (p.nw * want));
        p.nsp = (nsub + p.spw - 1) / p.spw;
        if (want == 1 || pages_records(p, B, KH, hd) <= limit) return p;
    }
}

// floats of the records: (O, maximum, sum) of every column and span, where there is more than one
inline size_t pages_records(const PagesPlan& p, int B, int KH, int hd) {
    return p.nsp == 1 ? 0 : (size_t)B * KH * p.ncg * p.nsp * p.cols * (hd + 4);
}

}  // namespace msd
