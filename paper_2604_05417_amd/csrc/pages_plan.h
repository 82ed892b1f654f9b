// How the attention over 4-bit pages (pages_attn.h) is split over workgroups.  Host code that needs nothing of HIP.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace msd {

constexpr int PA_NW = 4;       // wavefronts of a workgroup; each takes every fourth sub-block of 32 positions of its span

struct PagesPlan {
    int ct, pack;  // tiles of 16 columns that a workgroup carries through its span, and columns that a (row, query head) pair takes in a tile
    int cols;      // .. so many pairs in all
    int ncg;       // groups of `cols` pairs that a request can have
    int spw, nsp;  // sub-blocks of a span, spans of the longest context
};

// B requests of at most max_new rows and max_len positions, G query heads per K/V head.
//   pack: fp32 rows, whose q and weights are three bf16 terms, take three products per operand of K and V; where at most 4 (8) pairs
// share them, the terms of a pair lie in different columns of the same product instead, which leaves one (two).
inline PagesPlan plan_pages(int B, int KH, int G, int max_new, int max_len, int terms, int n_cu) {
    PagesPlan p{};
    const long cols = (long)max_new * G;
    p.ct = cols <= 16 ? 1 : 2;
    p.pack = terms == 1 || cols > 8 ? 1 : cols > 4 ? 2 : 4;
    p.cols = 16 * p.ct / p.pack;
    p.ncg = (int)((cols + p.cols - 1) / p.cols);
    const int nsub = std::max(1, (max_len + 31) / 32);
    const long wgs = (long)B * KH * p.ncg;
    int want = (int)std::max(1L, std::min(32L, (4L * n_cu + wgs - 1) / wgs));     // spans per context that fill the chip
    want = std::min(want, std::max(1, nsub / (2 * PA_NW)));
    p.spw = PA_NW * ((nsub + PA_NW * want - 1) / (PA_NW * want));
    p.nsp = (nsub + p.spw - 1) / p.spw;
    return p;
}

// floats of the records: (O, maximum, sum) of every column and span, where there is more than one
inline size_t pages_records(const PagesPlan& p, int B, int KH, int hd) {
    return p.nsp == 1 ? 0 : (size_t)B * KH * p.ncg * p.nsp * p.cols * (hd + 4);
}

}  // namespace msd
