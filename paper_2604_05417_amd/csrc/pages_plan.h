// How the attention over 4-bit pages (pages_attn.h) is split over workgroups.  Host code that needs nothing of HIP.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace msd {

constexpr int PA_NW = 4;       // wavefronts of a workgroup; each takes every fourth sub-block of 32 positions of its span

struct PagesPlan {
    int ct;        // tiles of 16 columns (row, query head of a K/V head) that a workgroup carries through its span
    int ncg;       // groups of 16 ct columns that a request can have
    int spw, nsp;  // sub-blocks of a span, spans of the longest context
};

// B requests of at most max_new rows and max_len positions, G query heads per K/V head.
inline PagesPlan plan_pages(int B, int KH, int G, int max_new, int max_len, int terms, int n_cu) {
    PagesPlan p{};
    const long cols = (long)max_new * G;
    p.ct = cols <= 16 ? 1 : cols <= 32 || terms == 2 ? 2 : 4;
    p.ncg = (int)((cols + 16 * p.ct - 1) / (16 * p.ct));
    const int nsub = std::max(1, (max_len + 31) / 32);
    const long wgs = (long)B * KH * p.ncg;
    int want = (int)std::max(1L, std::min(16L, (2L * n_cu + wgs - 1) / wgs));     // spans per context that fill the chip
    if (wgs >= n_cu) want = 1;
    want = std::min(want, std::max(1, nsub / PA_NW));
    p.spw = PA_NW * ((nsub + PA_NW * want - 1) / (PA_NW * want));
    p.nsp = (nsub + p.spw - 1) / p.spw;
    return p;
}

// floats of the records: (O, maximum, sum) of every column and span, where there is more than one
inline size_t pages_records(const PagesPlan& p, int B, int KH, int hd) {
    return p.nsp == 1 ? 0 : (size_t)B * KH * p.ncg * p.nsp * 16 * p.ct * (hd + 4);
}

}  // namespace msd
