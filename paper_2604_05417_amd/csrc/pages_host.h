// What the paged 4-bit caches (pages.hip) and the contexts (metasd.hip) know of each other: host side.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/metasd.h"

namespace msd {

// Notes the message of a call without a context and returns its code (metasd.hip).
int fail_global(int code, const char* fmt, ...);

// The attention of metasd_attn_pages on fp32 rows, for callers inside the library: split != 0 writes the rows as two bf16 terms (store_terms4,
// lo_off); the launch is planned for what `rec` holds (floats).  Returns hipSuccess or the launch's error.
struct AttnPagesCall {
    const float* q;
    void* out;
    size_t ldq, ldo, lo_off;
    int split, rows, H;
    const int *table, *start, *lens;
    int batch, width, max_new, max_len;
    float scale;
    float* rec;
    size_t rec_floats;
};
hipError_t attn_pages_f32(const metasd_pages& pages, const AttnPagesCall& a, int n_cu, hipStream_t st);

// An empty pool's book: nothing held, every page free.
hipError_t page_book_init(int* table, int batch, int width, int* held, int* ring, int n_pages, int* state, hipStream_t st);

// lens, n_new and their sums of up to METASD_MAX_BATCH requests into device arrays.
struct PageLens { int lens[METASD_MAX_BATCH], n_new[METASD_MAX_BATCH]; };
hipError_t page_lens_set(const PageLens& l, int batch, int* lens, int* n_new, int* total, hipStream_t st);

// x[0 .. n) += the ns - 1 sets of n floats behind it (n % 4 == 0).
hipError_t sum_sets(float* x, int ns, size_t n, hipStream_t st);

}  // namespace msd
