// Host side of the paged 4-bit caches and of the verification against probabilities: the C ABI's checks and launches.
#include "pages_host.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "accept_probs.h"
#include "pages.h"
#include "pages_attn.h"

using namespace msd;

namespace {

// Rows of a call: a launch holds fewer than 2^32 work-items (1024 a row at most), and rows times heads of a group stay within 31 bits.
constexpr int MAX_LAUNCH_ROWS = 1 << 22;

bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }
size_t tile_bytes(int hd) { return (size_t)17 * hd; }
bool shape_ok(int32_t KH, int32_t hd, int32_t page) {
    return KH >= 1 && KH <= 1024 && (hd == 32 || hd == 64 || hd == 128) && page >= 16 && page <= 1024 && (page & (page - 1)) == 0;
}
int shift_of(int page) { return __builtin_ctz((unsigned)page); }

// nullptr, or what is wrong with the pages
const char* check_pages(const metasd_pages* p, bool pool) {
    if (!p) return "NULL pages";
    if (!shape_ok(p->n_kv_heads, p->head_dim, p->page)) return "head_dim 32, 64 or 128, page a power of two from 16 to 1024, n_kv_heads 1..1024";
    if (!pool) return nullptr;
    if (!p->pool || !aligned(p->pool)) return "pool must be 16-byte aligned";
    if (p->n_pages < 1 || (int64_t)p->n_pages * p->page > INT32_MAX) return "n_pages * page must be within 31 bits";
    if (p->page_stride % 16 || p->page_stride < (size_t)p->n_kv_heads * (p->page / 16) * tile_bytes(p->head_dim)) return "page_stride must be a multiple of 16 and hold a page";
    return nullptr;
}
Pool pool_of(const metasd_pages& p) { return Pool{(unsigned char*)p.pool, p.page_stride, p.n_pages, shift_of(p.page), p.n_kv_heads}; }

// CUs of the current device, 0 if it cannot be asked; asked for once per device
int n_cu_of_device() {
    constexpr int MAX_DEV = 64;
    static std::atomic<int> known[MAX_DEV];
    int dev = -1, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 0;
    if (dev < MAX_DEV && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) return 0;
    if (dev < MAX_DEV) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

const char* check_rope(const metasd_rope& r, int hd) {
    if (r.style != METASD_ROPE_HALF && r.style != METASD_ROPE_PAIRS) return "style";
    if (r.rot_dim < 0 || r.rot_dim > hd || r.rot_dim % 2) return "rot_dim must be even and within the head";
    if (r.rot_dim == 0) return nullptr;
    if (!(r.theta > 1.f) || !std::isfinite(r.theta)) return "theta must be above 1";
    if (!std::isfinite(r.gain) || r.gain == 0.f) return "gain";
    if (r.scaling < METASD_ROPE_PLAIN || r.scaling > METASD_ROPE_INDEX) return "scaling";
    if (r.scaling != METASD_ROPE_PLAIN && (!(r.factor >= 0x1p-16f) || !std::isfinite(r.factor))) return "factor must be at least 2^-16";       // angles stay below 2^47
    if (r.scaling >= METASD_ROPE_WAVE && (r.orig_ctx < 1 || !(r.low > 0.f) || !(r.high > r.low) || !std::isfinite(r.high))) return "orig_ctx >= 1 and 0 < low < high";
    return nullptr;
}

// Angle per position of every pair (metasd.h has the formulas).
void rope_table(const metasd_rope& r, RopeTab* t) {
    constexpr double TWO_PI = 6.283185307179586476925;
    const double n = r.rot_dim, theta = r.theta;
    t->style = r.style;
    t->rot = r.rot_dim;
    t->blocks = r.rot_dim % (r.style == METASD_ROPE_HALF ? 16 : 8) == 0;
    t->gain = r.gain;
    // theta^(-2 i / n) as the product of the powers at the bits of i: six calls instead of 64
    double bit[6];
    for (int k = 0; k < 6; ++k) bit[k] = 2 << k < n ? std::pow(theta, -(double)(2 << k) / n) : 1.0;
    double a = 0, b = 0;
    if (r.scaling == METASD_ROPE_INDEX) {
        auto place = [&](double turns) { return n * std::log(r.orig_ctx / (turns * TWO_PI)) / (2.0 * std::log(theta)); };
        a = std::max(0.0, std::floor(place(r.high)));
        b = std::min(n - 1, std::ceil(place(r.low)));
    }
    for (int i = 0; i < r.rot_dim / 2; ++i) {
        double f = 1.0;
        for (int k = 0; k < 6; ++k) if (i >> k & 1) f *= bit[k];
        if (r.scaling == METASD_ROPE_LINEAR) f /= r.factor;
        else if (r.scaling == METASD_ROPE_WAVE) {
            const double turns = r.orig_ctx * f / TWO_PI, keep = std::min(1.0, std::max(0.0, (turns - r.low) / ((double)r.high - r.low)));
            f *= keep + (1.0 - keep) / r.factor;
        } else if (r.scaling == METASD_ROPE_INDEX) {
            const double slow = std::min(1.0, std::max(0.0, (i - a) / std::max(b - a, 0.001)));
            f *= (1.0 - slow) + slow / r.factor;
        }
        t->freq[i] = f;
    }
}

template <typename T>
const char* check_rows(const char* what, const T* p, int64_t ld, int64_t n, size_t elem, const char** msg) {
    if (!aligned(p) || ld < n || (ld * (int64_t)elem) % 16) *msg = what;
    return *msg;
}

template <typename T, int HD>
void launch_rope(const RopeArgs<T>& a, int rows, const RopeTab& rt, const Pool& pl, int n_cu, hipStream_t st) {
    const int units = (a.q ? a.H : 0) + (a.k ? pl.KH : 0);
    constexpr int UN = 256 / (HD / 8);
    const int splits = std::max(1, std::min((units + UN - 1) / UN, 4 * n_cu / rows));      // few rows: the heads of one over several workgroups
    hipLaunchKernelGGL((rope_append_kernel<T, HD>), dim3(rows, splits), dim3(256), 0, st, a, rt, pl);
}

template <int HD, int TERMS>
void launch_attn(const PagesAttn& a, const Pool& pl, const PagesPlan& p, hipStream_t st) {
    const dim3 grid((unsigned)((size_t)a.B * pl.KH * a.nsp * a.ncg)), block(64 * p.nw);
#define GO(CT, PACK, NW) hipLaunchKernelGGL((attn_pages_kernel<HD, CT, TERMS, PACK, NW>), grid, block, 0, st, a, pl)
#define GO1(PACK) if (p.nw == 16) GO(1, PACK, 16); else GO(1, PACK, 4)
    if (p.wide) {
        const dim3 wide((unsigned)(8 * (((size_t)a.B * pl.KH + 7) / 8) * a.nsp * a.ncg));
        hipLaunchKernelGGL((attn_pages_long_kernel<HD, TERMS>), wide, block, 0, st, a, pl);
    } else if (p.ct == 2) GO(2, 1, 4);
    else if (TERMS == 1 || p.pack == 1) { GO1(1); }
    else if constexpr (TERMS > 1) { if (p.pack == 2) { GO1(2); } else { GO1(4); } }
#undef GO1
#undef GO
    if (a.nsp > 1) {
        constexpr int UN = 256 / (HD / 4);
        const size_t units = (size_t)a.B * a.max_new * a.H;
        hipLaunchKernelGGL((pages_merge_kernel<HD, TERMS>), dim3((unsigned)((units + UN - 1) / UN)), dim3(256), 0, st, a, pl, p.cols);
    }
}

// dtype as in metasd_attn_pages
void launch_attn_any(const metasd_pages& pages, int dtype, const PagesAttn& a, const PagesPlan& p, hipStream_t st) {
    const Pool pl = pool_of(pages);
#define GO(HD) if (dtype == METASD_BF16) launch_attn<HD, 1>(a, pl, p, st); else launch_attn<HD, 3>(a, pl, p, st)
    if (pages.head_dim == 128) { GO(128); }
    else if (pages.head_dim == 64) { GO(64); }
    else { GO(32); }
#undef GO
}

// nullptr, or what is wrong with the sizes of an attention call
const char* check_attn(int32_t batch, int32_t n_heads, int32_t KH, int32_t hd, int32_t max_new, int32_t max_len) {
    if (batch < 1 || batch > 65535) return "batch must be 1..65535";
    if (!shape_ok(KH, hd, 16) || n_heads < 1 || n_heads % KH || n_heads / KH > 256) return "n_heads must be a multiple of n_kv_heads (up to 256 times), head_dim 32, 64 or 128";
    if (max_new < 1 || max_new > (1 << 20) || max_len < 1) return "max_new must be 1..2^20, max_len positive";
    // at most 2^23 workgroups of 256 (a launch holds fewer than 2^32 work-items), and 2^26 columns for the merge
    if ((int64_t)batch * KH > (1 << 22) || (int64_t)batch * n_heads * max_new > (1 << 26)) return "too much for one launch: batch * n_kv_heads <= 2^22, batch * n_heads * max_new <= 2^26";
    return nullptr;
}

}  // namespace

namespace msd {

hipError_t attn_pages_f32(const metasd_pages& pages, const AttnPagesCall& c, int n_cu, hipStream_t st) {
    const int KH = pages.n_kv_heads;
    const PagesPlan p = plan_pages(c.batch, KH, c.H / KH, pages.head_dim, c.max_new, c.max_len, 3, n_cu, c.rec_floats);
    if (pages_records(p, c.batch, KH, pages.head_dim) > c.rec_floats) return hipErrorOutOfMemory;      // (one span needs none)
    const PagesAttn a{c.q, c.out, c.ldq, c.ldo, c.lo_off, c.table, c.start, c.lens, c.rec, c.scale * 1.44269504088896341f, c.split, c.batch, c.width, c.rows, c.H, c.H / KH,
                      c.max_new, p.spw, p.nsp, p.ncg};
    launch_attn_any(pages, METASD_F32, a, p, st);
    return hipGetLastError();
}

hipError_t page_book_init(int* table, int batch, int width, int* held, int* ring, int n_pages, int* state, hipStream_t st) {
    hipLaunchKernelGGL(page_book_init_kernel, dim3(1), dim3(1024), 0, st, table, batch * width, held, batch, ring, n_pages, state);
    return hipGetLastError();
}

hipError_t page_lens_set(const PageLens& l, int batch, int* lens, int* n_new, int* total, hipStream_t st) {
    static_assert(METASD_MAX_BATCH <= 64, "one lane per request");
    hipLaunchKernelGGL(page_lens_kernel, dim3(1), dim3(64), 0, st, l, batch, lens, n_new, total);
    return hipGetLastError();
}

hipError_t sum_sets(float* x, int ns, size_t n, hipStream_t st) {
    if (ns <= 1) return hipSuccess;
    hipLaunchKernelGGL(sum_sets_kernel, dim3((unsigned)((n / 4 + 255) / 256)), dim3(256), 0, st, reinterpret_cast<f32x4*>(x), ns, n / 4);
    return hipGetLastError();
}

}  // namespace msd

extern "C" {

int32_t metasd_page_bytes(int32_t n_kv_heads, int32_t head_dim, int32_t page, size_t* bytes_out) {
    if (!bytes_out) return fail_global(METASD_E_INVALID, "page_bytes: NULL pointer");
    if (!shape_ok(n_kv_heads, head_dim, page)) return fail_global(METASD_E_INVALID, "page_bytes: head_dim 32, 64 or 128, page a power of two from 16 to 1024, n_kv_heads 1..1024");
    *bytes_out = (size_t)n_kv_heads * (page / 16) * tile_bytes(head_dim);
    return METASD_OK;
}

int32_t metasd_page_plan(int32_t* table, int32_t batch, int32_t width, int32_t* held, int32_t* ring, int32_t n_pages, int32_t* state, const int32_t* lens,
                         const int32_t* n_new, int32_t page, int32_t rows, int32_t* slots, int32_t* pos, int32_t* start, int32_t* served, void* hip_stream) {
    if (!table || !held || !ring || !state || !lens || !n_new || (rows > 0 && (!slots || !pos)) || !start || !served) return fail_global(METASD_E_INVALID, "page_plan: NULL pointer");
    if (batch < 1 || batch > METASD_PLAN_MAX_BATCH || width < 1 || (int64_t)batch * width > INT32_MAX) return fail_global(METASD_E_INVALID, "page_plan: batch 1..%d, width >= 1, batch * width within 31 bits", METASD_PLAN_MAX_BATCH);
    if (!shape_ok(1, 32, page)) return fail_global(METASD_E_INVALID, "page_plan: page must be a power of two from 16 to 1024");
    if (n_pages < 1 || (int64_t)n_pages * page > INT32_MAX) return fail_global(METASD_E_INVALID, "page_plan: n_pages * page must be within 31 bits");
    if (rows < 0 || rows > (1 << 30)) return fail_global(METASD_E_INVALID, "page_plan: rows must be 0..2^30");
    static_assert(METASD_PLAN_MAX_BATCH == PLAN_BATCH, "requests of a plan");
    const PlanArgs a{table, held, ring, state, lens, n_new, slots, pos, start, served, batch, width, n_pages, shift_of(page), rows};
    hipStream_t st = (hipStream_t)hip_stream;
#define GO(NT) hipLaunchKernelGGL((page_plan_kernel<NT>), dim3(std::max(1, (rows + NT - 1) / NT)), dim3(NT), 0, st, a)
    // A call of few requests and few rows is bound by its barriers: four wavefronts meet sooner than sixteen (32 requests, 256 rows: 4.2 us against
    // 5.6).  Sixteen repeat the scan over the requests for fewer groups of rows (126 000 rows: 8.5 us against 11.4 with four).
    if (batch <= 256 * PLAN_PER && rows <= 1024) GO(256); else GO(1024);
#undef GO
    if (hipGetLastError() != hipSuccess) return fail_global(METASD_E_HIP, "page_plan: launch failed");
    return METASD_OK;
}

int32_t metasd_rope_append(const metasd_rope* rope, const metasd_pages* pages, int32_t dtype, int32_t rows, int32_t n_heads, const void* q, int64_t q_ld,
                           void* q_out, int64_t q_out_ld, const void* k, int64_t k_ld, const void* v, int64_t v_ld, const int32_t* pos, const int32_t* slots,
                           void* hip_stream) {
    if (const char* bad = check_pages(pages, k != nullptr)) return fail_global(METASD_E_INVALID, "rope_append: %s", bad);
    if (!rope || !pos || (!q && !k) || !q != !q_out || !k != !v || (k && !slots)) return fail_global(METASD_E_INVALID, "rope_append: NULL pointer (q and q_out, or k, v and slots, may be NULL together)");
    if (dtype != METASD_F32 && dtype != METASD_BF16) return fail_global(METASD_E_INVALID, "rope_append: dtype");
    if (rows < 1 || rows > MAX_LAUNCH_ROWS || (q && (n_heads < 1 || n_heads > 65535))) return fail_global(METASD_E_INVALID, "rope_append: rows 1..2^22, n_heads 1..65535");
    if (const char* bad = check_rope(*rope, pages->head_dim)) return fail_global(METASD_E_INVALID, "rope_append: %s", bad);
    const int hd = pages->head_dim;
    const size_t es = dtype == METASD_BF16 ? 2 : 4;
    const char* bad = nullptr;
    if (q) { check_rows("q", q, q_ld, (int64_t)n_heads * hd, es, &bad); check_rows("q_out", q_out, q_out_ld, (int64_t)n_heads * hd, es, &bad); }
    if (k) { check_rows("k", k, k_ld, (int64_t)pages->n_kv_heads * hd, es, &bad); check_rows("v", v, v_ld, (int64_t)pages->n_kv_heads * hd, es, &bad); }
    if (q == q_out && q && q_ld != q_out_ld) bad = "q_out";
    if (bad) return fail_global(METASD_E_INVALID, "rope_append: rows of %s must start on 16 bytes and not overlap", bad);
    RopeTab tab{};
    rope_table(*rope, &tab);
    const int n_cu = n_cu_of_device();
    if (!n_cu) return fail_global(METASD_E_HIP, "rope_append: cannot query the device");
    const Pool pl = pool_of(*pages);
    hipStream_t st = (hipStream_t)hip_stream;
#define GO(T)                                                                                                                                                    \
    {                                                                                                                                                            \
        const RopeArgs<T> a{(const T*)q, (const T*)k, (const T*)v, (T*)q_out, (size_t)q_ld, (size_t)k_ld, (size_t)v_ld, (size_t)q_out_ld, pos, slots, n_heads}; \
        if (hd == 128) launch_rope<T, 128>(a, rows, tab, pl, n_cu, st);                                                                                                \
        else if (hd == 64) launch_rope<T, 64>(a, rows, tab, pl, n_cu, st);                                                                                             \
        else launch_rope<T, 32>(a, rows, tab, pl, n_cu, st);                                                                                                           \
    }
    if (dtype == METASD_BF16) GO(bf16_t) else GO(float)
#undef GO
    if (hipGetLastError() != hipSuccess) return fail_global(METASD_E_HIP, "rope_append: launch failed");
    return METASD_OK;
}

int32_t metasd_kv_rows(const metasd_pages* pages, const int32_t* slots, int32_t rows, int32_t dtype, void* k, void* v, void* hip_stream) {
    if (const char* bad = check_pages(pages, true)) return fail_global(METASD_E_INVALID, "kv_rows: %s", bad);
    if (!slots || !k || !v || !aligned(k) || !aligned(v)) return fail_global(METASD_E_INVALID, "kv_rows: NULL pointer, or k, v off 16 bytes");
    if (dtype != METASD_F32 && dtype != METASD_BF16) return fail_global(METASD_E_INVALID, "kv_rows: dtype");
    if (rows < 1 || rows > (1 << 30)) return fail_global(METASD_E_INVALID, "kv_rows: rows must be 1..2^30");
    const Pool pl = pool_of(*pages);
    hipStream_t st = (hipStream_t)hip_stream;
    const size_t n = (size_t)rows * pl.KH * (pages->head_dim / 8);
    const dim3 grid((unsigned)std::min<size_t>((n + 255) / 256, 1 << 20));
#define GO(HD)                                                                                                                          \
    if (dtype == METASD_BF16) hipLaunchKernelGGL((kv_rows_kernel<bf16_t, HD>), grid, dim3(256), 0, st, pl, slots, rows, (bf16_t*)k, (bf16_t*)v); \
    else hipLaunchKernelGGL((kv_rows_kernel<float, HD>), grid, dim3(256), 0, st, pl, slots, rows, (float*)k, (float*)v)
    if (pages->head_dim == 128) { GO(128); }
    else if (pages->head_dim == 64) { GO(64); }
    else { GO(32); }
#undef GO
    if (hipGetLastError() != hipSuccess) return fail_global(METASD_E_HIP, "kv_rows: launch failed");
    return METASD_OK;
}

int32_t metasd_attn_pages_scratch(int32_t batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype, int32_t max_new, int32_t max_len, size_t* bytes_out) {
    if (!bytes_out) return fail_global(METASD_E_INVALID, "attn_pages_scratch: NULL pointer");
    if (const char* bad = check_attn(batch, n_heads, n_kv_heads, head_dim, max_new, max_len)) return fail_global(METASD_E_INVALID, "attn_pages_scratch: %s", bad);
    if (dtype != METASD_F32 && dtype != METASD_BF16) return fail_global(METASD_E_INVALID, "attn_pages_scratch: dtype");
    const int n_cu = n_cu_of_device();
    if (!n_cu) return fail_global(METASD_E_HIP, "attn_pages_scratch: cannot query the device");
    const PagesPlan p = plan_pages(batch, n_kv_heads, n_heads / n_kv_heads, head_dim, max_new, max_len, dtype == METASD_BF16 ? 1 : 3, n_cu);
    *bytes_out = pages_records(p, batch, n_kv_heads, head_dim) * sizeof(float);
    return METASD_OK;
}

int32_t metasd_attn_pages(const metasd_pages* pages, int32_t dtype, int32_t rows, int32_t n_heads, const void* q, int64_t q_ld, void* out, int64_t out_ld,
                          const int32_t* table, int32_t batch, int32_t width, const int32_t* start, const int32_t* lens, int32_t max_new, int32_t max_len,
                          float scale, void* scratch, size_t scratch_bytes, void* hip_stream) {
    if (const char* bad = check_pages(pages, true)) return fail_global(METASD_E_INVALID, "attn_pages: %s", bad);
    if (!q || !out || !table || !start || !lens) return fail_global(METASD_E_INVALID, "attn_pages: NULL pointer");
    if (dtype != METASD_F32 && dtype != METASD_BF16) return fail_global(METASD_E_INVALID, "attn_pages: dtype");
    const int hd = pages->head_dim, KH = pages->n_kv_heads;
    if (const char* bad = check_attn(batch, n_heads, KH, hd, max_new, max_len)) return fail_global(METASD_E_INVALID, "attn_pages: %s", bad);
    if (rows < 1 || rows > MAX_LAUNCH_ROWS || width < 1 || (int64_t)batch * width > INT32_MAX || (int64_t)width * pages->page > INT32_MAX)
        return fail_global(METASD_E_INVALID, "attn_pages: rows 1..2^22, width >= 1, batch * width and width * page within 31 bits");
    if (!(scale > 0.f) || !std::isfinite(scale)) return fail_global(METASD_E_INVALID, "attn_pages: scale must be positive");
    const char* bad = nullptr;
    const size_t es = dtype == METASD_BF16 ? 2 : 4;
    check_rows("q", q, q_ld, (int64_t)n_heads * hd, es, &bad);
    check_rows("out", out, out_ld, (int64_t)n_heads * hd, es, &bad);
    if (q == out) bad = "out (which is q)";
    if (bad) return fail_global(METASD_E_INVALID, "attn_pages: rows of %s must start on 16 bytes and not overlap", bad);
    const int n_cu = n_cu_of_device();
    if (!n_cu) return fail_global(METASD_E_HIP, "attn_pages: cannot query the device");
    const PagesPlan p = plan_pages(batch, KH, n_heads / KH, hd, max_new, max_len, dtype == METASD_BF16 ? 1 : 3, n_cu);
    const size_t need = pages_records(p, batch, KH, hd) * sizeof(float);
    if (need && (!scratch || !aligned(scratch) || scratch_bytes < need)) return fail_global(METASD_E_WORKSPACE, "attn_pages: scratch of %zu bytes, 16-byte aligned, needed (metasd_attn_pages_scratch)", need);
    const PagesAttn a{q, out, (size_t)q_ld, (size_t)out_ld, 0, table, start, lens, (float*)scratch, scale * 1.44269504088896341f, 0, batch, width, rows, n_heads, n_heads / KH,
                      max_new, p.spw, p.nsp, p.ncg};
    launch_attn_any(*pages, dtype, a, p, (hipStream_t)hip_stream);
    if (hipGetLastError() != hipSuccess) return fail_global(METASD_E_HIP, "attn_pages: launch failed");
    return METASD_OK;
}

int32_t metasd_accept_probs(const float* P, int64_t p_row, int64_t p_pos, const float* Q, int64_t q_row, int64_t q_pos, const int32_t* d, const int32_t* n_draft,
                            const float* u, const float* w, int32_t rows, int32_t gamma, int32_t V, int32_t* n_acc, int32_t* tokens, void* hip_stream) {
    if (!P || !d || !u || !w || !n_acc || !tokens) return fail_global(METASD_E_INVALID, "accept_probs: NULL pointer (Q and n_draft may be NULL)");
    if (rows < 1 || rows > MAX_LAUNCH_ROWS / 2 || gamma < 1 || gamma > 1024 || V < 1 || V > METASD_ACCEPT_PROBS_MAX_VOCAB)
        return fail_global(METASD_E_INVALID, "accept_probs: rows 1..2^21, gamma 1..1024, V 1..%d", METASD_ACCEPT_PROBS_MAX_VOCAB);
    if (p_pos < V || (rows > 1 && p_row < V) || (Q && (q_pos < V || (rows > 1 && q_row < V)))) return fail_global(METASD_E_INVALID, "accept_probs: rows of probabilities must not overlap");
    const int vec = aligned(P) && p_row % 4 == 0 && p_pos % 4 == 0 && (!Q || (aligned(Q) && q_row % 4 == 0 && q_pos % 4 == 0));
    const AcceptProbs a{P, Q, (size_t)p_row, (size_t)p_pos, (size_t)q_row, (size_t)q_pos, d, n_draft, u, w, gamma, V, vec, n_acc, tokens};
    hipLaunchKernelGGL(accept_probs_kernel, dim3(rows), dim3(AP_NT), 0, (hipStream_t)hip_stream, a);
    if (hipGetLastError() != hipSuccess) return fail_global(METASD_E_HIP, "accept_probs: launch failed");
    return METASD_OK;
}

}  // extern "C"
