// Kernels of the paged 4-bit caches: block tables and slots, rotation with the append, rows read back.
#pragma once

#include "common.h"
#include "pages_host.h"

namespace msd {

// Layout of a page: [K/V head][page / 16 tiles][17 hd bytes].  A tile is 16 positions of one head: K codes, V codes (8 hd bytes each), K
// scales, V scales (hd / 2 each), ordered so that a wavefront's loads are the operands of its MFMAs (pages_attn.h):
//   K codes  [(d % 32) / 8][p][d / 32][(d % 8) / 2]     lane 16 g + p holds the dimensions 32 c + 8 g .. + 7 of position p, 4 bytes per c
//   V codes  [p / 4][(d % 32) / 2][d / 32][p % 4]       lane 16 g + i holds the dimensions 32 j + 2 i, + 1 of the positions 4 g .. 4 g + 3
//   K scales [p][d / 32]      V scales [p / 4][d / 32][p % 4]
// A byte holds the dimensions (d, d + 1), the even one in its low half.
template <int HD>
struct Tile {
    static constexpr int BYTES = 17 * HD, V = 8 * HD, KS = 16 * HD, VS = 16 * HD + HD / 2;
    static constexpr int LB = HD / 8;                  // code bytes of a lane per tile, and the stride of its V scales
    static __device__ __forceinline__ int kcode(int p, int d) { return ((d & 31) / 8 * 16 + p) * LB + d / 32 * 4 + (d & 7) / 2; }
    static __device__ __forceinline__ int vcode(int p, int d) { return V + (p / 4 * 16 + (d & 31) / 2) * LB + d / 32 * 4 + (p & 3); }
    static __device__ __forceinline__ int kscale(int p, int c) { return KS + p * (HD / 32) + c; }
    static __device__ __forceinline__ int vscale(int p, int c) { return VS + p / 4 * LB + c * 4 + (p & 3); }
};

struct Pool {
    unsigned char* base;
    size_t stride;           // bytes between pages
    int n_pages, shift, KH;  // page = 1 << shift positions
};
template <int HD>
__device__ __forceinline__ unsigned char* tile_at(const Pool& pl, int page, int head, int in_page) {
    return pl.base + (size_t)page * pl.stride + ((size_t)head << (pl.shift - 4)) * Tile<HD>::BYTES + (size_t)in_page * Tile<HD>::BYTES;
}

// ------------------------------------------------------------------------------------------
// Block tables and slots.  A workgroup does everything for a row per thread: every workgroup sums the requests' rows and pages for itself (at
// most PLAN_BATCH of them, 20 bytes each, from L2), so that nothing has to be handed from one to another; the pages that change hands are
// dealt out over all of them.  Pages are taken from the front of the ring and given back behind its last, two stretches that do not meet
// because the ring has room for every page there is.  The counts of the state and of the requests are read by all and written by the
// workgroup that comes to its end last.  Bound by the chain of requests, three sums and their barriers, a search and a page number: 4.2 us for 32
// requests and 256 rows, 8.5 for 300 and 126 000 (1.2 MB, under 1 us of HBM).
constexpr int PLAN_BATCH = 4096, PLAN_PER = 4;      // requests of a call, and of a thread

struct PlanArgs {
    int *table, *held, *ring, *state;
    const int *lens, *n_new;
    int *slots, *pos, *start, *served;
    int B, width, n_pages, shift, rows;
};

// Inclusive sum over the workgroup of one value per thread; *total: of all.
template <int NT, typename T>
__device__ __forceinline__ T block_scan(T v, T* wave_tot, T* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T y = __shfl_up(v, o, 64);
        if (lane >= o) v += y;
    }
    __syncthreads();                                   // the sums of a scan before have been read
    if (lane == 63) wave_tot[wave] = v;
    __syncthreads();
    T before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        const T x = wave_tot[w];
        before += w < wave ? x : (T)0;
        all += x;
    }
    *total = all;
    return v + before;
}

// first i with end[i] > x (end is not decreasing)
__device__ __forceinline__ int first_above(const int* end, int n, int x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (end[mid] > x) hi = mid; else lo = mid + 1;
    }
    return lo;
}

template <int NT>
__global__ __launch_bounds__(NT) void page_plan_kernel(PlanArgs a) {
    __shared__ int row_end[NT * PLAN_PER], take_end[NT * PLAN_PER], back_end[NT * PLAN_PER];
    __shared__ long long tot64[NT / 64];
    __shared__ int tot32[NT / 64];
    __shared__ int last;
    const int tid = threadIdx.x, per = (a.B + NT - 1) / NT, b0 = tid * per;
    const int page = 1 << a.shift;
    int head = a.state[0] % a.n_pages, count = min(max(a.state[1], 0), a.n_pages);
    if (head < 0) head += a.n_pages;
    int need[PLAN_PER], had[PLAN_PER], take[PLAN_PER], back[PLAN_PER];
    long long end[PLAN_PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        if (i >= per) break;
        const int b = b0 + i;
        const bool on = b < a.B;
        const int len = on ? max(a.lens[b], 0) : 0, n = on ? max(a.n_new[b], 0) : 0;
        had[i] = on ? min(max(a.held[b], 0), a.width) : 0;
        need[i] = (int)(((long long)len + n + page - 1) >> a.shift);
        sum += n;
        end[i] = sum;
    }
    long long all64;
    const long long rows_before = block_scan<NT>(sum, tot64, &all64) - sum;
    int t = 0, r = 0;
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        if (i >= per) break;
        end[i] += rows_before;
        const bool fits = need[i] <= a.width && end[i] <= a.rows;
        take[i] = fits ? max(need[i] - had[i], 0) : 0;
        back[i] = max(had[i] - need[i], 0);
        t += take[i];
        r += back[i];
        need[i] = fits ? need[i] : -need[i] - 1;       // (marked: not served whatever the ring holds)
    }
    int all_t, all_r;
    int upto_t = block_scan<NT>(t, tot32, &all_t) - t, upto_r = block_scan<NT>(r, tot32, &all_r) - r;
    int new_held[PLAN_PER], served_to = 0;
    __shared__ int taken_wave[NT / 64];
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        if (i >= per) break;
        const int b = b0 + i;
        upto_t += take[i];
        upto_r += back[i];
        const bool fits = need[i] >= 0, ok = fits && (take[i] == 0 || upto_t <= count);
        const int nd = fits ? need[i] : -need[i] - 1;
        new_held[i] = ok ? nd : min(nd, had[i]);
        if (take[i] > 0 && ok) served_to = upto_t;
        if (b < a.B) {
            row_end[b] = (int)min(end[i], (long long)INT32_MAX);
            take_end[b] = ok ? upto_t : -upto_t - 1;   // (marked: its rows get no slots)
            back_end[b] = upto_r;
        }
    }
    // pages taken: those who are served and take any come first, so the largest sum among them
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) served_to = max(served_to, __shfl_xor(served_to, o, 64));
    if ((tid & 63) == 0) taken_wave[tid >> 6] = served_to;
    __syncthreads();
    int taken = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) taken = max(taken, taken_wave[w]);
    auto upto = [&](int b) { const int x = take_end[b]; return x < 0 ? -x - 1 : x; };
    // ---- rows
    const int r0 = blockIdx.x * NT + tid;
    if (r0 < a.rows) {
        int slot = -1, p = -1;
        const int b = first_above(row_end, a.B, r0);
        if (b < a.B) {
            p = max(a.lens[b], 0) + r0 - (b ? row_end[b - 1] : 0);
            if (take_end[b] >= 0) {
                const int j = p >> a.shift, h = min(max(a.held[b], 0), a.width);
                int id;
                if (j < h) id = a.table[(size_t)b * a.width + j];
                else {
                    const int nd = (int)(((long long)max(a.lens[b], 0) + max(a.n_new[b], 0) + page - 1) >> a.shift);
                    id = a.ring[(int)(((long long)head + take_end[b] - (nd - h) + (j - h)) % a.n_pages)];
                }
                slot = id * page + (p & (page - 1));
            }
        }
        a.slots[r0] = slot;
        a.pos[r0] = p;
    }
    // ---- pages that change hands
    const int grid = gridDim.x * NT;
    for (int i = r0; i < taken; i += grid) {
        int lo = 0, hi = a.B;
        while (lo < hi) { const int mid = (lo + hi) >> 1; if (upto(mid) > i) hi = mid; else lo = mid + 1; }
        const int h = min(max(a.held[lo], 0), a.width), before = lo ? upto(lo - 1) : 0;
        a.table[(size_t)lo * a.width + h + (i - before)] = a.ring[(int)(((long long)head + i) % a.n_pages)];
    }
    for (int i = r0; i < all_r; i += grid) {
        const int b = first_above(back_end, a.B, i), before = b ? back_end[b - 1] : 0;
        const int nd = (int)(((long long)max(a.lens[b], 0) + max(a.n_new[b], 0) + page - 1) >> a.shift);
        a.ring[(int)(((long long)head + count + i) % a.n_pages)] = a.table[(size_t)b * a.width + nd + (i - before)];
    }
    if (blockIdx.x == 0)
        for (int b = tid; b <= a.B; b += NT) {
            a.start[b] = b ? row_end[b - 1] : 0;
            if (b < a.B) a.served[b] = take_end[b] >= 0;
        }
    // ---- the counts, once nobody reads them any more: a workgroup's reads are done when its ticket goes out, because what they returned has
    // been used, so the order of the tickets needs no fence
    __syncthreads();
    if (tid == 0) last = gridDim.x == 1 || __hip_atomic_fetch_add(a.state + 2, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        if (i >= per) break;
        if (b0 + i < a.B) a.held[b0 + i] = new_held[i];
    }
    if (tid == 0) {
        a.state[0] = (int)(((long long)head + taken) % a.n_pages);
        a.state[1] = min(count - taken + all_r, a.n_pages);
        a.state[2] = 0;
    }
}

// grid 1, block 1024
__global__ void page_book_init_kernel(int* __restrict__ table, int entries, int* __restrict__ held, int batch, int* __restrict__ ring, int n_pages, int* __restrict__ state) {
    for (int i = threadIdx.x; i < entries; i += blockDim.x) table[i] = 0;
    for (int i = threadIdx.x; i < batch; i += blockDim.x) held[i] = 0;
    for (int i = threadIdx.x; i < n_pages; i += blockDim.x) ring[i] = i;
    if (threadIdx.x < 4) state[threadIdx.x] = threadIdx.x == 1 ? n_pages : 0;
}
// grid 1, block 64
__global__ void page_lens_kernel(PageLens l, int batch, int* __restrict__ lens, int* __restrict__ n_new, int* __restrict__ total) {
    const int b = threadIdx.x;
    if (b < batch) { lens[b] = l.lens[b]; n_new[b] = l.n_new[b]; total[b] = l.lens[b] + l.n_new[b]; }
}
// grid ceil(n4 / 256), block 256
__global__ void sum_sets_kernel(f32x4* x, int ns, size_t n4) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n4) return;
    f32x4 y = x[i];
    for (int s = 1; s < ns; ++s) y += x[(size_t)s * n4 + i];
    x[i] = y;
}

// ------------------------------------------------------------------------------------------
// Rotation and append.  Angles are formed in 64 bits (a position times a frequency loses nothing that matters at any position), their
// sines and cosines rounded to 32 bits, and every product and sum of the rotation rounded on its own, so that the rotated values - and
// with them the 4-bit codes - do not hang on how a compiler contracts them.
constexpr int ROPE_MAX_PAIRS = 64;
struct RopeTab {
    int style, rot;          // rot: components that are rotated, 0: none
    int blocks;              // the rotated components and their partners are whole blocks of eight
    float gain;
    double freq[ROPE_MAX_PAIRS];
};

// The largest magnitude of a block of 32 as its bits (non-finite: 0x7f800000 and more) -> the byte e + 127 of its scale: the smallest e with
// amax <= 7 * 2^e, so that saturating at 6 costs no more than a rounding there.
__device__ __forceinline__ int scale_byte(uint32_t amax) {
    const int e = (int)(amax >> 23) - 127 - 2 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return min(max(e, -125), 125) + 127;
}
// eight values -> their codes, ties to even
__device__ __forceinline__ uint32_t codes8(const float* x, float scale) {
    uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* x) {
    if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* x) {
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        *reinterpret_cast<uint4*>(p) = make_uint4(f2bf2(x[0], x[1]), f2bf2(x[2], x[3]), f2bf2(x[4], x[5]), f2bf2(x[6], x[7]));
    }
}

template <typename T>
struct RopeArgs {
    const T *q, *k, *v;
    T* q_out;
    size_t ldq, ldk, ldv, ldo;
    const int *pos, *slots;
    int H;
};

// gain * (cos a, sin a) of an angle of up to 2^31 periods, off by some 1e-15 before it is rounded: a less the nearest multiple of pi / 2, taken
// off in two parts of it, then the Taylor series up to the 14th power (0.79^15 / 15! = 2e-14).
__device__ __forceinline__ float2 turn_of(double a, double gain) {
    const double n = rint(a * 0.63661977236758134308);
    double r = fma(-n, 1.57079632679489661923, a);
    r = fma(-n, 6.12323399573676588614e-17, r);
    const double z = r * r;
    double s = 1.0 / 6227020800.0;
    s = fma(s, z, -1.0 / 39916800.0);
    s = fma(s, z, 1.0 / 362880.0);
    s = fma(s, z, -1.0 / 5040.0);
    s = fma(s, z, 1.0 / 120.0);
    s = fma(s, z, -1.0 / 6.0);
    s = fma(s * z, r, r);
    double c = -1.0 / 87178291200.0;
    c = fma(c, z, 1.0 / 479001600.0);
    c = fma(c, z, -1.0 / 3628800.0);
    c = fma(c, z, 1.0 / 40320.0);
    c = fma(c, z, -1.0 / 720.0);
    c = fma(c, z, 1.0 / 24.0);
    c = fma(c, z, -0.5);
    c = fma(c, z, 1.0);
    const int q = (int)(n - 4.0 * floor(n * 0.25));
    const double x = q & 1 ? s : c, y = q & 1 ? c : s;
    return make_float2((float)((q + 1) & 2 ? -x * gain : x * gain), (float)(q & 2 ? -y * gain : y * gain));
}

// A workgroup takes a row and every gridDim.y-th of its heads, HD / 8 lanes a head, eight components each (a head's lanes are in one
// wavefront).  Units 0 .. H - 1 are query heads, H .. H + KH - 1 K/V heads.
// What bounds it: HBM, for few rows the chain position - angle - rows.  1999 rows of 32 + 32 heads of 128 in bf16 (74 MB): 19.5 - 20.3 us, of which 6
// for the 8.7 MB of codes, whose 16-byte pieces share cache lines with those of the next positions; 16 rows a workgroup, which brings
// such lines together in one L2, 21.4 us.   grid (rows, splits), block 256
template <typename T, int HD>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeArgs<T> a, RopeTab rt, Pool pl) {
#pragma clang fp contract(off)
    constexpr int LN = HD / 8, UN = 256 / LN;         // lanes of a unit, units at a time
    __shared__ __align__(16) float2 turn[ROPE_MAX_PAIRS];
    __shared__ __align__(16) float xs[UN][HD + 4];
    const int tid = threadIdx.x, half = rt.rot >> 1, row = blockIdx.x;
    if (tid < half) turn[tid] = turn_of((double)a.pos[row] * rt.freq[tid], (double)rt.gain);
    __syncthreads();
    const int u = tid / LN, l = tid % LN, d0 = l * 8;
    const int HQ = a.q ? a.H : 0, NU = HQ + (a.k ? pl.KH : 0);
    float* x = xs[u];
    // y: this lane's eight components, in and out.  A unit's lanes are in one wavefront, whose LDS accesses are carried out in order.
    auto rotate = [&](float* y) {
        if (rt.blocks) {
            if (d0 >= rt.rot) return;                  // these lanes' partners are at or beyond rt.rot too
            if (rt.style == 0) {
                __builtin_amdgcn_wave_barrier();
                store8(x + d0, y);
                __builtin_amdgcn_wave_barrier();
                const bool first = d0 < half;
                const int j0 = first ? d0 : d0 - half;
                float o[8], cs[16];
                load8(x + (first ? d0 + half : j0), o);
                load8(reinterpret_cast<const float*>(turn + j0), cs);
                load8(reinterpret_cast<const float*>(turn + j0 + 4), cs + 8);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p1 = y[i] * cs[2 * i], p2 = o[i] * cs[2 * i + 1];
                    y[i] = first ? p1 - p2 : p1 + p2;
                }
            } else {
                float cs[8];
                load8(reinterpret_cast<const float*>(turn + d0 / 2), cs);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a1 = y[2 * i] * cs[2 * i], b1 = y[2 * i + 1] * cs[2 * i + 1], a2 = y[2 * i + 1] * cs[2 * i], b2 = y[2 * i] * cs[2 * i + 1];
                    y[2 * i] = a1 - b1;
                    y[2 * i + 1] = a2 + b2;
                }
            }
            return;
        }
        __builtin_amdgcn_wave_barrier();
        store8(x + d0, y);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int d = d0 + i;
            if (d >= rt.rot) break;
            const bool first = rt.style == 0 ? d < half : (d & 1) == 0;
            const int j = rt.style == 0 ? (first ? d : d - half) : d >> 1;
            const float other = x[rt.style == 0 ? (first ? d + half : d - half) : d ^ 1];
            const float2 cs = turn[j];
            const float p1 = y[i] * cs.x, p2 = other * cs.y;
            y[i] = first ? p1 - p2 : p1 + p2;
        }
    };
    for (int i0 = blockIdx.y * UN; i0 < NU; i0 += gridDim.y * UN) {
        const int h = min(i0 + u, NU - 1);
        const bool on = i0 + u < NU;
        float y[8];
        if (h < HQ) {
            load8(a.q + (size_t)row * a.ldq + (size_t)h * HD + d0, y);
            rotate(y);
            if (on) store8(a.q_out + (size_t)row * a.ldo + (size_t)h * HD + d0, y);
        } else {
            const int kh = h - HQ, slot = a.slots[row];
            float z[8];
            load8(a.k + (size_t)row * a.ldk + (size_t)kh * HD + d0, y);
            load8(a.v + (size_t)row * a.ldv + (size_t)kh * HD + d0, z);
            rotate(y);
            uint32_t ka = 0, va = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ka = max(ka, __float_as_uint(y[e]) & 0x7fffffffu);
                va = max(va, __float_as_uint(z[e]) & 0x7fffffffu);
            }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) { ka = max(ka, (uint32_t)__shfl_xor((int)ka, o, 64)); va = max(va, (uint32_t)__shfl_xor((int)va, o, 64)); }
            uint32_t worst = max(ka, va);
#pragma unroll
            for (int o = 4; o < LN; o <<= 1) worst = max(worst, (uint32_t)__shfl_xor((int)worst, o, 64));
            if (on && slot >= 0 && (slot >> pl.shift) < pl.n_pages) {
                int kb = scale_byte(ka), vb = scale_byte(va);
                uint32_t kc = codes8(y, __uint_as_float((uint32_t)kb << 23)), vc = codes8(z, __uint_as_float((uint32_t)vb << 23));
                if (worst >= 0x7f800000u) { kc = vc = 0; kb = 255; vb = 2; }       // not finite: marked in K's scales, V holds zeros
                unsigned char* t = tile_at<HD>(pl, slot >> pl.shift, kh, (slot & ((1 << pl.shift) - 1)) >> 4);
                const int p = slot & 15, c = d0 / 32;
                *reinterpret_cast<uint32_t*>(t + Tile<HD>::kcode(p, d0)) = kc;
#pragma unroll
                for (int e = 0; e < 4; ++e) t[Tile<HD>::vcode(p, d0 + 2 * e)] = (unsigned char)(vc >> (8 * e));
                if ((l & 3) == 0) { t[Tile<HD>::kscale(p, c)] = (unsigned char)kb; t[Tile<HD>::vscale(p, c)] = (unsigned char)vb; }
            }
        }
    }
}

// Rows read back: the values that the codes stand for; rows without a slot are zeros.  Bound by HBM and two rounds of its chain slot - codes -
// rows: 1999 rows of 32 heads of 128 in bf16 (41 MB) 12 us, 3.4 TB/s.
//  grid-stride over (row, head, 8 components), block 256
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv_rows_kernel(Pool pl, const int* __restrict__ slots, int rows, T* __restrict__ k, T* __restrict__ v) {
    constexpr int LN = HD / 8;
    const size_t n = (size_t)rows * pl.KH * LN;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
        const int l = (int)(i % LN), kh = (int)(i / LN % pl.KH), row = (int)(i / LN / pl.KH), slot = slots[row], d0 = l * 8;
        float y[8] = {}, z[8] = {};
        if (slot >= 0 && (slot >> pl.shift) < pl.n_pages) {
            const unsigned char* t = tile_at<HD>(pl, slot >> pl.shift, kh, (slot & ((1 << pl.shift) - 1)) >> 4);
            const int p = slot & 15, c = d0 / 32;
            const int kb = t[Tile<HD>::kscale(p, c)];
            const float ks = __uint_as_float((uint32_t)kb << 23), vs = __uint_as_float((uint32_t)(kb == 255 ? 255 : t[Tile<HD>::vscale(p, c)]) << 23);
            const uint32_t kc = *reinterpret_cast<const uint32_t*>(t + Tile<HD>::kcode(p, d0));
            uint32_t vc = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) vc |= (uint32_t)t[Tile<HD>::vcode(p, d0 + 2 * e)] << (8 * e);
#define PAIR(E)                                                                                                                          \
    {                                                                                                                                    \
        const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kc, ks, E));                           \
        const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vc, vs, E));                           \
        y[2 * E] = __uint_as_float(a << 16); y[2 * E + 1] = __uint_as_float(a & 0xffff0000u);                                            \
        z[2 * E] = __uint_as_float(b << 16); z[2 * E + 1] = __uint_as_float(b & 0xffff0000u);                                            \
    }
            PAIR(0) PAIR(1) PAIR(2) PAIR(3)
#undef PAIR
        }
        store8(k + i * 8, y);
        store8(v + i * 8, z);
    }
}

}  // namespace msd
