// Group norm with an activation, channels last (int8 and bf16), for gfx950.
//
// Per sample b and group g of cpg = C / G channels, n = pixels * cpg values:
//   bf16  y = act(weight_c (x - mean) / sqrt(var + eps) + bias_c + res), one rounding at the end
//   int8  S1 = sum x, S2 = sum x^2 (exact integers), d = n x - S1, m_c = weight_c 2^f / (n sqrt((n S2 - S1^2) / n^2 + eps)),
//         y = clamp(floor(d m_c + (bias_c 2^f + 1/2) + res 2^rs), lo, hi) in 64-bit floats: d is exact, so a constant group gives its bias on
//         every machine and the results are whole numbers that do not depend on the order of a sum; every operation is rounded by itself
// Statistics of bf16: every lane adds up the differences of at most 64 of its values from one that is near them, and their squares, has from those their mean and sum of squared differences from it, and
// such pairs are merged
// (n = na + nb, delta = mb - ma: mean = ma + delta nb / n, M2 = M2a + M2b + delta^2 na nb / n), so that a mean far from zero costs nothing.
//
// Bound by memory.  A workgroup has a window of whole groups (columns of 16 bytes, a power of two of them) and some pixels of one sample; a lane has one
// column and every NT / columns-th pixel.  Where the window of a whole sample fits a workgroup's registers it is one launch that reads x once; else two:
// statistics of chunks of pixels, then every workgroup of the second launch merges the chunks of its sample and writes its part (x is read again).
// int8 results: in float arithmetic, and again in 64 bits where that is too near to a whole number to say on which side (about one vector of 16 in a thousand).
#include <algorithm>
#include <type_traits>

#include "../ee_internal.hpp"
#include "../igemm_device.hpp"

namespace ee {
namespace {

struct NormKernelArgs {
    const void* x; const void* res; void* y;
    const float* weight; const float* bias;
    void* part;                      // two launches: [sample][chunk][group] pairs
    int64_t x_sample, x_pixel, r_sample, r_pixel, y_sample, y_pixel;      // strides in elements
    int pixels, c, groups, cpg;
    int cw, wlog;                    // channels of a window (whole groups), log2 of its columns (idle ones included)
    int windows, chunks, chunk_pixels, units;                             // units: workgroups with work
    float eps;
    double out_scale, res_scale;     // int8: 2^frac_bits, 2^res_shift
    int act, lo, hi;
};

// what a lane knows of a part of a group: n values, their mean and the sum of squared differences from it
struct Moments { float n, mean, m2; };
// a part without values changes nothing and one that joins it is taken as it is: w is 1 there but for the rounding of the reciprocal, which gave a constant group of 1003 a variance and results of 0.02,
// and the square of a mean of 2e19 is infinite
__device__ __forceinline__ void merge(Moments& a, float nb, float mb, float m2b)
{
    const float n = a.n + nb, w = nb * __builtin_amdgcn_rcpf(fmaxf(n, 1.f)), d = a.n > 0.f && nb > 0.f ? mb - a.mean : 0.f;
    a.mean = a.n > 0.f ? fmaf(d, w, a.mean) : mb;
    a.m2 += fmaf(d * d, a.n * w, m2b);
    a.n = n;
}
// int8: the sum and the sum of squares
struct Sums { int s1; long long s2; };

template <int ES> struct elem;
template <> struct elem<1> { typedef int8_t type; };
template <> struct elem<2> { typedef uint16_t type; };

template <int ES, int VEC>
struct Pack {       // VEC elements of a pixel, as loaded
    typedef typename std::conditional<VEC == 1, typename elem<ES>::type, v4i>::type raw;
    static __device__ __forceinline__ float f(const raw& r, int e)
    {
        static_assert(ES == 2);
        if constexpr (VEC == 1) return __uint_as_float((uint32_t)r << 16);
        else return __uint_as_float(e & 1 ? (uint32_t)r[e >> 1] & 0xFFFF0000u : (uint32_t)r[e >> 1] << 16);
    }
    static __device__ __forceinline__ int i(const raw& r, int e)
    {
        static_assert(ES == 1);
        if constexpr (VEC == 1) return r;
        else return (int)(signed char)((uint32_t)r[e >> 2] >> (8 * (e & 3)));
    }
};

// The pixels of a window and chunk as a lane sees them: `step` pixels on from its first, by buffer instructions, which drop what lies behind the last pixel (loads read zeros there).  A lane
// without channels is behind it everywhere.  The host bounds what a sample spans by 2 GiB
template <int ES, int VEC>
struct View {
    typedef typename Pack<ES, VEC>::raw raw;
    __amdgpu_buffer_rsrc_t r;
    unsigned off;
    int pitch;
    __device__ __forceinline__ View(const void* base, int64_t pixel, int pixels, int channels, bool live, int row, int col)
    {
        pitch = (int)pixel * ES;
        r = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, pixels ? (pixels - 1) * pitch + channels * ES : 0, 0x00020000);
        off = live ? (unsigned)(row * pitch + col * VEC * ES) : 0x80000000u;
    }
    // past: past the caches (non-temporal)
    __device__ __forceinline__ raw load(int step, bool past = false) const
    {
        if constexpr (VEC > 1) return past ? __builtin_bit_cast(raw, __builtin_amdgcn_raw_buffer_load_b128(r, off + (unsigned)(step * pitch), 0, 2)) : __builtin_bit_cast(raw, __builtin_amdgcn_raw_buffer_load_b128(r, off + (unsigned)(step * pitch), 0, 0));
        else if constexpr (ES == 2) return __builtin_bit_cast(raw, (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, off + (unsigned)(step * pitch), 0, 0));
        else return __builtin_bit_cast(raw, (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(r, off + (unsigned)(step * pitch), 0, 0));
    }
    __device__ __forceinline__ void store(raw v, int step, bool past = false) const
    {
        typedef unsigned v4u __attribute__((ext_vector_type(4)));
        if constexpr (VEC > 1) {
            if (past) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, v), r, off + (unsigned)(step * pitch), 0, 2);
            else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, v), r, off + (unsigned)(step * pitch), 0, 0);
        }
        else if constexpr (ES == 2) __builtin_amdgcn_raw_buffer_store_b16(v, r, off + (unsigned)(step * pitch), 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b8((uint8_t)v, r, off + (unsigned)(step * pitch), 0, 0);
    }
};

template <int ACT>
__device__ __forceinline__ float activate(float v)               // a NaN stays one
{
    if constexpr (ACT == EE_ACT_RELU) return v < 0.f ? 0.f : v;
    if constexpr (ACT == EE_ACT_RELU6) return v < 0.f ? 0.f : v > 6.f ? 6.f : v;
    if constexpr (ACT == EE_ACT_SILU) return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * v));
    return v;
}

// the pair of lanes that differ in bit `off` of their number: both get the merged value, from the same order
__device__ __forceinline__ void merge_pair(Moments& m, float nb, float mb, float qb, bool second)
{
    Moments lo = m;
    if (second) { lo = {nb, mb, qb}; merge(lo, m.n, m.mean, m.m2); }
    else merge(lo, nb, mb, qb);
    m = lo;
}
__device__ __forceinline__ void merge_lanes(Moments& m, int off, int lane) { merge_pair(m, __shfl_xor(m.n, off), __shfl_xor(m.mean, off), __shfl_xor(m.m2, off), lane & off); }
__device__ __forceinline__ void merge_lanes(Sums& s, int off, int)
{
    s.s1 += __shfl_xor(s.s1, off);
    s.s2 += __shfl_xor(s.s2, off);
}

// FORM 0: the whole sample's window in one workgroup, 1: statistics of a chunk, 2: merge the chunks of the sample, write one chunk.
// GPV: partial results per column (each of VEC / GPV channels of one group); PAST: y is written, and the residual read, past the caches
template <int ES, int VEC, int GPV, int NT, int NV, int FORM, bool PAST>
__global__ __launch_bounds__(NT) void group_norm_kernel(NormKernelArgs a)
{
    using P = Pack<ES, VEC>;
    using T = typename elem<ES>::type;
    using raw = typename P::raw;
    typedef typename std::conditional<ES == 2, Moments, Sums>::type stat_t;
    typedef typename std::conditional<ES == 2, float2, Sums>::type pair_t;
    constexpr int SUB = VEC / GPV, LOG_NT = NT == 256 ? 8 : NT == 512 ? 9 : 10;
    static_assert(NT == 256 || NT == 512 || NT == 1024);
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int u = xcd_unit(blockIdx.x, a.units);
    if (u < 0) return;
    const int tid = threadIdx.x, lane = tid & 63, cols = 1 << a.wlog, col = tid & (cols - 1), row = tid >> a.wlog, rows = NT >> a.wlog;
    const int win = u % a.windows, uc = u / a.windows, chunk = uc % a.chunks, b = uc / a.chunks;
    const int c0 = win * a.cw, cw = min(a.cw, a.c - c0), wgroups = cw / a.cpg;
    const int p0 = chunk * a.chunk_pixels, end = min(a.pixels, p0 + a.chunk_pixels);
    const bool live = col * VEC < cw;
    const int p1 = live ? end : p0;                                  // a lane without channels has no pixels
    const View<ES, VEC> x((const T*)a.x + b * a.x_sample + p0 * a.x_pixel + c0, a.x_pixel, end - p0, cw, live, row, col);

    const int slices = NT / max(64, cols);
    float* const l_n = (float*)lds;                                                                  // bf16: values of the lanes of a slice and column
    pair_t* const l_part = (pair_t*)(lds + (ES == 2 ? 4 * slices * cols : 0));                       // [slice][column][GPV]
    unsigned char* const l_group = (unsigned char*)(l_part + slices * cols * GPV);                   // per group: bf16 mean and 1 / deviation; int8 S1 and n deviation
    const double n_all = (double)a.pixels * a.cpg;
    auto settle = [&](int g, const stat_t& s) {
        if constexpr (ES == 2) ((float2*)l_group)[g] = float2{s.mean, rsqrtf(s.m2 / (float)n_all + a.eps) + 0.f * s.m2};      // squares past float's range: NaN, as those in a lane's own sums
        else {
            const long long n = (long long)a.pixels * a.cpg;
            const double var = (double)(n * s.s2 - (long long)s.s1 * s.s1) / (n_all * n_all);
            ((double2*)l_group)[g] = double2{(double)s.s1, n_all * sqrt(var + (double)a.eps)};
        }
    };
    // every group of the window, 2^sl lanes each that take its `entries` in turn: s = sum of get(group, entry); then f(group, s) in one lane
    auto per_group = [&](int entries, auto&& get, auto&& f) {
        int sl = 0;
        while (sl < 6 && (1 << sl) < entries && wgroups << (sl + 1) <= NT) ++sl;      // all groups at once, if they are no more than threads
        const int lanes = 1 << sl, sub = tid & (lanes - 1);
        for (int g0 = 0; g0 < wgroups; g0 += NT >> sl) {
            const int g = g0 + (tid >> sl);
            stat_t s{};
            if (g < wgroups)
#pragma unroll 4
                for (int e = sub; e < entries; e += lanes) get(g, e, s);
#pragma unroll 1
            for (int off = 1; off < lanes; off <<= 1) merge_lanes(s, off, lane);
            if (g < wgroups && sub == 0) f(g, s);
        }
    };

    raw data[NV];                                                     // two launches: one of two sets
    const bool has_res = FORM != 1 && a.res;
    const View<ES, VEC> res((const T*)a.res + b * a.r_sample + p0 * a.r_pixel + c0, a.r_pixel, has_res ? end - p0 : 0, cw, live, row, col);
#pragma unroll
    for (int i = 0; i < NV; ++i) data[i] = x.load(i * rows);         // pixels are counted from p0 from here on
    const int count = end - p0, mine = p1 - p0;
    // the lane's channels' factors, loaded with the first pixels
    constexpr bool AFFINE = FORM != 1 && (ES == 2 || VEC == 1);
    float weight[AFFINE ? VEC : 1], bias[AFFINE ? VEC : 1];
    if constexpr (AFFINE)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int c = min(c0 + col * VEC + e, a.c - 1);
            weight[e] = a.weight ? a.weight[c] : 1.f;
            bias[e] = a.bias ? a.bias[c] : 0.f;
        }
    // what was unpacked from a vector is not kept for the next time
    auto forget = [&](raw& v) {
        if constexpr (VEC > 1) asm volatile("" : "+v"(v));
    };

    if constexpr (FORM != 2) {
        // bf16: sums of x - pivot and of its square, the pivot first a value of the lane's own: as far from the mean as values of the group are.  mean and m2 hold them until 64 values (FORM 0: at most
        // 32) are added; these become a pair, which is merged with those before (`all`), and the next pivot is the mean up to there, rounded to bf16.  One sum over all values of a lane, up to
        // 16,384 of them, lost what a first value far from the others left of the variance: 1024 x 1024 pixels of one value but for the first were 6 to 45 % off.
        // Vectors behind the lane's last pixel read as what adds nothing: pivots, int8 zeros
        stat_t st[GPV] = {}, all[ES == 2 && FORM == 1 ? GPV : 1] = {};
        float pivot[ES == 2 ? GPV : 1];
        const int values = row < mine ? ((mine - row - 1) >> (LOG_NT - a.wlog)) + 1 : 0;      // vectors of the lane
        int left = values;                                           // of them not in `all` yet
        raw fill{};
        auto fill_up = [&] {
            if constexpr (ES == 2) {
                if constexpr (VEC == 1) fill = (raw)(__float_as_uint(pivot[0]) >> 16);
                else
#pragma unroll
                    for (int e = 0; e < VEC; e += 2) fill[e >> 1] = (int)(__float_as_uint(pivot[e / SUB]) >> 16 | (__float_as_uint(pivot[(e + 1) / SUB]) & 0xFFFF0000u));
            }
        };
        if constexpr (ES == 2) {
#pragma unroll
            for (int j = 0; j < GPV; ++j) pivot[j] = values ? P::f(data[0], j * SUB) : 0.f;
            fill_up();
        }
        // the sums of `vectors` vectors become the number of values, their mean and the sum of squared differences from it
        auto pairs = [&](int vectors) {
            if constexpr (ES == 2) {
                const float n = (float)(vectors * SUB), inv = __builtin_amdgcn_rcpf(fmaxf(n, 1.f));
#pragma unroll
                for (int j = 0; j < GPV; ++j) {
                    const float d = st[j].mean * inv;
                    st[j].n = n;
                    st[j].m2 = fmaxf(fmaf(-d, st[j].mean, st[j].m2), 0.f) + 0.f * st[j].m2;      // not below 0 by rounding; a NaN stays one
                    st[j].mean = pivot[j] + d;
                }
            }
        };
        auto merge_all = [&](int vectors) {
            if constexpr (ES == 2 && FORM == 1) {
                vectors = min(vectors, left);
                left -= vectors;
                pairs(vectors);
#pragma unroll
                for (int j = 0; j < GPV; ++j) {
                    merge(all[j], st[j].n, st[j].mean, st[j].m2);
                    st[j] = stat_t{};
                    pivot[j] = (float)(__bf16)all[j].mean;
                }
                fill_up();
            }
        };
        auto add = [&](raw (&v)[NV], int base) {
            if (base + NV * rows > count)
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (base + i * rows + row >= mine) v[i] = fill;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
#pragma unroll
                for (int j = 0; j < GPV; ++j) {
                    if constexpr (ES == 2) {
#pragma unroll
                        for (int e = 0; e < SUB; ++e) {
                            const float d = P::f(v[i], j * SUB + e) - pivot[j];
                            st[j].mean += d;
                            st[j].m2 = fmaf(d, d, st[j].m2);
                        }
                    } else {
                        int q = 0;
                        if constexpr (SUB % 4 == 0)
#pragma unroll
                            for (int e = 0; e < SUB / 4; ++e) {
                                const int w = v[i][j * SUB / 4 + e];
                                st[j].s1 = __builtin_amdgcn_sdot4(w, 0x01010101, st[j].s1, false);
                                q = __builtin_amdgcn_sdot4(w, w, q, false);
                            }
                        else
#pragma unroll
                            for (int e = 0; e < SUB; ++e) {
                                const int x1 = P::i(v[i], j * SUB + e);
                                st[j].s1 += x1;
                                q += x1 * x1;
                            }
                        st[j].s2 += q;
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        if constexpr (FORM == 0) add(data, 0);
        else {                                                       // the next pixels are on their way while these are added
            constexpr int TURNS = std::max(1, 64 / (2 * NV * SUB));  // that add 64 values
            raw d2[NV];
            int turn = 0;
#pragma unroll 1
            for (int base = 0; base < count; base += 2 * NV * rows) {
#pragma unroll
                for (int i = 0; i < NV; ++i) d2[i] = x.load(base + (NV + i) * rows);
                add(data, base);
#pragma unroll
                for (int i = 0; i < NV; ++i) data[i] = x.load(base + (2 * NV + i) * rows);
                add(d2, base + NV * rows);
                if (ES == 2 && ++turn == TURNS) {
                    turn = 0;
                    merge_all(TURNS * 2 * NV);
                }
            }
        }
        if constexpr (ES == 2 && FORM == 1) {
            merge_all(left);
#pragma unroll
            for (int j = 0; j < GPV; ++j) st[j] = all[j];
        } else pairs(values);
        // lanes of a wavefront with the same column, then slices of the workgroup through LDS
#pragma unroll 1
        for (int off = cols; off < 64; off <<= 1) {
            if constexpr (ES == 2) {
                const float nb = __shfl_xor(st[0].n, off);
#pragma unroll
                for (int j = 0; j < GPV; ++j) merge_pair(st[j], nb, __shfl_xor(st[j].mean, off), __shfl_xor(st[j].m2, off), lane & off);
            } else
#pragma unroll
                for (int j = 0; j < GPV; ++j) merge_lanes(st[j], off, lane);
        }
        if (cols >= 64 || lane < cols) {
            const int slice = cols >= 64 ? row : tid >> 6, at = slice * cols + col;
            if constexpr (ES == 2) l_n[at] = st[0].n;
#pragma unroll
            for (int j = 0; j < GPV; ++j) {
                if constexpr (ES == 2) l_part[at * GPV + j] = float2{st[j].mean, st[j].m2};
                else l_part[at * GPV + j] = st[j];
            }
        }
        __syncthreads();
        const int per = a.cpg / SUB;                                 // a group is so many neighbouring partials of every slice
        per_group(per * slices,
                  [&](int g, int e, stat_t& s) {
                      const int slice = e / per, slot = g * per + e - slice * per, at = slice * cols + slot / GPV;
                      const pair_t v = l_part[at * GPV + slot % GPV];
                      if constexpr (ES == 2) merge(s, l_n[at], v.x, v.y);
                      else { s.s1 += v.s1; s.s2 += v.s2; }
                  },
                  [&](int g, const stat_t& s) {
                      if constexpr (FORM == 1) {
                          const size_t at = ((size_t)b * a.chunks + chunk) * a.groups + c0 / a.cpg + g;
                          if constexpr (ES == 2) ((float2*)a.part)[at] = float2{s.mean, s.m2};
                          else ((Sums*)a.part)[at] = s;
                      } else settle(g, s);
                  });
    }
    if constexpr (FORM == 1) return;
    if constexpr (FORM == 2) {
        per_group(a.chunks,
                  [&](int g, int k, stat_t& s) {
                      const size_t at = ((size_t)b * a.chunks + k) * a.groups + c0 / a.cpg + g;
                      if constexpr (ES == 2) {
                          const float2 v = ((const float2*)a.part)[at];
                          merge(s, (float)(min(a.chunk_pixels, a.pixels - k * a.chunk_pixels)) * a.cpg, v.x, v.y);
                      } else {
                          const Sums v = ((const Sums*)a.part)[at];
                          s.s1 += v.s1;
                          s.s2 += v.s2;
                      }
                  },
                  settle);
    }
    __syncthreads();

    // ---- normalise, residual, activation --------------------------------------------------------------------------------
    const View<ES, VEC> y((const T*)a.y + b * a.y_sample + p0 * a.y_pixel + c0, a.y_pixel, end - p0, cw, live, row, col);
    // f(x, residual) -> y for every vector of the lane, four at a time, the next four's residuals (FORM 2: and x) on their way
    auto tiles = [&](auto res_tag, auto&& f) {
        constexpr bool RES = decltype(res_tag)::value;
        constexpr int BV = NV < 4 ? NV : 4;
        raw r[2][BV], d2[BV];
        auto residuals = [&](raw (&to)[BV], int i0) {
            if constexpr (RES)
#pragma unroll
                for (int i = 0; i < BV; ++i) to[i] = res.load(i0 + i * rows, PAST);
        };
        auto four = [&](raw* d, raw (&rr)[BV], int i0) {
#pragma unroll
            for (int i = 0; i < BV; ++i) {
                forget(d[i]);
                y.store(f(d[i], rr[i]), i0 + i * rows, PAST);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        residuals(r[0], 0);
        if constexpr (FORM == 0) {
#pragma unroll
            for (int k = 0; k < NV / BV; ++k) {
                if (k + 1 < NV / BV) residuals(r[(k + 1) & 1], (k + 1) * BV * rows);
                four(data + k * BV, r[k & 1], k * BV * rows);
            }
        } else {
#pragma unroll 1
            for (int base = 0; base < count; base += 2 * BV * rows) {
#pragma unroll
                for (int i = 0; i < BV; ++i) d2[i] = x.load(base + (BV + i) * rows);
                residuals(r[1], base + BV * rows);
                four(data, r[0], base);
#pragma unroll
                for (int i = 0; i < BV; ++i) data[i] = x.load(base + (2 * BV + i) * rows);
                residuals(r[0], base + 2 * BV * rows);
                four(d2, r[1], base + BV * rows);
            }
        }
    };
    if constexpr (ES == 2) {
        float mean[GPV];
#pragma unroll
        for (int j = 0; j < GPV; ++j) {
            const float2 g = ((const float2*)l_group)[min((col * VEC + j * SUB) / a.cpg, wgroups - 1)];
            mean[j] = g.x;
#pragma unroll
            for (int e = 0; e < SUB; ++e) weight[j * SUB + e] *= g.y;
        }
        auto run = [&](auto act_tag, auto res_tag) {
            constexpr int ACT = decltype(act_tag)::value;
            constexpr bool RES = decltype(res_tag)::value;
            tiles(res_tag, [&](const raw& d, const raw& r) {
                float v[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    v[e] = fmaf(P::f(d, e) - mean[e / SUB], weight[e], bias[e]);
                    if constexpr (RES) v[e] += P::f(r, e);
                    v[e] = activate<ACT>(v[e]);
                }
                if constexpr (VEC == 1) return __builtin_bit_cast(uint16_t, (__bf16)v[0]);
                else {
                    v4i o;
#pragma unroll
                    for (int e = 0; e < VEC; e += 2) o[e >> 1] = (int)pack2_bf16(v[e], v[e + 1]);
                    return o;
                }
            });
        };
        auto with = [&](auto act_tag) {
            if (has_res) run(act_tag, std::true_type{});
            else run(act_tag, std::false_type{});
        };
        if (a.act == EE_ACT_NONE) with(std::integral_constant<int, EE_ACT_NONE>{});
        else if (a.act == EE_ACT_RELU) with(std::integral_constant<int, EE_ACT_RELU>{});
        else if (a.act == EE_ACT_RELU6) with(std::integral_constant<int, EE_ACT_RELU6>{});
        else with(std::integral_constant<int, EE_ACT_SILU>{});
    } else {
        auto group_of = [&](int e) { return ((const double2*)l_group)[min((col * VEC + e) / a.cpg, wgroups - 1)]; };
        // per channel, in 64 bits: factor, offset
        auto channel = [&](float w, float bi, double2 g) { return double2{(double)w * a.out_scale / g.y, (double)bi * a.out_scale + 0.5}; };
        auto in_64 = [&](int v, int r, double s1, double2 c) {       // the definition, each operation rounded by itself: products that lie halfway between whole numbers are ordinary (n deviation is whole for a group of two values)
#pragma clang fp contract(off)
            double t = (n_all * v - s1) * c.x;
            t += c.y;
            if (has_res) t += r * a.res_scale;
            return (int)fmin(fmax(floor(t), (double)a.lo), (double)a.hi);
        };
        if constexpr (VEC == 1) {
            const double2 c = channel(weight[0], bias[0], group_of(0));
            const double s1 = group_of(0).x;
            if (has_res) tiles(std::true_type{}, [&](const raw& d, const raw& r) { return (int8_t)in_64(d, r, s1, c); });
            else tiles(std::false_type{}, [&](const raw& d, const raw&) { return (int8_t)in_64(d, 0, s1, c); });
        } else {
            // in float, of bytes + 128 (one instruction turns a byte without sign into a float), the result moved up by 128 as well: t = x f + h + (r + 128) rs
            // The factors of a channel in 64 bits, once per workgroup.  Worked out from memory where they were needed they made 16 x 2000x128 with the same weight for all channels, where a value near
            // a whole number is one in all of them, 22 to 44 us (now 14)
            double2* const l_channel = (double2*)(l_group + 16 * (a.cw / a.cpg));
            const float rs = has_res ? (float)a.res_scale : 0.f;
            for (int k = tid; k < cw; k += NT) l_channel[k] = channel(a.weight ? a.weight[c0 + k] : 1.f, a.bias ? a.bias[c0 + k] : 0.f, ((const double2*)l_group)[k / a.cpg]);
            __syncthreads();
            const int c1 = min(col * VEC, cw - VEC), own = c1 / a.cpg;       // the column's first channel, its group (the only one, with GPV 1)
            double first = 0.0;                                              // what the offset takes off for a group: S1 + 128 n
            float f[VEC], h[VEC], most = 0.f;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const double2 c = l_channel[c1 + e];
                if (e % SUB == 0) first = ((const double2*)l_group)[GPV == 1 ? own : (c1 + e) / a.cpg].x + 128.0 * n_all;
                f[e] = (float)(n_all * c.x);
                h[e] = (float)(c.y + 128.0 - first * c.x - 128.0 * rs);
                most = fmaxf(most, 256.f * fabsf(f[e]) + fabsf(h[e]));
                if (!(fabsf(f[e]) < 1e30f) || !(fabsf(h[e]) < 1e30f)) most = 1e30f;
            }
            // how far t can be off, in half steps of 2^-24: a byte times its rounded factor, the rounded offset, the sum, the sum with the residual (results past the bounds do not matter).
            // t is kept half a unit inside the bounds: all that is cut off there has the bound as its result, and is not near a whole number
            const float safe = 0.5f - 5.97e-8f * (most + 256.f * rs + 520.f);
            const float lo = (float)(a.lo + 128) + 0.5f, hi = (float)(a.hi + 128) + 0.5f;
            auto run = [&](auto res_tag) {
                constexpr bool RES = decltype(res_tag)::value;
                tiles(res_tag, [&](const raw& d, const raw& r) {
                    v4i o;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t xd = (uint32_t)d[w] ^ 0x80808080u, xr = RES ? (uint32_t)r[w] ^ 0x80808080u : 0u;
                        uint32_t q = 0;
                        float far = 0.f;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int e = 4 * w + k;
                            float t = fmaf((float)(xd >> (8 * k) & 255u), f[e], h[e]);
                            if constexpr (RES) t = fmaf((float)(xr >> (8 * k) & 255u), rs, t);
                            t = clamp_f32(t, lo, hi);
                            const float part = __builtin_amdgcn_fractf(t);
                            far = fmaxf(far, fabsf(part - 0.5f));
                            q = __builtin_amdgcn_cvt_pk_u8_f32(t - part, k, q);
                        }
                        q ^= 0x80808080u;
                        if (!(far < safe)) {                         // near a whole number
                            q = 0;
#pragma unroll 1
                            for (int k = 0; k < 4; ++k) {
                                const int c = c1 + 4 * w + k, v = (int)(signed char)((uint32_t)d[w] >> (8 * k)), rv = RES ? (int)(signed char)((uint32_t)r[w] >> (8 * k)) : 0;
                                q |= ((uint32_t)in_64(v, rv, ((const double2*)l_group)[GPV == 1 ? own : c / a.cpg].x, l_channel[c]) & 255u) << (8 * k);
                            }
                        }
                        o[w] = (int)q;
                    }
                    return o;
                });
            };
            if (has_res) run(std::true_type{});
            else run(std::false_type{});
        }
    }
}

enum { NORM_LDS = 160 * 1024 };
int gcd_i(int a, int b) { while (b) { const int t = a % b; a = b; b = t; } return a; }
int log2_up(int v) { int k = 0; while ((1 << k) < v) ++k; return k; }

// how a call is cut up: the kernel's window, its threads and vectors per lane, chunks of pixels; split: two launches
struct NormPlan { int vec, gpv, nt, nv, wv, wlog, windows, chunks, chunk_pixels, batch; bool ok, split, past; };

size_t norm_lds(int es, int gpv, int nt, int wlog, int window_groups, int window_channels)
{
    const size_t cells = (size_t)(nt / std::max(64, 1 << wlog)) << wlog;
    return (es == 2 ? 4 : 0) * cells + (es == 2 ? 8 : 16) * cells * gpv + 16 * (size_t)window_groups + (es == 1 ? 16 * (size_t)window_channels : 0);
}

bool plan_norm_vec(const NormArgs& a, int vec, NormPlan& p)
{
    const int es = a.dtype == EE_I8 ? 1 : 2, cpg = a.c / a.groups;
    if (cpg > 8192) return false;                                     // bf16: columns of 1024 threads; int8: their factors in LDS
    const int unit = cpg / gcd_i(cpg, vec);                           // columns of the smallest window of whole groups
    p.vec = vec;
    p.gpv = vec == 1 || cpg % vec == 0 ? 1 : cpg % (vec / 4) == 0 ? 4 : vec;
    const int all = a.c / vec;                                        // columns of the tensor, a multiple of unit
    auto window = [&](int want) {
        p.wv = std::min(all, unit * std::max(1, want / unit));
        p.wlog = log2_up(p.wv);
        p.windows = (all + p.wv - 1) / p.wv;
    };
    auto fits = [&] { return (1 << p.wlog) <= p.nt && norm_lds(es, p.gpv, p.nt, p.wlog, p.wv * vec / cpg, p.wv * vec) <= NORM_LDS; };
    // one launch.  The largest window that 256 threads hold, of at least 128 workgroups if there are such: what a workgroup does before its first result is the same for any.  bf16, columns of 16 bytes
    // and us: 1000 x 3x3x256 4 29, 8 19, 32 12.4; 512 x 4x4x1024 8 35, 16 34, 64 13.8; 256 x 7x7x512 4 17, 8 14.7, 16 13.4; 78 x 180x128 2 7.5, 4 6.2; 1 x 7x7x2048 8 5.6, 16 6.4
    const int least = vec == 1 ? 16 : 2;
    p.chunks = 1;
    p.chunk_pixels = a.pixels;
    NormPlan held{};
    for (int want = 256; want >= least; want /= 2) {
        window(want);
        p.nt = 256;
        const int64_t vectors = (int64_t)a.pixels << p.wlog;
        p.nv = vectors <= 256 ? 1 : 4;
        if (vectors > 1024 || !fits()) continue;
        held = p;
        held.ok = true;
        if ((int64_t)a.b * p.windows >= 128) break;
    }
    if (held.ok) { p = held; return true; }
    // the smallest window and more threads; 1024 only while all workgroups are at work at once.  This / two launches, bf16, us: 41 x 770x256 13.2 / 15.4, 256 x 900x256 54.8 / 57.0;
    // 1024 threads 16 x 1600x256 11.8 / 14.3, 64 x 2000x128 23.7 / 19.9, 256 x 1100x64 34 / 21
    window(least);
    p.nv = 4;
    for (p.nt = 512; p.nt <= 1024; p.nt *= 2)
        if (fits() && (int64_t)a.pixels << p.wlog <= 4 * p.nt && (p.nt == 512 || (int64_t)a.b * p.windows <= 256)) return true;
    // two launches, of whole pixels where they are up to 1 KiB.  Few long workgroups: what one does before its first result is worth tens of KB.  256 / 512 / 1024 / 2048 of them, bf16, us:
    // 64 x 56x56x256 with residual 69, 68, 75, 79, 16 of these 24, 27, 31, 31; 256 x 112x112x64 225, 222, 224, 221
    for (int want = 64; want >= 8; want /= 2) {
        window(want);
        p.nt = p.wlog > 8 ? 1024 : 256;
        p.nv = 8;                                                     // the kernel's two sets of NV = 4
        if (!fits()) continue;
        const int tile = p.nv * (p.nt >> p.wlog);                     // pixels a workgroup holds at once
        const int64_t tiles = ((int64_t)a.pixels + tile - 1) / tile, units = (int64_t)a.b * p.windows;
        p.chunks = (int)std::min<int64_t>(tiles, std::min<int64_t>(64, std::max<int64_t>(1, 512 / units)));
        const int64_t per = (tiles + p.chunks - 1) / p.chunks;
        p.chunk_pixels = (int)std::min<int64_t>(per * tile, a.pixels);
        p.chunks = (int)(((int64_t)a.pixels + p.chunk_pixels - 1) / p.chunk_pixels);
        p.split = true;
        return true;
    }
    return false;
}

// Two launches read x twice: so many samples at a time that the last-level cache (256 MB) still holds them for the second.  256 x 112x112x64 bf16 (411 MB) 233 us in one part, 213 in two, 243 in
// four; 256 x 56x56x256 with residual 307, 276, 321
int norm_batch(const NormArgs& a)
{
    const double bytes = (double)a.b * a.pixels * a.c * (a.dtype == EE_I8 ? 1 : 2);
    const int parts = (int)std::min((double)a.b, std::ceil(bytes / (224.0 * 1048576.0)));
    return parts > 1 ? (a.b + parts - 1) / parts : a.b;
}

NormPlan plan_norm(const NormArgs& a, bool aligned)
{
    NormArgs part = a;
    part.b = norm_batch(a);
    NormPlan p{};
    const int full = a.dtype == EE_I8 ? 16 : 8;
    p.ok = (aligned && a.c % full == 0 && plan_norm_vec(part, full, p)) || plan_norm_vec(part, 1, p);
    p.batch = p.split ? part.b : a.b;
    // a launch has less than 2^32 threads, and xcd_unit counts up to 2^28 workgroups: more samples than that are worked through in parts
    if (p.ok) p.batch = (int)std::min<int64_t>(p.batch, std::min((1ll << 32) / p.nt - 8, (1ll << 28) - 8) / ((int64_t)p.chunks * p.windows));
    // a large result is written past the caches: left in them, writing it back would fall on the next kernel.  64 x 56x56x256 bf16 with residual, both launches 89 -> 77 us, 256 x 112x112x64 247 -> 232
    p.past = (double)a.b * a.pixels * a.c * (a.dtype == EE_I8 ? 1 : 2) >= 64e6;
    return p;
}

template <int ES, int VEC, int GPV, int NT, int NV, int FORM, bool PAST = false>
hipError_t launch_norm_form(const NormKernelArgs& k, hipStream_t s)
{
    static const hipError_t granted = hipFuncSetAttribute(reinterpret_cast<const void*>(&group_norm_kernel<ES, VEC, GPV, NT, NV, FORM, PAST>), hipFuncAttributeMaxDynamicSharedMemorySize, NORM_LDS);
    if (granted != hipSuccess) return granted;
    EE_LAUNCH((group_norm_kernel<ES, VEC, GPV, NT, NV, FORM, PAST>), dim3(xcd_grid(k.units)), dim3(NT), (unsigned)norm_lds(ES, GPV, NT, k.wlog, k.cw / k.cpg, k.cw), s, k);
    return hipGetLastError();
}

template <int ES, int VEC, int GPV>
hipError_t launch_norm_gpv(const NormKernelArgs& k, const NormPlan& p, hipStream_t s, TimedLaunches& timed, bool last)
{
    timed.before(last && !p.split);
    if (p.split && p.nt == 256) {
        const hipError_t e = launch_norm_form<ES, VEC, GPV, 256, 4, 1>(k, s);
        if (e != hipSuccess) return e;
        timed.before(last);
        return p.past ? launch_norm_form<ES, VEC, GPV, 256, 4, 2, true>(k, s) : launch_norm_form<ES, VEC, GPV, 256, 4, 2>(k, s);
    }
    if (p.nt == 256) return p.nv == 1 ? launch_norm_form<ES, VEC, GPV, 256, 1, 0>(k, s) : launch_norm_form<ES, VEC, GPV, 256, 4, 0>(k, s);
    if (p.nt == 512) return launch_norm_form<ES, VEC, GPV, 512, 4, 0>(k, s);
    if (!p.split) return launch_norm_form<ES, VEC, GPV, 1024, 4, 0>(k, s);
    // two launches of 1,024 threads are for windows of more than 256 columns, a partial of each group for every thread: with sixteen groups to a column (int8) more than LDS holds, so no plan has them
    if constexpr ((ES == 2 ? 8 : 16) * 1024 * GPV <= NORM_LDS) {
        // int8's second launch keeps 16 to 20 registers in memory (128 are a thread's): 16 x 900x8192, groups of 8,192 channels 75 us, of 4,096, with 256 threads, 64
        const hipError_t e = launch_norm_form<ES, VEC, GPV, 1024, 4, 1>(k, s);
        timed.before(last);
        return e == hipSuccess ? launch_norm_form<ES, VEC, GPV, 1024, 4, 2>(k, s) : e;
    }
    return hipErrorInvalidValue;
}

bool norm_aligned(const NormArgs& a)
{
    const int full = a.dtype == EE_I8 ? 16 : 8;
    auto ok = [&](const void* p, int64_t sample, int64_t pixel) { return ((uintptr_t)p & 15) == 0 && sample % full == 0 && pixel % full == 0; };
    return ok(a.x, a.x_sample, a.x_pixel) && ok(a.y, a.y_sample, a.y_pixel) && (!a.res || ok(a.res, a.res_sample, a.res_pixel));
}

}  // namespace

int group_norm_check(const NormArgs& a)
{
    const NormPlan p = plan_norm(a, norm_aligned(a));
    return !p.ok ? EE_ERR_UNSUPPORTED : p.batch < 1 ? EE_ERR_OVERFLOW : EE_OK;
}

// a call whose alignment is not known yet may be cut either way
size_t group_norm_workspace(const NormArgs& a)
{
    size_t most = 0;
    for (const bool aligned : {false, true}) {
        const NormPlan p = plan_norm(a, aligned);
        if (p.ok && p.split) most = std::max(most, (size_t)p.batch * p.chunks * a.groups * 16);
    }
    return most;
}

hipError_t launch_group_norm(const NormArgs& a, void* workspace, hipStream_t s)
{
    const NormPlan p = plan_norm(a, norm_aligned(a));
    NormKernelArgs k{};
    k.weight = a.weight; k.bias = a.bias; k.part = workspace;
    k.x_sample = a.x_sample; k.x_pixel = a.x_pixel; k.r_sample = a.res_sample; k.r_pixel = a.res_pixel; k.y_sample = a.y_sample; k.y_pixel = a.y_pixel;
    k.pixels = a.pixels; k.c = a.c; k.groups = a.groups; k.cpg = a.c / a.groups;
    k.cw = p.wv * p.vec; k.wlog = p.wlog; k.windows = p.windows; k.chunks = p.chunks; k.chunk_pixels = p.chunk_pixels;
    k.eps = a.eps; k.act = a.act;
    k.out_scale = std::ldexp(1.0, a.frac_bits); k.res_scale = std::ldexp(1.0, a.res_shift);
    k.lo = a.act == EE_ACT_NONE ? -128 : 0;
    k.hi = a.act == EE_ACT_RELU6 ? (int)std::min(127.0, 6.0 * k.out_scale) : 127;
    const int64_t es = a.dtype == EE_I8 ? 1 : 2;
    auto at = [&](const void* base, int64_t b, int64_t sample) { return base ? (void*)((char*)base + b * sample * es) : nullptr; };
    TimedLaunches timed;
    for (int64_t b = 0; b < a.b; b += p.batch) {
        const bool last = a.b - b <= p.batch;
        k.x = at(a.x, b, a.x_sample); k.res = at(a.res, b, a.res_sample); k.y = at(a.y, b, a.y_sample);
        k.units = (int)std::min<int64_t>(p.batch, a.b - b) * p.chunks * p.windows;
        const hipError_t e = a.dtype == EE_I8 ? (p.vec == 1 ? launch_norm_gpv<1, 1, 1>(k, p, s, timed, last) : p.gpv == 1 ? launch_norm_gpv<1, 16, 1>(k, p, s, timed, last) : p.gpv == 4 ? launch_norm_gpv<1, 16, 4>(k, p, s, timed, last) : launch_norm_gpv<1, 16, 16>(k, p, s, timed, last))
                           : p.vec == 1 ? launch_norm_gpv<2, 1, 1>(k, p, s, timed, last) : p.gpv == 1 ? launch_norm_gpv<2, 8, 1>(k, p, s, timed, last) : p.gpv == 4 ? launch_norm_gpv<2, 8, 4>(k, p, s, timed, last) : launch_norm_gpv<2, 8, 8>(k, p, s, timed, last);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ee
