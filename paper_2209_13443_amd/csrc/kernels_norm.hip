// Group norm with an activation, channels last (int8 and bf16), for gfx950.
//
// Per sample b and group g of cpg = C / G channels, n = pixels * cpg values:
//   bf16  y = act(weight_c (x - mean) / sqrt(var + eps) + bias_c + res), one rounding at the end
//   int8  S1 = sum x, S2 = sum x^2 (exact integers), d = n x - S1, m_c = weight_c 2^f / (n sqrt((n S2 - S1^2) / n^2 + eps)),
//         y = clamp(floor(d m_c + (bias_c 2^f + 1/2) + res 2^rs), lo, hi) in 64-bit floats: d is exact, so a constant group gives its bias on
//         every machine and the results are whole numbers that do not depend on the order of a sum
// Statistics of bf16: every thread has the mean and the sum of squared differences from it of its own values, in registers, and the pairs are merged
// (n = na + nb, delta = mb - ma: mean = ma + delta nb / n, M2 = M2a + M2b + delta^2 na nb / n), so that a mean far from zero costs nothing.
//
// Bound by memory.  A workgroup has a window of whole groups (columns of 16 bytes, a power of two of them) and some pixels of one sample; a lane has one
// column and every NT / columns-th pixel.  Where the window of a whole sample fits a workgroup's registers it is one launch that reads x once; else two:
// statistics of chunks of pixels, then every workgroup of the second launch merges the chunks of its sample and writes its part (x is read again).
#include <algorithm>
#include <type_traits>

#include "ee_internal.hpp"
#include "igemm_device.hpp"

namespace ee {
namespace {

struct NormKernelArgs {
    const void* x; const void* res; void* y;
    const float* weight; const float* bias;
    void* part;                      // split form: [sample][chunk][group] pairs
    int64_t x_sample, x_pixel, r_sample, r_pixel, y_sample, y_pixel;      // strides in elements
    int pixels, c, groups, cpg;
    int cw, wlog;                    // channels of a window (whole groups), log2 of its columns (idle ones included)
    int windows, chunks, chunk_pixels;
    float eps;
    double out_scale, res_scale;     // int8: 2^frac_bits, 2^res_shift
    int act, lo, hi;
};

// what a lane knows of a part of a group: n values, their mean and the sum of squared differences from it
struct Moments { float n, mean, m2; };
__device__ __forceinline__ void merge(Moments& a, float nb, float mb, float m2b)
{
    const float n = a.n + nb, w = nb * __builtin_amdgcn_rcpf(fmaxf(n, 1.f)), d = mb - a.mean;
    a.mean = fmaf(d, w, a.mean);
    a.m2 += fmaf(d * d, a.n * w, m2b);
    a.n = n;
}
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

__device__ __forceinline__ float activate(float v, int act)      // a NaN stays one
{
    if (act == EE_ACT_RELU) return v < 0.f ? 0.f : v;
    if (act == EE_ACT_RELU6) return v < 0.f ? 0.f : v > 6.f ? 6.f : v;
    if (act == EE_ACT_SILU) return v * __builtin_amdgcn_rcpf(1.f + __expf(-v));
    return v;
}

// MODE 0: the whole sample's window in one workgroup, 1: statistics of a chunk, 2: merge the chunks of the sample, write one chunk.
// GPV: partial results per column (each of VEC / GPV channels of one group)
template <int ES, int VEC, int GPV, int NT, int NV, int MODE>
__global__ __launch_bounds__(NT) void group_norm_kernel(NormKernelArgs a)
{
    using P = Pack<ES, VEC>;
    using T = typename elem<ES>::type;
    constexpr int SUB = VEC / GPV;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, cols = 1 << a.wlog, col = tid & (cols - 1), row = tid >> a.wlog, rows = NT >> a.wlog;
    int u = blockIdx.x;
    const int win = u % a.windows; u /= a.windows;
    const int chunk = u % a.chunks, b = u / a.chunks;
    const int c0 = win * a.cw, cw = min(a.cw, a.c - c0), wgroups = cw / a.cpg;
    const bool live = col * VEC < cw;
    const int p0 = chunk * a.chunk_pixels, p1 = min(a.pixels, p0 + a.chunk_pixels);
    const T* const x = (const T*)a.x + b * a.x_sample + c0 + col * VEC;

    // ---- LDS: per-lane partials of the reduction | per group | per channel --------------------------------------------
    const int slices = NT / max(64, cols);
    float* const l_n = (float*)lds;                                  // [slices][cols] counts (bf16)
    unsigned char* const l_part = lds + (ES == 2 ? 4 * slices * cols : 0);
    // pairs [slices][cols][GPV]
    typedef typename std::conditional<ES == 2, float2, Sums>::type pair_t;
    pair_t* const part = (pair_t*)l_part;
    float2* const l_group = (float2*)(l_part + sizeof(pair_t) * slices * cols * GPV);      // bf16: mean, 1 / sqrt(var + eps); int8: S1 and factor as doubles
    double2* const l_group_d = (double2*)l_group;
    const double n_all = (double)a.pixels * a.cpg;

    typename P::raw data[NV];
    auto load = [&](int base) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = base + row + i * rows;
            if (live && p < p1) data[i] = *(const typename P::raw*)(x + p * a.x_pixel);
        }
    };
    auto have = [&](int base) { return !live || base + row >= p1 ? 0 : min(NV, (p1 - base - row - 1) / rows + 1); };

    // ---- statistics ---------------------------------------------------------------------------------------------------
    if constexpr (MODE != 2) {
        Moments mo[GPV];
        Sums su[GPV];
#pragma unroll
        for (int j = 0; j < GPV; ++j) { mo[j] = {0.f, 0.f, 0.f}; su[j] = {0, 0}; }
        for (int base = p0; base < p1; base += NV * rows) {
            load(base);
            const int cnt = have(base);
            if constexpr (ES == 2) {
                const float nb = (float)(cnt * SUB);
#pragma unroll
                for (int j = 0; j < GPV; ++j) {
                    float s = 0.f, q = 0.f;
#pragma unroll
                    for (int i = 0; i < NV; ++i)
                        if (i < cnt)
#pragma unroll
                            for (int e = 0; e < SUB; ++e) s += P::f(data[i], j * SUB + e);
                    const float m = s / fmaxf(nb, 1.f);                  // a division: equal values have exactly their value as mean
#pragma unroll
                    for (int i = 0; i < NV; ++i)
                        if (i < cnt)
#pragma unroll
                            for (int e = 0; e < SUB; ++e) {
                                const float d = P::f(data[i], j * SUB + e) - m;
                                q = fmaf(d, d, q);
                            }
                    if (cnt) merge(mo[j], nb, m, q);
                }
            } else {
#pragma unroll
                for (int j = 0; j < GPV; ++j) {
                    int s = 0, q = 0;
#pragma unroll
                    for (int i = 0; i < NV; ++i)
                        if (i < cnt)
#pragma unroll
                            for (int e = 0; e < SUB; ++e) {
                                const int v = P::i(data[i], j * SUB + e);
                                s += v;
                                q += v * v;
                            }
                    su[j].s1 += s;
                    su[j].s2 += q;
                }
            }
        }
        // lanes of a wavefront with the same column, then slices of the workgroup through LDS
        const int lane = tid & 63;
#pragma unroll 1
        for (int off = cols; off < 64; off <<= 1) {
            if constexpr (ES == 2) {
                const float nb = __shfl_xor(mo[0].n, off);
#pragma unroll
                for (int j = 0; j < GPV; ++j) {
                    const float mb = __shfl_xor(mo[j].mean, off), qb = __shfl_xor(mo[j].m2, off);
                    // both lanes of a pair merge in the same order
                    Moments lo = mo[j];
                    if (lane & off) { lo = {nb, mb, qb}; merge(lo, mo[j].n, mo[j].mean, mo[j].m2); }
                    else merge(lo, nb, mb, qb);
                    mo[j] = lo;
                }
            } else {
#pragma unroll
                for (int j = 0; j < GPV; ++j) {
                    su[j].s1 += __shfl_xor(su[j].s1, off);
                    su[j].s2 += __shfl_xor(su[j].s2, off);
                }
            }
        }
        if (cols >= 64 || lane < cols) {
            const int slice = cols >= 64 ? row : tid >> 6, at = slice * cols + col;
            if constexpr (ES == 2) {
                l_n[at] = mo[0].n;
#pragma unroll
                for (int j = 0; j < GPV; ++j) part[at * GPV + j] = float2{mo[j].mean, mo[j].m2};
            } else {
#pragma unroll
                for (int j = 0; j < GPV; ++j) part[at * GPV + j] = su[j];
            }
        }
        __syncthreads();
        // a group is cpg / SUB neighbouring partials of every slice: 2^sl lanes of a wavefront take them in turn
        const int per = a.cpg / SUB, entries = per * slices;
        int sl = 0;
        while (sl < 6 && (1 << sl) < entries) ++sl;
        const int lanes = 1 << sl, sub = tid & (lanes - 1);
        for (int g0 = 0; g0 < wgroups; g0 += NT >> sl) {
            const int g = g0 + (tid >> sl);
            Moments m = {0.f, 0.f, 0.f};
            Sums s = {0, 0};
            if (g < wgroups)
                for (int e = sub; e < entries; e += lanes) {
                    const int slice = e / per, slot = g * per + e - slice * per;           // slot: partial of the window
                    const int at = slice * cols + slot / GPV;
                    if constexpr (ES == 2) {
                        const float2 v = part[at * GPV + slot % GPV];
                        merge(m, l_n[at], v.x, v.y);
                    } else {
                        const Sums v = part[at * GPV + slot % GPV];
                        s.s1 += v.s1;
                        s.s2 += v.s2;
                    }
                }
#pragma unroll 1
            for (int off = 1; off < lanes; off <<= 1) {
                if constexpr (ES == 2) {
                    const float nb = __shfl_xor(m.n, off), mb = __shfl_xor(m.mean, off), qb = __shfl_xor(m.m2, off);
                    Moments lo = m;
                    if (sub & off) { lo = {nb, mb, qb}; merge(lo, m.n, m.mean, m.m2); }
                    else merge(lo, nb, mb, qb);
                    m = lo;
                } else {
                    s.s1 += __shfl_xor(s.s1, off);
                    s.s2 += __shfl_xor(s.s2, off);
                }
            }
            if (g < wgroups && sub == 0) {
                if constexpr (MODE == 1) {
                    const size_t at = ((size_t)b * a.chunks + chunk) * a.groups + c0 / a.cpg + g;
                    if constexpr (ES == 2) ((float2*)a.part)[at] = float2{m.mean, m.m2};
                    else ((Sums*)a.part)[at] = s;
                } else if constexpr (ES == 2) l_group[g] = float2{m.mean, rsqrtf(m.m2 / (float)n_all + a.eps)};
                else {
                    const long long n = (long long)a.pixels * a.cpg;
                    const double var = (double)(n * s.s2 - (long long)s.s1 * s.s1) / (n_all * n_all);
                    l_group_d[g] = double2{(double)s.s1, 1.0 / (n_all * sqrt(var + (double)a.eps))};
                }
            }
        }
    }
    if constexpr (MODE == 1) return;
    if constexpr (MODE == 2) {
        int sl = 0;
        while (sl < 6 && (1 << sl) < a.chunks) ++sl;
        const int lanes = 1 << sl, sub = tid & (lanes - 1);
        for (int g0 = 0; g0 < wgroups; g0 += NT >> sl) {
            const int g = g0 + (tid >> sl);
            Moments m = {0.f, 0.f, 0.f};
            long long s1 = 0, s2 = 0;
            if (g < wgroups)
                for (int k = sub; k < a.chunks; k += lanes) {
                    const size_t at = ((size_t)b * a.chunks + k) * a.groups + c0 / a.cpg + g;
                    if constexpr (ES == 2) {
                        const float2 v = ((const float2*)a.part)[at];
                        merge(m, (float)(min(a.chunk_pixels, a.pixels - k * a.chunk_pixels)) * a.cpg, v.x, v.y);
                    } else {
                        const Sums v = ((const Sums*)a.part)[at];
                        s1 += v.s1;
                        s2 += v.s2;
                    }
                }
#pragma unroll 1
            for (int off = 1; off < lanes; off <<= 1) {
                if constexpr (ES == 2) {
                    const float nb = __shfl_xor(m.n, off), mb = __shfl_xor(m.mean, off), qb = __shfl_xor(m.m2, off);
                    Moments lo = m;
                    if (sub & off) { lo = {nb, mb, qb}; merge(lo, m.n, m.mean, m.m2); }
                    else merge(lo, nb, mb, qb);
                    m = lo;
                } else {
                    s1 += __shfl_xor(s1, off);
                    s2 += __shfl_xor(s2, off);
                }
            }
            if (g < wgroups && sub == 0) {
                if constexpr (ES == 2) l_group[g] = float2{m.mean, rsqrtf(m.m2 / (float)n_all + a.eps)};
                else {
                    const long long n = (long long)a.pixels * a.cpg;
                    const double var = (double)(n * s2 - s1 * s1) / (n_all * n_all);
                    l_group_d[g] = double2{(double)s1, 1.0 / (n_all * sqrt(var + (double)a.eps))};
                }
            }
        }
    }
    __syncthreads();
    if (!live) return;

    // ---- normalise, residual, activation --------------------------------------------------------------------------------
    const T* const res = a.res ? (const T*)a.res + b * a.r_sample + c0 + col * VEC : nullptr;
    T* const y = (T*)a.y + b * a.y_sample + c0 + col * VEC;
    if constexpr (ES == 2) {
        float mean[VEC], scale[VEC], shift[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int c = c0 + col * VEC + e;
            const float2 g = l_group[(col * VEC + e) / a.cpg];
            mean[e] = g.x;
            scale[e] = g.y * (a.weight ? a.weight[c] : 1.f);
            shift[e] = a.bias ? a.bias[c] : 0.f;
        }
        for (int base = p0; base < p1; base += NV * rows) {
            if constexpr (MODE == 2) load(base);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int p = base + row + i * rows;
                if (p >= p1) continue;
                typename P::raw r{};
                if (res) r = *(const typename P::raw*)(res + p * a.r_pixel);
                float v[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    v[e] = fmaf(P::f(data[i], e) - mean[e], scale[e], shift[e]);
                    if (res) v[e] += P::f(r, e);
                    v[e] = activate(v[e], a.act);
                }
                if constexpr (VEC == 1) y[p * a.y_pixel] = __builtin_bit_cast(uint16_t, (__bf16)v[0]);
                else {
                    v4i o;
#pragma unroll
                    for (int e = 0; e < VEC; e += 2) o[e >> 1] = (int)pack2_bf16(v[e], v[e + 1]);
                    *(v4i*)(y + p * a.y_pixel) = o;
                }
            }
        }
    } else {
        for (int base = p0; base < p1; base += NV * rows) {
            if constexpr (MODE == 2) load(base);
            int q[NV][VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int c = c0 + col * VEC + e;
                const double2 g = l_group_d[(col * VEC + e) / a.cpg];
                const double m = (a.weight ? (double)a.weight[c] : 1.0) * a.out_scale * g.y, o = (a.bias ? (double)a.bias[c] : 0.0) * a.out_scale + 0.5;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int p = base + row + i * rows;
                    if (p >= p1) continue;
                    double t = fma(n_all * P::i(data[i], e) - g.x, m, o);
                    if (res) t += res[p * a.r_pixel + e] * a.res_scale;
                    q[i][e] = (int)fmin(fmax(floor(t), (double)a.lo), (double)a.hi);
                }
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int p = base + row + i * rows;
                if (p >= p1) continue;
                if constexpr (VEC == 1) y[p * a.y_pixel] = (int8_t)q[i][0];
                else {
                    v4i o;
#pragma unroll
                    for (int e = 0; e < VEC; e += 4) o[e >> 2] = (int)pack4_i8(q[i][e], q[i][e + 1], q[i][e + 2], q[i][e + 3]);
                    *(v4i*)(y + p * a.y_pixel) = o;
                }
            }
        }
    }
}

int gcd_i(int a, int b) { while (b) { const int t = a % b; a = b; b = t; } return a; }
int log2_up(int v) { int k = 0; while ((1 << k) < v) ++k; return k; }

// how a call is cut up: the kernel's window, its threads and vectors per lane, chunks of pixels (1: one launch)
struct NormPlan { int vec, gpv, nt, nv, wv, wlog, windows, chunks, chunk_pixels; bool ok; };

size_t norm_lds(int es, int gpv, int nt, int wlog, int window_groups)
{
    const size_t cells = (size_t)(nt / std::max(64, 1 << wlog)) << wlog;
    return (es == 2 ? 4 : 0) * cells + (es == 2 ? 8 : 16) * cells * gpv + 16 * (size_t)window_groups;
}

bool plan_norm_vec(const NormArgs& a, int vec, NormPlan& p)
{
    const int es = a.dtype == EE_I8 ? 1 : 2, cpg = a.c / a.groups;
    const int unit = cpg / gcd_i(cpg, vec);                           // columns of the smallest window of whole groups
    p.vec = vec;
    p.gpv = vec == 1 || cpg % vec == 0 ? 1 : cpg % (vec / 4) == 0 ? 4 : vec;
    const int all = a.c / vec;                                        // columns of the tensor, a multiple of unit
    auto window = [&](int want) {
        p.wv = std::min(all, unit * std::max(1, want / unit));
        p.wlog = log2_up(p.wv);
        p.windows = (all + p.wv - 1) / p.wv;
    };
    auto fits = [&] { return (1 << p.wlog) <= p.nt && norm_lds(es, p.gpv, p.nt, p.wlog, p.wv * vec / cpg) <= 65536; };
    window(vec == 1 ? 64 : 8);
    static const int forms[][2] = {{256, 1}, {256, 4}, {256, 16}, {1024, 8}, {1024, 16}};
    for (const auto& f : forms) {
        p.nt = f[0]; p.nv = f[1];
        if (!fits() || (int64_t)p.nv * (p.nt >> p.wlog) < a.pixels) continue;
        p.chunks = 1; p.chunk_pixels = a.pixels;
        return true;
    }
    for (int want = 64; want >= 8; want /= 2) {
        window(want);
        p.nt = p.wlog > 8 ? 1024 : 256;
        p.nv = 8;
        if (!fits()) continue;
        const int tile = p.nv * (p.nt >> p.wlog);                     // pixels a workgroup holds at once
        const int64_t tiles = ((int64_t)a.pixels + tile - 1) / tile;
        p.chunks = (int)std::min<int64_t>(tiles, 64);
        const int64_t per = (tiles + p.chunks - 1) / p.chunks;
        p.chunk_pixels = (int)std::min<int64_t>(per * tile, a.pixels);
        p.chunks = (int)(((int64_t)a.pixels + p.chunk_pixels - 1) / p.chunk_pixels);
        return true;
    }
    return false;
}

NormPlan plan_norm(const NormArgs& a, bool aligned)
{
    NormPlan p{};
    const int full = a.dtype == EE_I8 ? 16 : 8;
    p.ok = (aligned && a.c % full == 0 && plan_norm_vec(a, full, p)) || plan_norm_vec(a, 1, p);
    return p;
}

template <int ES, int VEC, int GPV, int NT, int NV, int MODE>
hipError_t launch_norm_form(const NormKernelArgs& k, int b, hipStream_t s)
{
    const size_t lds = norm_lds(ES, GPV, NT, k.wlog, k.cw / k.cpg);
    EE_LAUNCH((group_norm_kernel<ES, VEC, GPV, NT, NV, MODE>), dim3((unsigned)((int64_t)b * k.chunks * k.windows)), dim3(NT), (unsigned)lds, s, k);
    return hipGetLastError();
}

template <int ES, int VEC, int GPV>
hipError_t launch_norm_gpv(const NormKernelArgs& k, const NormPlan& p, int b, hipStream_t s)
{
    if (p.chunks > 1) {
        if (p.nt == 256) {
            const hipError_t e = launch_norm_form<ES, VEC, GPV, 256, 8, 1>(k, b, s);
            return e == hipSuccess ? launch_norm_form<ES, VEC, GPV, 256, 8, 2>(k, b, s) : e;
        }
        const hipError_t e = launch_norm_form<ES, VEC, GPV, 1024, 8, 1>(k, b, s);
        return e == hipSuccess ? launch_norm_form<ES, VEC, GPV, 1024, 8, 2>(k, b, s) : e;
    }
    if (p.nt == 256) return p.nv == 1 ? launch_norm_form<ES, VEC, GPV, 256, 1, 0>(k, b, s) : p.nv == 4 ? launch_norm_form<ES, VEC, GPV, 256, 4, 0>(k, b, s) : launch_norm_form<ES, VEC, GPV, 256, 16, 0>(k, b, s);
    return p.nv == 8 ? launch_norm_form<ES, VEC, GPV, 1024, 8, 0>(k, b, s) : launch_norm_form<ES, VEC, GPV, 1024, 16, 0>(k, b, s);
}

bool norm_aligned(const NormArgs& a)
{
    const int full = a.dtype == EE_I8 ? 16 : 8;
    auto ok = [&](const void* p, int64_t sample, int64_t pixel) { return ((uintptr_t)p & 15) == 0 && sample % full == 0 && pixel % full == 0; };
    return ok(a.x, a.x_sample, a.x_pixel) && ok(a.y, a.y_sample, a.y_pixel) && (!a.res || ok(a.res, a.res_sample, a.res_pixel));
}

}  // namespace

bool group_norm_supported(const NormArgs& a) { return plan_norm(a, norm_aligned(a)).ok; }

bool group_norm_grid_fits(const NormArgs& a)
{
    const NormPlan p = plan_norm(a, norm_aligned(a));
    return (int64_t)a.b * p.chunks * p.windows < 1ll << 31;
}

// a call whose alignment is not known yet may be cut either way
size_t group_norm_workspace(const NormArgs& a)
{
    size_t most = 0;
    for (const bool aligned : {false, true}) {
        const NormPlan p = plan_norm(a, aligned);
        if (p.ok && p.chunks > 1) most = std::max(most, (size_t)a.b * p.chunks * a.groups * 16);
    }
    return most;
}

hipError_t launch_group_norm(const NormArgs& a, void* workspace, hipStream_t s)
{
    const NormPlan p = plan_norm(a, norm_aligned(a));
    NormKernelArgs k{};
    k.x = a.x; k.res = a.res; k.y = a.y; k.weight = a.weight; k.bias = a.bias; k.part = workspace;
    k.x_sample = a.x_sample; k.x_pixel = a.x_pixel; k.r_sample = a.res_sample; k.r_pixel = a.res_pixel; k.y_sample = a.y_sample; k.y_pixel = a.y_pixel;
    k.pixels = a.pixels; k.c = a.c; k.groups = a.groups; k.cpg = a.c / a.groups;
    k.cw = p.wv * p.vec; k.wlog = p.wlog; k.windows = p.windows; k.chunks = p.chunks; k.chunk_pixels = p.chunk_pixels;
    k.eps = a.eps; k.act = a.act;
    k.out_scale = std::ldexp(1.0, a.frac_bits); k.res_scale = std::ldexp(1.0, a.res_shift);
    k.lo = a.act == EE_ACT_NONE ? -128 : 0;
    k.hi = a.act == EE_ACT_RELU6 ? (int)std::min(127.0, 6.0 * k.out_scale) : 127;
    if (a.dtype == EE_I8) {
        if (p.vec == 1) return launch_norm_gpv<1, 1, 1>(k, p, a.b, s);
        return p.gpv == 1 ? launch_norm_gpv<1, 16, 1>(k, p, a.b, s) : p.gpv == 4 ? launch_norm_gpv<1, 16, 4>(k, p, a.b, s) : launch_norm_gpv<1, 16, 16>(k, p, a.b, s);
    }
    if (p.vec == 1) return launch_norm_gpv<2, 1, 1>(k, p, a.b, s);
    return p.gpv == 1 ? launch_norm_gpv<2, 8, 1>(k, p, a.b, s) : p.gpv == 4 ? launch_norm_gpv<2, 8, 4>(k, p, a.b, s) : launch_norm_gpv<2, 8, 8>(k, p, a.b, s);
}

}  // namespace ee
