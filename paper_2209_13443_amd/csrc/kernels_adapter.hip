// A shared projection with each request's low-rank adapter beside it (bf16), for gfx950.
//
//   y[m][o] = sum_c x[m][c] W[o][c] + bias[o] + sum_r B_a[o][r] u[m][r],   u[m][r] = scale_a sum_c A_a[r][c] x[m][c],   a: the adapter of row m, or none
//
// Two launches.  The first computes u (adapter_shrink_kernel) and the adapter of every row; u is kept as the sum of bf16 numbers (head and remainders:
// two of them, relative error 2^-18, for bf16 results, three, 2^-26, for float ones), so that the second half of an adapter runs on the matrix cores as well.  The second is the projection, with the adapters as
// further steps of its reduction: for each adapter among a wavefront's rows, the rows of others read zeros.
//
// Weights are laid out once as operands of the matrix instructions: blocks of 32 rows x steps of 16 columns, [lane][8]: lane l holds row l % 32, columns
// 8 (l / 32) .. + 7.  A wavefront reads its block as one contiguous KiB per step.  Rows and columns are padded with zeros.
#include <algorithm>

#include "ee_internal.hpp"
#include "igemm_device.hpp"

namespace ee {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));

struct AdapterKernelArgs {
    const uint16_t* x; const uint16_t* w; const float* bias; void* y;
    const uint16_t* a; const uint16_t* b; const float* scale;        // the adapters: first and second halves, factors
    const int* ids; const int* offsets; int* row_ids; uint16_t* u;
    const uint16_t* zeros;                                           // 16 readable zero bytes
    int64_t ldx, ldy;
    int rows, slots, per, ci, co, kp, np, rp, adapters, out_f32, parts;      // parts: bf16 numbers that make up an element of u
};

// ---- layouts -----------------------------------------------------------------------------------------------------------------
// dst[row block][step][lane][8] of src[rows][cols] (zeros outside), blocks x steps of them
__global__ __launch_bounds__(256) void adapter_pack_kernel(const uint16_t* src, int64_t ld, int rows, int cols, uint16_t* dst, int blocks, int steps)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;                 // one 16-byte piece
    if (at >= (int64_t)blocks * steps * 64) return;
    const int lane = (int)(at & 63), row = (int)(at / (64 * (int64_t)steps)) * 32 + (lane & 31), col = (int)(at / 64 % steps) * 16 + (lane >> 5) * 8;
    uint16_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = row < rows && col + e < cols ? src[row * ld + col + e] : (uint16_t)0;
    v4i o;
    __builtin_memcpy(&o, v, 16);
    *(v4i*)(dst + at * 8) = o;
}

__global__ __launch_bounds__(256) void adapter_bias_kernel(const float* src, int n, float* dst, int n_pad)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n_pad) dst[i] = src && i < n ? src[i] : 0.f;
}
__global__ void adapter_scale_kernel(float* dst, float v) { *dst = v; }

// rows that are no whole 16-byte pieces: dst[rows][cols_pad] with zeros behind a row's end
__global__ __launch_bounds__(256) void adapter_rows_kernel(const uint16_t* src, int64_t ld, int rows, int cols, uint16_t* dst, int cols_pad)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= (int64_t)rows * cols_pad) return;
    const int64_t row = at / cols_pad;
    const int col = (int)(at - row * cols_pad);
    dst[at] = col < cols ? src[row * ld + col] : (uint16_t)0;
}

// ---- first halves ------------------------------------------------------------------------------------------------------------
// the adapter of a row; -1: none, -2: the row is behind the last slot's
__device__ __forceinline__ int adapter_of(const AdapterKernelArgs& a, int row)
{
    int slot;
    if (a.offsets) {
        if (row < a.offsets[0] || row >= a.offsets[a.slots]) return -2;
        int lo = 0, hi = a.slots;                          // offsets[lo] <= row < offsets[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.offsets[mid] <= row) lo = mid;
            else hi = mid;
        }
        slot = lo;
    } else slot = row / a.per;
    const int id = a.ids ? a.ids[slot] : -1;
    return (unsigned)id < (unsigned)a.adapters ? id : -1;
}

// u of 16 rows: the wavefronts share the columns of x; 32 rank rows at a time
__global__ __launch_bounds__(256) void adapter_shrink_kernel(AdapterKernelArgs a)
{
    __shared__ float l_sum[4][32][33];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r0 = blockIdx.x * 32;
    const int m = r0 + (lane & 31), hi = lane >> 5;
    const int id = m < a.rows ? adapter_of(a, m) : -2;
    if (tid < 32 && m < a.rows) a.row_ids[m] = id;
    const uint16_t* const x = a.x + (int64_t)min(m, a.rows - 1) * a.ldx;
    const int steps = a.kp / 16;
    unsigned pending = (unsigned)__ballot(lane < 32 && id >= 0);
    while (pending) {
        const int who = __builtin_ctz(pending), ad = __builtin_amdgcn_readlane(id, who);
        pending &= ~(unsigned)__ballot(lane < 32 && id == ad);
        const float scale = a.scale[ad];
        for (int rb = 0; rb < a.rp; rb += 32) {
            const uint16_t* const w = a.a + ((int64_t)ad * (a.rp / 32) + rb / 32) * steps * 512 + lane * 8;
            v16f acc = {};
            for (int s = wave; s < steps; s += 4) {
                const int col = s * 16 + hi * 8;
                const v4i xv = col < a.ci ? *(const v4i*)(x + col) : v4i{0, 0, 0, 0};
                const v4i wv = *(const v4i*)(w + (int64_t)s * 512);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, wv), __builtin_bit_cast(v8bf, xv), acc, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) l_sum[wave][lane & 31][8 * (e >> 2) + 4 * hi + (e & 3)] = acc[e];
            __syncthreads();
            for (int i = tid; i < 1024; i += 256) {
                const int row = i >> 5, r = i & 31;
                if (__shfl(id, row) == ad) {
                    float v = scale * (l_sum[0][row][r] + l_sum[1][row][r] + l_sum[2][row][r] + l_sum[3][row][r]);
                    uint16_t* const u = a.u + (int64_t)(r0 + row) * a.parts * a.rp + rb + r;
                    for (int k = 0; k < a.parts; ++k) {
                        const __bf16 h = (__bf16)v;
                        u[k * a.rp] = __builtin_bit_cast(uint16_t, h);
                        v -= (float)h;
                    }
                }
            }
            __syncthreads();
        }
    }
}

// ---- the projection ------------------------------------------------------------------------------------------------------------
// WM x WN wavefronts, each with MB x NB blocks of 32 rows x 32 outputs.  Rows of x go through LDS, 64 columns at a time, a ring of three;
// weights straight into registers, eight steps ahead.
template <int MB, int NB, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void adapter_project_kernel(AdapterKernelArgs a, int gn)
{
    constexpr int NT = 64 * WM * WN, BM = 32 * MB * WM, COPIES = BM * 8 / NT, WR = 8;
    static_assert(COPIES * NT == BM * 8);
    __shared__ __attribute__((aligned(16))) unsigned char lds[3 * BM * 128];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hi = lane >> 5, frow = lane & 31;
    const int wm = wave % WM, wn = wave / WM;
    const int mt = blockIdx.x / gn, nt = blockIdx.x % gn, m0 = mt * BM, n0 = (nt * WN + wn) * NB;      // n0: first block of 32 outputs
    const unsigned lds0 = lds_addr(lds);
    const int iters = a.kp / 64, steps = iters * 4, blocks = a.np / 32;
    // copies: LDS position q = 8 row + pos holds chunk pos ^ (row & 7) of the row
    const uint16_t* src[COPIES];
    int chunk[COPIES];
#pragma unroll
    for (int j = 0; j < COPIES; ++j) {
        const int q = tid + NT * j, row = q >> 3;
        chunk[j] = (q & 7) ^ (row & 7);
        src[j] = a.x + (int64_t)min(m0 + row, a.rows - 1) * a.ldx;
    }
    auto copy = [&](int it) {
        const int slot = it % 3;
#pragma unroll
        for (int j = 0; j < COPIES; ++j) {
            const int col = it * 64 + chunk[j] * 8;
            dma16(lds0 + (unsigned)(slot * BM * 128 + (NT * j + 64 * wave) * 16), it < iters && col < a.ci ? src[j] + col : a.zeros);
        }
    };
    const uint16_t* w[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) w[n] = a.w + (int64_t)min(n0 + n, blocks - 1) * steps * 512 + lane * 8;
    auto weight = [&](int n, int s) { return *(const v4i*)(w[n] + (int64_t)min(s, steps - 1) * 512); };
    v4i wr[WR][NB];
    copy(0);
#pragma unroll
    for (int s = 0; s < WR; ++s)
#pragma unroll
        for (int n = 0; n < NB; ++n) wr[s][n] = weight(n, s);
    copy(1);
    v16f acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[i][n] = v16f{};
    auto iteration = [&](auto half, int it) {
        constexpr int H = decltype(half)::value * 4;
        // copies newer than this iteration's: one iteration's, and 4 NB weights of each of the last two iterations at least
        wait_all_then_barrier<COPIES + 4 * NB>();
        copy(it + 2);
        const unsigned char* const base = lds + (it % 3) * BM * 128 + (wm * MB * 32 + frow) * 128;
        static_for<4>([&](auto ks_tag) {
            constexpr int KS = decltype(ks_tag)::value;
            v4i xv[MB];
#pragma unroll
            for (int i = 0; i < MB; ++i) xv[i] = *(const v4i*)(base + i * 4096 + (((2 * KS + hi) ^ (frow & 7)) << 4));
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int n = 0; n < NB; ++n)
                    acc[i][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, wr[H + KS][n]), __builtin_bit_cast(v8bf, xv[i]), acc[i][n], 0, 0, 0);
#pragma unroll
            for (int n = 0; n < NB; ++n) wr[H + KS][n] = weight(n, it * 4 + KS + WR);
        });
    };
    int it = 0;
    for (; it + 2 <= iters; it += 2) {
        iteration(std::integral_constant<int, 0>{}, it);
        iteration(std::integral_constant<int, 1>{}, it + 1);
    }
    if (it < iters) iteration(std::integral_constant<int, 0>{}, it);

    // ---- adapters: further reductions (one per part of u) over the rank for each adapter among the rows ----------------
    int id[MB];
    unsigned pending[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int m = m0 + (wm * MB + i) * 32 + frow;
        id[i] = m < a.rows ? a.row_ids[m] : -2;
        pending[i] = (unsigned)__ballot(lane < 32 && id[i] >= 0);
    }
    for (;;) {
        int ad = -1;
#pragma unroll
        for (int i = 0; i < MB; ++i)
            if (ad < 0 && pending[i]) ad = __builtin_amdgcn_readlane(id[i], __builtin_ctz(pending[i]));
        if (ad < 0) break;
        const uint16_t* const wb = a.b + (int64_t)ad * blocks * (a.rp / 16) * 512 + lane * 8;
        for (int r = 0; r < a.rp; r += 16) {
            v4i bv[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n) bv[n] = *(const v4i*)(wb + ((int64_t)min(n0 + n, blocks - 1) * (a.rp / 16) + r / 16) * 512);
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const uint16_t* const u = a.u + (int64_t)(m0 + (wm * MB + i) * 32 + frow) * a.parts * a.rp + r + hi * 8;
                for (int part = 0; part < a.parts; ++part) {
                    const v4i uv = id[i] == ad ? *(const v4i*)(u + part * a.rp) : v4i{0, 0, 0, 0};
#pragma unroll
                    for (int n = 0; n < NB; ++n)
                        acc[i][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, bv[n]), __builtin_bit_cast(v8bf, uv), acc[i][n], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < MB; ++i) pending[i] &= ~(unsigned)__ballot(lane < 32 && id[i] == ad);
    }

    // ---- results: lane: row frow of a block, outputs 8 q + 4 hi + 0..3 of a block ---------------------------------------------
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int m = m0 + (wm * MB + i) * 32 + frow;
        if (m >= a.rows || id[i] == -2) continue;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int o = (n0 + n) * 32 + 8 * q + 4 * hi + e;
                    if (o >= a.co) continue;
                    const float v = acc[i][n][4 * q + e] + a.bias[o];
                    if (a.out_f32) ((float*)a.y)[m * a.ldy + o] = v;
                    else ((uint16_t*)a.y)[m * a.ldy + o] = __builtin_bit_cast(uint16_t, (__bf16)v);
                }
    }
}

int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

struct AdapterSizes {       // in bytes; everything a multiple of 256
    int64_t kp, np, rp, w, bias, a, b, scale;
    explicit AdapterSizes(const AdapterDims& d)
    {
        kp = up(d.ci, 64); np = up(d.co, 32); rp = up(std::max(d.rank, 1), 32);
        w = 2 * np * kp; bias = up(4 * np, 256);
        a = 2 * rp * kp * d.adapters; b = 2 * np * rp * d.adapters; scale = up(4ll * d.adapters, 256);
    }
};

hipError_t pack(const void* src, int64_t ld, int rows, int cols, void* dst, int64_t blocks, int64_t steps, hipStream_t s)
{
    EE_LAUNCH(adapter_pack_kernel, dim3((unsigned)((blocks * steps * 64 + 255) / 256)), dim3(256), 0, s, (const uint16_t*)src, ld, rows, cols, (uint16_t*)dst, (int)blocks, (int)steps);
    return hipGetLastError();
}

}  // namespace

// packed weights: operands | bias | 256 zero bytes; adapters: first halves | second halves | factors
int64_t adapter_weight_bytes(const AdapterDims& d) { const AdapterSizes z(d); return z.w + z.bias + 256; }
int64_t adapter_pool_bytes(const AdapterDims& d) { const AdapterSizes z(d); return std::max<int64_t>(256, z.a + z.b + z.scale); }
// u | adapters of the rows | a padded copy of x where its rows are no whole 16-byte pieces
int64_t adapter_workspace(const AdapterDims& d, int64_t rows) { const AdapterSizes z(d); return up(6 * rows * z.rp, 256) + up(4 * rows, 256) + (rows * z.kp * 2); }

hipError_t launch_adapter_pack(const AdapterDims& d, const void* w, int64_t ldw, const float* bias, void* packed, hipStream_t s)
{
    const AdapterSizes z(d);
    const hipError_t e = pack(w, ldw, d.co, d.ci, packed, z.np / 32, z.kp / 16, s);
    if (e != hipSuccess) return e;
    const int n = (int)((z.bias + 256) / 4);                                     // the zeros behind the bias as well
    EE_LAUNCH(adapter_bias_kernel, dim3((n + 255) / 256), dim3(256), 0, s, bias, d.co, (float*)((char*)packed + z.w), n);
    return hipGetLastError();
}

hipError_t launch_adapter_load(const AdapterDims& d, int i, int rank, const void* a, int64_t lda, const void* b, int64_t ldb, float scale, void* pool, hipStream_t s)
{
    const AdapterSizes z(d);
    char* const p = (char*)pool;
    hipError_t e = pack(a, lda, rank, d.ci, p + z.a / std::max(d.adapters, 1) * i, z.rp / 32, z.kp / 16, s);
    if (e == hipSuccess) e = pack(b, ldb, d.co, rank, p + z.a + z.b / d.adapters * i, z.np / 32, z.rp / 16, s);
    if (e != hipSuccess) return e;
    EE_LAUNCH(adapter_scale_kernel, dim3(1), dim3(1), 0, s, (float*)(p + z.a + z.b) + i, scale);
    return hipGetLastError();
}

hipError_t launch_adapter_project(const AdapterDims& d, const AdapterCall& c, hipStream_t s)
{
    const AdapterSizes z(d);
    AdapterKernelArgs k{};
    k.x = (const uint16_t*)c.x; k.ldx = c.ldx; k.y = c.y; k.ldy = c.ldy; k.out_f32 = c.out_f32;
    k.w = (const uint16_t*)c.packed; k.bias = (const float*)((const char*)c.packed + z.w); k.zeros = (const uint16_t*)((const char*)c.packed + z.w + z.bias);
    k.a = (const uint16_t*)c.pool; k.b = (const uint16_t*)((const char*)c.pool + z.a); k.scale = (const float*)((const char*)c.pool + z.a + z.b);
    k.ids = c.ids; k.offsets = c.offsets; k.rows = c.rows; k.slots = c.slots; k.per = c.per;
    k.ci = d.ci; k.co = d.co; k.kp = (int)z.kp; k.np = (int)z.np; k.rp = (int)z.rp; k.adapters = d.adapters; k.parts = c.out_f32 ? 3 : 2;
    char* ws = (char*)c.workspace;
    k.u = (uint16_t*)ws; ws += up(6ll * c.rows * z.rp, 256);
    k.row_ids = (int*)ws; ws += up(4ll * c.rows, 256);
    if (((uintptr_t)c.x & 15) || c.ldx % 8 || d.ci % 8) {
        EE_LAUNCH(adapter_rows_kernel, dim3((unsigned)(((int64_t)c.rows * z.kp + 255) / 256)), dim3(256), 0, s, k.x, k.ldx, c.rows, d.ci, (uint16_t*)ws, k.kp);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        k.x = (const uint16_t*)ws; k.ldx = k.kp; k.ci = k.kp;
    }
    EE_LAUNCH(adapter_shrink_kernel, dim3((c.rows + 31) / 32), dim3(256), 0, s, k);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (c.rows <= 64) {
        const int gn = (int)(z.np + 127) / 128;
        EE_LAUNCH((adapter_project_kernel<1, 1, 1, 4>), dim3((unsigned)((c.rows + 31) / 32 * gn)), dim3(256), 0, s, k, gn);
    } else {
        const int gn = (int)(z.np + 127) / 128;
        EE_LAUNCH((adapter_project_kernel<2, 2, 2, 2>), dim3((unsigned)((c.rows + 127) / 128 * gn)), dim3(256), 0, s, k, gn);
    }
    return hipGetLastError();
}

}  // namespace ee
