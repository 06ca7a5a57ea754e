// A shared projection with each request's low-rank adapter beside it (bf16), for gfx950.
//
//   y[m][o] = sum_c x[m][c] W[o][c] + bias[o] + sum_r B_a[o][r] u[m][r],   u[m][r] = scale_a sum_c A_a[r][c] x[m][c],   a: the adapter of row m, or none
//
// Two launches, or, for long slots and few outputs, one.  The first computes u (adapter_shrink_kernel) and the adapter of every row; u is kept as the sum of bf16 numbers, a head and remainders, so that
// the second half of an adapter runs on the matrix cores as well: three of them for float results, which hold all of a float, two for bf16 results, relative error 2^-18.  That is a 1,024th of a result's own
// rounding and, where terms cancel, what float sums of thousands of them lose as well; a third number for these too, us: 4096 -> 4096, 128 rows of 24 adapters of rank 16 32.7 / 38.0, 8,000 rows of rank 64 242 / 253, 12,544 rows
// 1024 -> 256 of rank 32 21.0 / 21.7, 4,096 rows 1024 -> 1024 of 32 adapters 27.6 / 30.2.  Few rows keep u in float.  The second launch is the projection, with the adapters as
// further steps of its reduction: for each adapter among a tile's rows, the rows of others read zeros.  A second half that has infinities or NaN, which zeros times it would give to the rows of
// others, is no step: its own rows add it element by element.
//
// Weights are laid out once as operands of the matrix instructions: blocks of 32 rows x steps of 16 columns, [lane][8]: lane l holds row l % 32, columns
// 8 (l / 32) .. + 7.  A wavefront reads its block as one contiguous KiB per step.  Rows and columns are padded with zeros.
#include <algorithm>

#include "../ee_internal.hpp"
#include "../igemm_device.hpp"

namespace ee {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));

struct AdapterKernelArgs {
    const uint16_t* x; const uint16_t* w; const float* bias; void* y;
    const uint16_t* a; const uint16_t* b; const float* scale; const int* info;        // the adapters: first and second halves, factors, 2 rank + whether the second half has infinities or NaN
    const int* ids; const int* offsets; int* row_ids; uint16_t* u;
    const uint16_t* zeros;                                           // 16 readable zero bytes
    int64_t ldx, ldy;
    int rows, slots, per, ci, co, kp, np, rp, ra, adapters, out_f32, parts, splits;      // parts: bf16 numbers that make up an element of u; 0: it is `splits` floats, to be added
};

// ---- layouts -----------------------------------------------------------------------------------------------------------------
enum { ODD = 1 << 30 };              // in the adapter of a row: its second half has infinities or NaN

// A launch has less than 2^32 threads, and layouts may have more elements: these kernels' threads take every so many'th of them
unsigned blocks_of(int64_t threads) { return (unsigned)std::min<int64_t>((threads + 255) / 256, 1 << 23); }

// dst[row block][step][lane][8] of src[rows][cols] (zeros outside), blocks x steps of them.  An adapter's first half: *info becomes 2 rank, *scale its factor; its second half behind that (scale null):
// the last bit of *info is set if an element is not finite
__global__ __launch_bounds__(256) void adapter_pack_kernel(const uint16_t* src, int64_t ld, int rows, int cols, uint16_t* dst, int blocks, int steps, int* info, int rank, float* scale, float factor)
{
    if (scale && blockIdx.x == 0 && threadIdx.x == 0) {
        *info = 2 * rank;
        *scale = factor;
    }
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < (int64_t)blocks * steps * 64; at += (int64_t)gridDim.x * 256) {      // 16-byte pieces
        const int lane = (int)(at & 63), row = (int)(at / (64 * (int64_t)steps)) * 32 + (lane & 31), col = (int)(at / 64 % steps) * 16 + (lane >> 5) * 8;
        uint16_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = row < rows && col + e < cols ? src[row * ld + col + e] : (uint16_t)0;
        if (info && !scale) {
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) odd |= (v[e] & 0x7F80) == 0x7F80;
            if (odd) *info = 2 * rank + 1;                 // by all that find one
        }
        v4i o;
        __builtin_memcpy(&o, v, 16);
        *(v4i*)(dst + at * 8) = o;
    }
}

__global__ __launch_bounds__(256) void adapter_bias_kernel(const float* src, int n, float* dst, int n_pad)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n_pad) dst[i] = src && i < n ? src[i] : 0.f;
}

// rows that are no whole 16-byte pieces: dst[rows][cols_pad] with zeros behind a row's end
__global__ __launch_bounds__(256) void adapter_rows_kernel(const uint16_t* src, int64_t ld, int rows, int cols, uint16_t* dst, int cols_pad)
{
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < (int64_t)rows * cols_pad; at += (int64_t)gridDim.x * 256) {
        const int64_t row = at / cols_pad;
        const int col = (int)(at - row * cols_pad);
        dst[at] = col < cols ? src[row * ld + col] : (uint16_t)0;
    }
}

// ---- first halves ------------------------------------------------------------------------------------------------------------
// the adapter of a row; -1: none, -2: the row is behind the last slot's
__device__ __forceinline__ int adapter_of(const AdapterKernelArgs& a, int row, const int* offsets)
{
    int slot;
    if (offsets) {
        if (row < offsets[0] || row >= offsets[a.slots]) return -2;
        int lo = 0, hi = a.slots;                          // offsets[lo] <= row < offsets[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (offsets[mid] <= row) lo = mid;
            else hi = mid;
        }
        slot = lo;
    } else slot = row / a.per;
    const int id = a.ids ? a.ids[slot] : -1;
    return (unsigned)id < (unsigned)a.adapters ? id : -1;
}

enum { SPLITS = 4 };                 // few rows: workgroups that may share an adapter's first half
enum { OFFSETS_LDS = 2048 };         // up to so many offsets are searched in LDS, more where they lie

// u of ROWS rows (16 or 32: a matrix instruction's), RT x ROWS rows of the adapters' first halves at a time.  Eight wavefronts share the columns of x, 64 at a time, and add up through LDS.
// 32 rows (many of them): a wavefront loads whole lines of 8 rows and turns them into operands through its own part of LDS; 16 rows: straight from memory, where latency counts.
// Workgroup `ord` of `ords` takes every ords-th of the different adapters among the rows; neighbours have the same ord, or the ones with nothing to do would leave whole XCDs idle
// (8,000 rows, 4096 -> 64: 135 us, all of the work on one XCD).
template <int ROWS, int RT>
__global__ __launch_bounds__(512) void adapter_shrink_kernel(AdapterKernelArgs a, int blocks, int ords)
{
    const int split = blockIdx.z;
    constexpr int NW = 8, KB = 512 / ROWS, GU = 64 / KB, XL = ROWS == 32 ? 4 : GU;       // KB: columns of a matrix instruction, GU: of them in 64, XL: loads of x a lane makes for them
    typedef typename std::conditional<ROWS == 32, v16f, v4f>::type acc_t;
    constexpr int SUM = NW * ROWS * (ROWS + 1) * 4, TURN = ROWS == 32 ? NW * 4096 : 0;
    __shared__ __attribute__((aligned(16))) unsigned char l_buf[SUM > TURN ? SUM : TURN];
    __shared__ int l_id[ROWS];
    __shared__ int l_off[OFFSETS_LDS];
    float (*const l_sum)[ROWS][ROWS + 1] = (float (*)[ROWS][ROWS + 1])l_buf;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), frow = lane & (ROWS - 1), kq = lane / ROWS;
    const int ord = blockIdx.x / blocks, block = blockIdx.x - ord * blocks, r0 = block * ROWS, rank0 = blockIdx.y * RT * ROWS;
    const bool in_lds = a.offsets && a.slots < OFFSETS_LDS;
    if (in_lds) {
        for (int i = tid; i <= a.slots; i += 512) l_off[i] = a.offsets[i];
        __syncthreads();
    }
    if (tid < ROWS) {
        const int m = r0 + tid, id = m < a.rows ? adapter_of(a, m, in_lds ? l_off : a.offsets) : -2;
        l_id[tid] = id;
        if (m < a.rows && ord == 0 && blockIdx.y == 0 && split == 0) a.row_ids[m] = id >= 0 && (a.info[id] & 1) ? id | ODD : id;
    }
    __syncthreads();
    const int id = l_id[frow];
    const int steps16 = a.kp / 16, chunks = a.kp / 64;
    // 32 rows: load j is of rows 8 j + lane / 8, 16 bytes each; in LDS piece c of row r is at c ^ (r / 2 & 7): 16 rows in 16 different quads of banks
    const uint16_t* x[XL];
    int xcol[XL];
#pragma unroll
    for (int j = 0; j < XL; ++j) {
        const int row = ROWS == 32 ? 8 * j + (lane >> 3) : frow;
        xcol[j] = ROWS == 32 ? (lane & 7) * 8 : j * KB + kq * 8;
        x[j] = a.x + (int64_t)min(r0 + row, a.rows - 1) * a.ldx + xcol[j];
    }
    unsigned char* const turn = l_buf + wave * 4096;
    unsigned pending = (unsigned)__ballot(lane < ROWS && id >= 0);
    for (int k = 0; pending; ++k) {
        const int ad = __builtin_amdgcn_readlane(id, __builtin_ctz(pending));
        pending &= ~(unsigned)__ballot(lane < ROWS && id == ad);
        if (k % ords != ord) continue;
        // operands: 32 rank rows x 16 columns are 64 pieces, columns 8 (piece / 32) .., row piece % 32
        const uint16_t* w[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int r = min(rank0 + t * ROWS, a.ra - ROWS);
            w[t] = a.a + ((int64_t)ad * (a.ra / 32) + r / 32) * steps16 * 512 + (ROWS == 32 ? lane * 8 : (kq >> 1) * 512 + ((kq & 1) * 32 + (r & 16) + frow) * 8);
        }
        const float scale = a.scale[ad];
        const int rank = a.info[ad] >> 1;
        acc_t acc[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t] = acc_t{};
        v4i xv[2][XL], wv[2][RT][GU];
        auto load = [&](auto buf, int c) {
            constexpr int B = decltype(buf)::value;
#pragma unroll
            for (int j = 0; j < XL; ++j) xv[B][j] = c < chunks && c * 64 + xcol[j] < a.ci ? *(const v4i*)(x[j] + c * 64) : v4i{0, 0, 0, 0};
#pragma unroll
            for (int u = 0; u < GU; ++u)
#pragma unroll
                for (int t = 0; t < RT; ++t) wv[B][t][u] = *(const v4i*)(w[t] + (int64_t)(min(c, chunks - 1) * 64 + u * KB) / 16 * 512);
        };
        auto multiply = [&](auto buf) {
            constexpr int B = decltype(buf)::value;
            v4i xo[GU];
            if constexpr (ROWS == 32) {
#pragma unroll
                for (int j = 0; j < XL; ++j) {
                    const int row = 8 * j + (lane >> 3);
                    *(v4i*)(turn + row * 128 + (((lane & 7) ^ (row >> 1 & 7)) << 4)) = xv[B][j];
                }
#pragma unroll
                for (int u = 0; u < GU; ++u) xo[u] = *(const v4i*)(turn + frow * 128 + (((2 * u + kq) ^ (frow >> 1 & 7)) << 4));
            } else
#pragma unroll
                for (int u = 0; u < GU; ++u) xo[u] = xv[B][u];
#pragma unroll
            for (int u = 0; u < GU; ++u)
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    if constexpr (ROWS == 32) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, wv[B][t][u]), __builtin_bit_cast(v8bf, xo[u]), acc[t], 0, 0, 0);
                    else acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, wv[B][t][u]), __builtin_bit_cast(v8bf, xo[u]), acc[t], 0, 0, 0);
                }
        };
        const int next = NW * a.splits;
        load(std::integral_constant<int, 0>{}, wave + NW * split);
        int c = wave + NW * split;
        for (; c + next < chunks; c += 2 * next) {
            load(std::integral_constant<int, 1>{}, c + next);
            multiply(std::integral_constant<int, 0>{});
            load(std::integral_constant<int, 0>{}, c + 2 * next);
            multiply(std::integral_constant<int, 1>{});
        }
        if (c < chunks) multiply(std::integral_constant<int, 0>{});              // not past the end: x is zeros there, but the adapter may have infinities
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            if (rank0 + t * ROWS >= a.rp) break;
            __syncthreads();                                                     // the sums lie over the operands
#pragma unroll
            for (int e = 0; e < (ROWS == 32 ? 16 : 4); ++e) l_sum[wave][frow][ROWS == 32 ? 8 * (e >> 2) + 4 * kq + (e & 3) : 4 * kq + e] = acc[t][e];
            __syncthreads();
            for (int i = tid; i < ROWS * ROWS; i += 512) {
                const int row = i / ROWS, r = i % ROWS;
                if (l_id[row] == ad && rank0 + t * ROWS + r < a.rp) {
                    float v = 0.f;
#pragma unroll
                    for (int q = 0; q < NW; ++q) v += l_sum[q][row][r];
                    v = rank0 + t * ROWS + r < rank ? v * scale : 0.f;           // behind the rank a row's infinity times zeros is NaN
                    if (a.parts == 0) ((float*)a.u)[((int64_t)split * a.rows + r0 + row) * a.rp + rank0 + t * ROWS + r] = v;
                    else {
                        uint16_t* const u = a.u + (int64_t)(r0 + row) * a.parts * a.rp + rank0 + t * ROWS + r;
                        for (int p = 0; p < a.parts; ++p) {
                            const __bf16 h = (__bf16)v;
                            u[p * a.rp] = __builtin_bit_cast(uint16_t, h);
                            v = __builtin_isfinite((float)h) ? v - (float)h : 0.f;
                        }
                    }
                }
            }
        }
        __syncthreads();
    }
}

// ---- the projection, few rows --------------------------------------------------------------------------------------------------
// A workgroup has 16 outputs and up to 16 MT rows; its eight wavefronts share the reduction, 64 columns at a time, and the adapters, and add up through LDS.  Nothing is staged: a weight is
// used once.  Reading W is what it is for.
template <int MT>
__global__ __launch_bounds__(512) void adapter_rows_project_kernel(AdapterKernelArgs a, int gn)
{
    constexpr int NW = 8;
    __shared__ float l_sum[NW][16 * MT][17];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), frow = lane & 15, kq = lane >> 4;
    const int nb = blockIdx.x % gn, m0 = blockIdx.x / gn * 16 * MT;          // nb: block of 16 outputs
    const int steps16 = a.kp / 16, chunks = a.kp / 64;
    const int piece = ((kq & 1) * 32 + (nb & 1) * 16 + frow) * 8;
    const uint16_t* const w = a.w + (int64_t)(nb >> 1) * steps16 * 512 + (kq >> 1) * 512 + piece;
    const uint16_t* x[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) x[i] = a.x + (int64_t)min(m0 + 16 * i + frow, a.rows - 1) * a.ldx + kq * 8;
    v4f acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = v4f{};
    v4i wv[2][2], xv[2][2][MT];
    auto load = [&](auto buf, int c) {
        constexpr int B = decltype(buf)::value;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int col = c * 64 + u * 32;
            wv[B][u] = *(const v4i*)(w + (int64_t)(min(c, chunks - 1) * 4 + 2 * u) * 512);
            const bool in = c < chunks && col + kq * 8 < a.ci;
#pragma unroll
            for (int i = 0; i < MT; ++i) xv[B][u][i] = in ? *(const v4i*)(x[i] + col) : v4i{0, 0, 0, 0};
        }
    };
    auto multiply = [&](auto buf) {
        constexpr int B = decltype(buf)::value;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < MT; ++i)
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, wv[B][u]), __builtin_bit_cast(v8bf, xv[B][u][i]), acc[i], 0, 0, 0);
    };
    // outputs a thread finishes: row tid / 16 + 32 j, output tid % 16 of the block; their adapters in vector arithmetic, 16 of the rank at a time, the first of them loaded up front
    constexpr int J = MT == 4 ? 2 : 1;
    const int o = nb * 16 + (tid & 15);
    int id[J];
    const float* u[J];
    const uint16_t* b[J];
    float uv[J][SPLITS];
    v4i bv[J][2];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int row = (tid >> 4) + 32 * j, m = m0 + row;
        id[j] = row < 16 * MT && m < a.rows ? a.row_ids ? a.row_ids[m] : -1 : -2;
        if (id[j] >= 0) id[j] &= ~ODD;                     // adapters are taken by row here
        u[j] = (const float*)a.u + (int64_t)m * a.rp + (tid & 15);
        b[j] = a.b + (((int64_t)id[j] * (a.np / 32) + (nb >> 1)) * (a.rp / 16) * 64 + (nb & 1) * 16 + (tid & 15)) * 8;
    }
    auto load_adapter = [&](int j, int r) {
        if (id[j] < 0) return;
#pragma unroll
        for (int e = 0; e < SPLITS; ++e) uv[j][e] = e < a.splits ? u[j][e * (int64_t)a.rows * a.rp + r] : 0.f;
#pragma unroll
        for (int e = 0; e < 2; ++e) bv[j][e] = *(const v4i*)(b[j] + (r / 16 * 64 + e * 32) * 8);
    };
    load(std::integral_constant<int, 0>{}, wave);
#pragma unroll
    for (int j = 0; j < J; ++j) load_adapter(j, 0);
    const float bias = a.bias[min(o, a.np - 1)];
    int c = wave;
    for (; c + NW < chunks; c += 2 * NW) {
        load(std::integral_constant<int, 1>{}, c + NW);
        multiply(std::integral_constant<int, 0>{});
        load(std::integral_constant<int, 0>{}, c + 2 * NW);
        multiply(std::integral_constant<int, 1>{});
    }
    if (c < chunks) multiply(std::integral_constant<int, 0>{});                      // not past the end: x is zeros there, but W may have infinities
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) l_sum[wave][16 * i + frow][4 * kq + e] = acc[i][e];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int row = (tid >> 4) + 32 * j;
        if (id[j] == -2) continue;
        float v = bias;
#pragma unroll
        for (int q = 0; q < NW; ++q) v += l_sum[q][row][tid & 15];
        if (id[j] >= 0) {
            float sum_b = 0.f;                                                   // by itself: up to 256 small terms, one by one onto a large v, would lose eight bits of theirs
            for (int r = 0; r < a.rp; r += 16) {
                if (r) load_adapter(j, r);
                float sum = uv[j][0];                                            // of element r + tid % 16; the row's sixteen threads show them to each other
#pragma unroll
                for (int e = 1; e < SPLITS; ++e) sum += uv[j][e];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t two = (uint32_t)bv[j][e >> 2][e & 3];
                    sum_b = fmaf(__shfl(sum, 2 * e, 16), __uint_as_float(two << 16), sum_b);
                    sum_b = fmaf(__shfl(sum, 2 * e + 1, 16), __uint_as_float(two & 0xFFFF0000u), sum_b);
                }
            }
            v += sum_b;
        }
        if (o >= a.co) continue;
        const int m = m0 + row;
        if (a.out_f32) ((float*)a.y)[m * a.ldy + o] = v;
        else ((uint16_t*)a.y)[m * a.ldy + o] = __builtin_bit_cast(uint16_t, (__bf16)v);
    }
}

// ---- the projection, many rows ---------------------------------------------------------------------------------------------------
// KG groups of WM x WN wavefronts share the reduction, a slab of 32 columns of x and W each at a time; a wavefront has MB x NB blocks of 32 rows x 32 outputs.  Slabs go through LDS, a ring
// of stages per group filled by asynchronous copies: those of step t + RING - 1 start, and those of t + 1 are waited for, at the barrier in front of step t, so that the operands of a step's
// first instructions are read before its barrier.
// The adapters are further slabs: for each different one among the tile's rows, the parts of u (rows of others: zeros) and its second half.
// FUSE: slots of at least BM - 1 rows, so that a tile has rows of two slots at most, and ranks up to 32: the first halves of both are 64 further outputs of the tile, wavefronts wn = 0 and 1 have one
// each; they go through LDS to the second halves, and there is no launch in front of this one.
template <int MB, int NB, int WM, int WN, int KG, int RING, bool F32, bool FUSE>
__global__ __launch_bounds__(64 * WM * WN * KG) void adapter_project_kernel(AdapterKernelArgs a, int gm, int gn)
{
    constexpr int NW = WM * WN, NT = 64 * NW * KG, BM = 32 * MB * WM, BN = 32 * NB * WN, STAGE = (BM + BN + (FUSE ? 64 : 0)) * 64;
    constexpr int XU = BM / 16 / NW, WU = BN / 16 / NW, AU = FUSE ? 4 / NW : 0, PU = XU + WU + AU;                    // KiB a wavefront copies per stage: of x, of W, of the first halves
    static_assert(XU * 16 * NW == BM && WU * 16 * NW == BN && BM <= 256 && BM % 64 == 0 && (!FUSE || (WN == 2 && NW == 4 && KG == 1)));
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    int* const l_list = (int*)(lds + KG * RING * STAGE);   // different adapters of the rows, their number
    int* const l_ids = l_list + BM + 4;                    // adapter of every row
    const int tid = threadIdx.x, lane = tid & 63, wave_all = __builtin_amdgcn_readfirstlane(tid >> 6), kg = wave_all / NW, wave = wave_all % NW, hi = lane >> 5, frow = lane & 31;
    const int wm = wave % WM, wn = wave / WM;
    // tiles in groups of four along the rows, in a group the rows first; each XCD an eighth of them, one behind the other: what its tiles read at a time fits its L2
    const int unit = xcd_unit(blockIdx.x, gm * gn);
    if (unit < 0) return;
    const int group = unit / (4 * gn), in = unit - group * 4 * gn, tall = min(4, gm - group * 4), nt = in / tall, mt = group * 4 + in - nt * tall;
    const int m0 = mt * BM, nb0 = nt * WN * NB, n0 = nb0 + wn * NB;      // nb0, n0: the tile's, the wavefront's first block of 32 outputs
    const unsigned lds0 = lds_addr(lds) + (unsigned)(kg * RING * STAGE);
    unsigned char* const ring = lds + kg * RING * STAGE;
    const int slabs = a.kp / 32, blocks = a.np / 32, kx = a.parts * a.rp, per = (kx + 31) / 32, rs = a.rp / 16;      // per: slabs an adapter takes
    int two[2] = {-1, -1};                                 // FUSE: the adapters of the tile's slots; l_ids: which of them
    if constexpr (FUSE) {
        const int slot = m0 / a.per, last = min(m0 + BM, a.rows) - 1;
        two[0] = a.ids[slot];
        two[1] = last / a.per != slot ? a.ids[slot + 1] : -1;
#pragma unroll
        for (int k = 0; k < 2; ++k) two[k] = __builtin_amdgcn_readfirstlane((unsigned)two[k] < (unsigned)a.adapters ? two[k] : -1);
        for (int r = tid; r < BM; r += NT) {
            const int which = (m0 + r) / a.per != slot;
            l_ids[r] = m0 + r >= a.rows ? -2 : (which ? two[1] : two[0]) >= 0 ? which : -1;
        }
    } else
        for (int r = tid; r < BM; r += NT) l_ids[r] = m0 + r < a.rows ? a.row_ids ? a.row_ids[m0 + r] : -1 : -2;
    // LDS of a stage: rows of 64 bytes, position p of row r holds chunk p ^ (r / 4 & 3) (16 rows are in 16 different quads of banks) | operands of W, a KiB per block and step of 16
    const unsigned char* const xt = (const unsigned char*)(a.x + (int64_t)m0 * a.ldx);
    unsigned from[XU];                                     // bytes from there: the host bounds 256 rows by 2 GiB
#pragma unroll
    for (int j = 0; j < XU; ++j) {
        const int row = 16 * (j * NW + wave) + (lane >> 2);
        from[j] = (unsigned)min(row, a.rows - 1 - m0) * (unsigned)(2 * a.ldx) + (unsigned)((lane & 3) ^ (row >> 2 & 3)) * 16u;
    }
    const unsigned char* w[WU];                            // uniform
#pragma unroll
    for (int j = 0; j < WU; ++j) {
        const int u = j * NW + wave;
        w[j] = (const unsigned char*)a.w + ((int64_t)min(nb0 + u / 2, blocks - 1) * slabs * 2 + u % 2) * 1024;
    }
    const unsigned wlane = (unsigned)lane * 16u;
    const unsigned char* halves = nullptr;                 // FUSE: the first half whose operands this wavefront copies (AU is 1), from its step of 16
    if constexpr (FUSE) halves = (const unsigned char*)a.a + ((int64_t)max(wave >= 2 ? two[1] : two[0], 0) * slabs * 2 + wave % 2) * 1024;
    // where step `it` goes in the ring, and the slab that is this group's
    auto stage = [&](int it) { return (unsigned)(it % RING * STAGE); };
    auto slab = [&](int it) { return it * KG + kg; };
    // piece j of a step: XU of x, then WU of W.  Slabs of whole 32 columns only
    auto piece = [&](int it, auto j_tag) {
        constexpr int J = decltype(j_tag)::value;
        const unsigned to = lds0 + stage(it) + (unsigned)(wave * 1024);
        if constexpr (J < XU) dma16(to + (unsigned)(NW * J * 1024), xt + (int64_t)slab(it) * 64, from[J]);
        else dma16(to + (unsigned)(BM * 64 + NW * (J - XU) * 1024), (J < XU + WU ? w[J < XU + WU ? J - XU : 0] : halves) + (int64_t)slab(it) * 2048, wlane);
    };
    // Piece j of a step that is no whole slab of x for certain.  ad >= 0: slab e of that adapter, where rows of others read zeros; else, e >= 0: past the end, zeros; else a slab of x, with zeros
    // behind the last column
    int ids[XU];                                           // the adapters of the rows this lane copies
    auto piece_of = [&](int it, auto j_tag, int ad, int e) {
        constexpr int J = decltype(j_tag)::value;
        const unsigned to = lds0 + stage(it) + (unsigned)(wave * 1024);
        if constexpr (J < XU) {
            const int row = 16 * (J * NW + wave) + (lane >> 2), k = ((lane & 3) ^ (row >> 2 & 3)) * 8;
            const void* at = a.zeros;
            if (e < 0) at = slab(it) * 32 + k < a.ci ? (const void*)(xt + (int64_t)slab(it) * 64 + from[J]) : at;
            else if (ad >= 0) at = ids[J] == ad && e * 32 + k < kx ? (const void*)(a.u + (int64_t)(m0 + row) * kx + e * 32 + k) : at;
            dma16(to + (unsigned)(NW * J * 1024), at);
        } else {
            const int u = (J - XU) * NW + wave;
            const unsigned char* b = (J < XU + WU ? w[J < XU + WU ? J - XU : 0] : halves) + (int64_t)slab(it) * 2048;
            if (ad >= 0) b = (const unsigned char*)a.b + (((int64_t)ad * blocks + min(nb0 + u / 2, blocks - 1)) * rs + (e * 2 + u % 2) % rs) * 1024;
            dma16(to + (unsigned)(BM * 64 + NW * (J - XU) * 1024), e < 0 || ad >= 0 ? (const void*)(b + wlane) : a.zeros);       // zeros past the end: W may have infinities
        }
    };
    constexpr int EARLY = KG <= 2 ? 2 / KG : 0;            // steps that are slabs of x for certain: kp is a multiple of 64
    static_for<EARLY>([&](auto k) { static_for<PU>([&](auto j) { piece_of(decltype(k)::value, j, -1, -1); }); });
    __syncthreads();
    if (!FUSE && wave_all == 0) {
        int mine[BM / 64], n = 0;
#pragma unroll
        for (int i = 0; i < BM / 64; ++i) mine[i] = l_ids[64 * i + lane] < ODD ? l_ids[64 * i + lane] : -1;
        for (;;) {
            int ad = -1;
#pragma unroll
            for (int i = 0; i < BM / 64; ++i) {
                const unsigned long long b = __ballot(mine[i] >= 0);
                if (ad < 0 && b) ad = __builtin_amdgcn_readlane(mine[i], __builtin_ctzll(b));
            }
            if (ad < 0) break;
#pragma unroll
            for (int i = 0; i < BM / 64; ++i) mine[i] = mine[i] == ad ? -1 : mine[i];
            if (lane == 0) l_list[n] = ad;
            ++n;
        }
        if (lane == 0) l_list[BM] = n;
    }
    lds_barrier();
    const int total = FUSE ? slabs : slabs + __builtin_amdgcn_readfirstlane(l_list[BM]) * per, iters = (total + KG - 1) / KG;
#pragma unroll
    for (int j = 0; j < XU; ++j) ids[j] = l_ids[16 * (j * NW + wave) + (lane >> 2)];
    // f(adapter, its slab) of step `it`, as piece_of takes them
    auto what = [&](int it, auto&& f) {
        const int s = slab(it), e = s - slabs;
        if (e < 0) f(-1, -1);
        else if (!FUSE && s < total) f(__builtin_amdgcn_readfirstlane(l_list[e / per]), e % per);
        else f(-1, 0);
    };
    for (int k = EARLY; k < RING - 1; ++k) what(k, [&](int ad, int e) { static_for<PU>([&](auto j) { piece_of(k, j, ad, e); }); });
    unsigned at[2];                                        // x, step of 16
#pragma unroll
    for (int k = 0; k < 2; ++k) at[k] = (unsigned)((wm * MB * 32 + frow) * 64 + (((2 * k + hi) ^ (frow >> 2 & 3)) << 4));
    const unsigned wat = (unsigned)(BM * 64 + wn * NB * 2048) + wlane;
    // operands are read two steps of 16 columns before they are used, into four sets in turn: a read takes as long as four to eight matrix instructions when all wavefronts read
    v4i xv[4][MB], wv[4][NB], fv[FUSE ? 4 : 1];
    auto read = [&](auto set, int it, auto step, auto n_tag) {           // operand n_tag of a step, in the order they are used: w 0, x 0, the rest of w, the rest of x
        constexpr int S = decltype(set)::value, K = decltype(step)::value, N = decltype(n_tag)::value, X = N == 1 ? 0 : N > NB ? N - NB : -1, W = N == 0 ? 0 : N - 1;
        const unsigned char* const base = ring + stage(it);
        if constexpr (N == MB + NB) fv[S] = *(const v4i*)(base + (BM + BN) * 64 + wlane + (wn * 2 + K) * 1024);
        else if constexpr (X >= 0) xv[S][X] = *(const v4i*)(base + at[K] + X * 2048);
        else wv[S][W] = *(const v4i*)(base + wat + (W * 2 + K) * 1024);
    };
    v16f acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[i][n] = v16f{};
    v16f half[FUSE ? MB : 1];                              // of the first half of adapter two[wn]
#pragma unroll
    for (int i = 0; i < (FUSE ? MB : 1); ++i) half[i] = v16f{};
    // the MB x NB instructions of a step (FUSE: and MB); behind instruction k: f(k)
    constexpr int INSTRUCTIONS = MB * NB + (FUSE ? MB : 0);
    auto multiply = [&](auto set, auto&& f) {
        constexpr int S = decltype(set)::value;
        static_for<INSTRUCTIONS>([&](auto k_tag) {
            constexpr int K = decltype(k_tag)::value, I = K < MB * NB ? K / NB : K - MB * NB, N = K % NB;
            if constexpr (K >= MB * NB) half[I] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, fv[S]), __builtin_bit_cast(v8bf, xv[S][I]), half[I], 0, 0, 0);
            else acc[I][N] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, wv[S][N]), __builtin_bit_cast(v8bf, xv[S][I]), acc[I][N], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            f(k_tag);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // things 0 .. count - 1, as evenly behind the first SLOTS instructions as whole numbers allow
    auto spread = [&](auto k_tag, auto count, auto slots, auto&& g) {
        constexpr int K = decltype(k_tag)::value, COUNT = decltype(count)::value, SLOTS = decltype(slots)::value, LO = K < SLOTS ? K * COUNT / SLOTS : COUNT, HI = K < SLOTS ? (K + 1) * COUNT / SLOTS : COUNT;
        static_for<HI - LO>([&](auto d) { g(std::integral_constant<int, LO + decltype(d)::value>{}); });
    };
    using operands = std::integral_constant<int, MB + NB + FUSE>;
    using pieces = std::integral_constant<int, PU>;
    using every = std::integral_constant<int, INSTRUCTIONS>;
    using front = std::integral_constant<int, (INSTRUCTIONS + 1) / 2>;
    // Step `it` of parity P; the copies go out between matrix instructions: all of a workgroup's at once would hold up the instructions behind them
    auto iteration = [&](auto parity, int it, auto fast) {
        constexpr int P = decltype(parity)::value;
        constexpr bool FAST = decltype(fast)::value;
        wait_copies_then_barrier<(RING - 3) * PU>();      // step it + 1 is there, step it - 1 has been read by all
        int ad = -1, e = -1;
        if constexpr (!FAST) what(it + RING - 1, [&](int ad_, int e_) { ad = ad_; e = e_; });
        static_for<2>([&](auto step) {
            constexpr int K = decltype(step)::value;
            multiply(std::integral_constant<int, 2 * P + K>{}, [&](auto k) {
                spread(k, operands{}, front{}, [&](auto n) { read(std::integral_constant<int, 2 * (1 - P) + K>{}, it + 1, step, n); });
                if constexpr (K == 0)
                    spread(k, pieces{}, every{}, [&](auto j) {
                        if constexpr (FAST) piece(it + RING - 1, j);
                        else piece_of(it + RING - 1, j, ad, e);
                    });
            });
        });
    };
    wait_copies_then_barrier<(RING - 2) * PU>();
    static_for<2>([&](auto k) { static_for<MB + NB + FUSE>([&](auto n) { read(k, 0, k, n); }); });
    int it = 0;
    const int full = min(a.ci / 32 / KG, iters) - (RING - 1);   // steps that copy whole slabs of x
    for (; it + 2 <= full; it += 2) static_for<2>([&](auto p) { iteration(p, it + decltype(p)::value, std::true_type{}); });
    for (; it < iters; it += 2)                            // where the number is odd one step more, of zeros
        static_for<2>([&](auto p) { iteration(p, it + decltype(p)::value, std::false_type{}); });

    // ---- results: a lane has row frow of a block, outputs 8 q + 4 hi + 0..3; through LDS, a wavefront's 32 rows of 32 NB outputs at a time, to whole pieces of 16 bytes ----
    constexpr int ES = F32 ? 4 : 2, VEC = 16 / ES, PIECES = 32 * NB / VEC, PITCH = 32 * NB * ES + 16;
    // the results' part of LDS is behind the groups' sums, or the first halves
    constexpr int PARTS = F32 ? 3 : 2, SUMS = FUSE ? 2 * WM * MB * PARTS * 2048 : KG > 1 ? (KG - 1) * NW * MB * NB * 4096 : 0;
    static_assert(SUMS + NW * 32 * PITCH <= KG * RING * STAGE);
    unsigned char* const mine = lds + SUMS + wave * 32 * PITCH;
    const int first = n0 * 32;
    const bool whole = ((uintptr_t)a.y & 15) == 0 && a.ldy % VEC == 0;
    v4f bias[NB][4];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) bias[n][q] = first < a.np && first + n * 32 < a.np ? *(const v4f*)(a.bias + first + n * 32 + 8 * q + 4 * hi) : v4f{0.f, 0.f, 0.f, 0.f};
    wait_all_then_barrier<0>();                            // every wavefront is done with the ring, its copies are too
    if constexpr (KG > 1) {                                // the groups' sums, through LDS, to the first one
        static_assert((KG - 1) * NW * MB * NB * 4096 <= KG * RING * STAGE);
        v4f* const l_part = (v4f*)lds + (size_t)wave * MB * NB * 256 + lane;                  // [group][wavefront][block][quad][lane]
        if (kg > 0)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        v4f v;
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = acc[i][n][4 * q + e];
                        l_part[((kg - 1) * NW * MB * NB + i * NB + n) * 256 + q * 64] = v;
                    }
        lds_barrier();
        if (kg > 0) return;
#pragma unroll
        for (int g = 0; g < KG - 1; ++g)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const v4f v = l_part[(g * NW * MB * NB + i * NB + n) * 256 + q * 64];
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][n][4 * q + e] += v[e];
                    }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    if constexpr (FUSE) {
        // first halves as operands in LDS: [adapter][wm][block][part][step of 16][lane][16]; a lane has elements 8 q + 4 hi + 0..3 of its row
        auto cell = [&](int which, int i, int p, int step) { return lds + ((((which * WM + wm) * MB + i) * PARTS + p) * 2 + step) * 1024; };
        const int ad = wn ? two[1] : two[0], rank = ad >= 0 ? a.info[ad] >> 1 : 0;
        const float scale = ad >= 0 ? a.scale[ad] : 0.f;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = 8 * q + 4 * hi + e < rank ? half[i][4 * q + e] * scale : 0.f;
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    uint16_t h[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const __bf16 b = (__bf16)v[e];
                        h[e] = __builtin_bit_cast(uint16_t, b);
                        v[e] = __builtin_isfinite((float)b) ? v[e] - (float)b : 0.f;
                    }
                    *(uint2*)(cell(wn, i, p, q >> 1) + (frow + 32 * (q & 1)) * 16 + 8 * hi) = uint2{h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16};
                }
            }
        lds_barrier();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (two[k] < 0) continue;
            const bool odd = a.info[two[k]] & 1;           // infinities: element by element, of the parts' sums
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                if (odd) {
#pragma unroll
                    for (int i = 0; i < MB; ++i)
                        if (l_ids[(wm * MB + i) * 32 + frow] == k)
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const int o = min((n0 + n) * 32 + 8 * (e >> 2) + 4 * hi + (e & 3), a.np - 1);
                                const uint16_t* const b = a.b + ((int64_t)two[k] * blocks + (o >> 5)) * rs * 512 + (o & 31) * 8;
#pragma unroll 1
                                for (int r = 0; r < a.rp; ++r) {
                                    float v = 0.f;
                                    for (int p = PARTS - 1; p >= 0; --p) v += __uint_as_float((uint32_t)*(const uint16_t*)(cell(k, i, p, r >> 4) + (frow + 32 * (r >> 3 & 1)) * 16 + (r & 7) * 2) << 16);
                                    acc[i][n][e] = fmaf(v, __uint_as_float((uint32_t)b[(r >> 4) * 512 + (r >> 3 & 1) * 256 + (r & 7)] << 16), acc[i][n][e]);
                                }
                            }
                    continue;
                }
                v4i b[2];
#pragma unroll
                for (int step = 0; step < 2; ++step) b[step] = *(const v4i*)((const unsigned char*)a.b + (((int64_t)two[k] * blocks + min(n0 + n, blocks - 1)) * rs + min(step, rs - 1)) * 1024 + wlane);
#pragma unroll
                for (int i = 0; i < MB; ++i) {
                    v16f t{};
#pragma unroll
                    for (int step = 0; step < 2; ++step)
                        if (step < rs)
#pragma unroll
                            for (int p = 0; p < PARTS; ++p)
                                t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, b[step]), __builtin_bit_cast(v8bf, *(const v4i*)(cell(k, i, p, step) + wlane)), t, 0, 0, 0);
                    const bool own = l_ids[(wm * MB + i) * 32 + frow] == k;                  // rows of others keep their sums, whatever the second half holds
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][n][e] += own ? t[e] : 0.f;
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int r0 = (wm * MB + i) * 32;
        if (const int id = l_ids[r0 + frow]; id >= ODD)
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int o = min(first + n * 32 + 8 * (e >> 2) + 4 * hi + (e & 3), a.np - 1);
                    const uint16_t* const b = a.b + ((int64_t)(id & ~ODD) * blocks + (o >> 5)) * rs * 512 + (o & 31) * 8;
                    const uint16_t* const u = a.u + (int64_t)(m0 + r0 + frow) * kx;
#pragma unroll 1
                    for (int r = 0; r < a.rp; ++r) {
                        float v = 0.f;
                        for (int q = a.parts - 1; q >= 0; --q) v += __uint_as_float((uint32_t)u[q * a.rp + r] << 16);
                        acc[i][n][e] = fmaf(v, __uint_as_float((uint32_t)b[(r >> 4) * 512 + (r >> 3 & 1) * 256 + (r & 7)] << 16), acc[i][n][e]);
                    }
                }
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                v4f v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][n][4 * q + e] + bias[n][q][e];
                unsigned char* const cell = mine + frow * PITCH + (n * 32 + 8 * q + 4 * hi) * ES;
                if constexpr (F32) *(v4f*)cell = v;
                else *(uint2*)cell = uint2{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])};
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int c = 0; c < 32 * PIECES / 64; ++c) {
            const int q = 64 * c + lane, row = q / PIECES, o = first + q % PIECES * VEC;
            const v4i v = *(const v4i*)(mine + row * PITCH + q % PIECES * 16);
            if (l_ids[r0 + row] == -2 || o >= a.co) continue;
            unsigned char* const y = (unsigned char*)a.y + ((int64_t)(m0 + r0 + row) * a.ldy + o) * ES;
            if (whole && o + VEC <= a.co) *(v4i*)y = v;
            else
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (o + e < a.co) {
                        if constexpr (F32) ((int*)y)[e] = v[e];
                        else ((uint16_t*)y)[e] = (uint16_t)((unsigned)v[e >> 1] >> (16 * (e & 1)));
                    }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
int64_t u_bytes(int64_t rows) { return rows <= 1024 ? 4 * SPLITS : 6; }      // of an element of u
// Few rows leave most CUs idle in the first half, where what a workgroup reads is a chain: up to four share the columns.  One / two / four, both launches, us: 4096 -> 4096 12 rows 15.7 / 13.5 / 12.5;
// 2048 -> 1000 64 rows 11.5 / 10.4 / 10.0, 128 rows 13.5 / 12.5 / 13.4, 256 rows 18.5 / 18.9 / 20.5; 512 -> 1000 no difference
int splits_of(const AdapterKernelArgs& k) { return k.parts || k.rows > 1024 ? 1 : std::clamp(std::min(k.kp / 512, 256 / k.rows), 1, (int)SPLITS); }

struct AdapterSizes {       // in bytes; everything a multiple of 256
    int64_t kp, np, rp, ra, w, bias, a, b, scale;          // rp, ra: the rank as a reduction's length, as rows
    explicit AdapterSizes(const AdapterDims& d)
    {
        kp = up(d.ci, 64); np = up(d.co, 32); rp = up(std::max(d.rank, 1), 16); ra = up(rp, 32);
        w = 2 * np * kp; bias = up(4 * np, 256);
        a = 2 * ra * kp * d.adapters; b = 2 * np * rp * d.adapters; scale = up(8ll * d.adapters, 256);
    }
};

hipError_t launch_shrink(const AdapterKernelArgs& k, hipStream_t s)
{
    // few rows: 16 at a time, and a workgroup for every adapter that may be among them; many rows of one slot each: two may be, of packed ones any number
    const int rows = k.rows <= 1024 ? 16 : 32, blocks = (k.rows + rows - 1) / rows, most = k.offsets ? 4 : k.per >= rows ? 2 : rows;
    int ords = 1;
    while (ords < (rows == 16 ? 16 : most) && 2 * ords * blocks <= 2048) ords *= 2;
    auto go = [&](auto kernel, int rt) {
        EE_LAUNCH(kernel, dim3((unsigned)(blocks * ords), (unsigned)((k.rp + rt * rows - 1) / (rt * rows)), (unsigned)k.splits), dim3(512), 0, s, k, blocks, ords);
        return hipGetLastError();
    };
    if (rows == 16) return k.rp <= 16 ? go(adapter_shrink_kernel<16, 1>, 1) : k.rp <= 32 ? go(adapter_shrink_kernel<16, 2>, 2) : go(adapter_shrink_kernel<16, 4>, 4);
    return k.rp <= 32 ? go(adapter_shrink_kernel<32, 1>, 1) : go(adapter_shrink_kernel<32, 2>, 2);
}

// Whether the kernel for few rows is the one: up to 32 rows; up to 64 where 64 rows to a workgroup are no more than 256 of these; else by what both take, in us, with K the reduction in thousands, G
// the workgroups in 256s, R the rank in 16s behind the first, S the slabs that the adapters among a tile's 64 rows add.  This kernel 4.5 + 0.7 K + 0.5 R + G (2.4 + 4.3 K + R), tiles (up to 256 of
// 64 x 64) 8 + 2.8 K + 0.3 S.  Measured, both launches, eight adapters of rank 16, this kernel / tiles: 512 -> 1000 256 rows 9.8 / 12.2, 512 rows 14.5 / 12.3 (24 adapters 16.4 / 19.0); 1024 -> 256
// 512 rows 9.1 / 13.4, 1024 rows 13.3 / 14.8, 2048 rows 28 / 22; 2048 -> 1000 128 rows 11.8 / 16.1, 256 rows 17.8 / 16.3 (24 adapters 18.7 / 22.1); 4096 -> 1024 128 rows 16.1 / 21.9,
// 256 rows 27.9 / 25.6; 176 -> 3176 96 rows 10.1 / 11.6, 256 rows 17.3 / 11.8 (rank 64 28.5 / 18.5); 4096 -> 4096 32 rows 16.2 / 24.4, 64 rows 24.4 / 26.9, 128 rows 43 / 27
bool few_rows(const AdapterKernelArgs& k)
{
    const int64_t groups = (int64_t)((k.rows + 63) / 64) * ((k.co + 15) / 16);
    if (k.rows <= 32 || (k.rows <= 64 && groups <= 256)) return true;
    const int different = std::min(std::min(k.adapters, k.slots), 64 / std::max(1, k.rows / k.slots) + 1);
    const double thousands = k.kp / 1024.0, more = k.rp / 16 - 1, slabs = different * (((k.out_f32 ? 3 : 2) * k.rp + 31) / 32);
    return groups / 256.0 * (2.4 + 4.3 * thousands + more) < 3.5 + 2.1 * thousands + 0.3 * slabs - 0.5 * more;
}

hipError_t launch_few_rows(const AdapterKernelArgs& k, hipStream_t s)
{
    const int gn = (k.co + 15) / 16;
    auto go = [&](auto kernel, int mt) {
        EE_LAUNCH(kernel, dim3((unsigned)((k.rows + 16 * mt - 1) / (16 * mt) * gn)), dim3(512), 0, s, k, gn);
        return hipGetLastError();
    };
    // As few rows to a workgroup as 256 workgroups allow, as long as there are such rows.  16 / 32 / 64 rows, us: 2048 -> 1000 64 rows 10.0 / 11.1 / 15.4, 128 rows 14.7 / 12.5 / 16.1;
    // 4096 -> 4096 32 rows 17.6 / 16.8 / 18.7
    auto fits = [&](int r) { return k.rows <= r || (int64_t)((k.rows + r - 1) / r) * gn <= 256; };
    return fits(16) ? go(adapter_rows_project_kernel<1>, 1) : fits(32) ? go(adapter_rows_project_kernel<2>, 2) : go(adapter_rows_project_kernel<4>, 4);
}

template <int MB, int NB, int WM, int WN, int KG, int RING, bool F32, bool FUSE>
hipError_t launch_tiles(const AdapterKernelArgs& k, hipStream_t s)
{
    constexpr int BM = 32 * MB * WM, BN = 32 * NB * WN;
    constexpr unsigned LDS = KG * RING * (BM + BN + (FUSE ? 64 : 0)) * 64 + 8 * BM + 16;
    static const hipError_t granted = hipFuncSetAttribute(reinterpret_cast<const void*>(&adapter_project_kernel<MB, NB, WM, WN, KG, RING, F32, FUSE>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (granted != hipSuccess) return granted;
    const int gm = (k.rows + BM - 1) / BM, gn = (k.co + BN - 1) / BN;
    EE_LAUNCH((adapter_project_kernel<MB, NB, WM, WN, KG, RING, F32, FUSE>), dim3(xcd_grid((long long)gm * gn)), dim3(64 * WM * WN * KG), LDS, s, k, gm, gn);
    return hipGetLastError();
}

template <int MB, int NB, int WM, int WN, int KG, int RING, bool FUSE = false>
hipError_t launch_form(const AdapterKernelArgs& k, hipStream_t s) { return k.out_f32 ? launch_tiles<MB, NB, WM, WN, KG, RING, true, FUSE>(k, s) : launch_tiles<MB, NB, WM, WN, KG, RING, false, FUSE>(k, s); }

// Whether tiles compute the first halves themselves: slots as long as a tile, and outputs that few tiles share, or x would be multiplied with the first halves too often: one column of tiles, or one round
// of tiles, two columns of them or a short reduction.  Both launches / this, us, rank 32: 12544 rows 1024 -> 128 24.3 / 20.1, -> 256 27.2 / 22.1, -> 512 34 / 38; 38400 rows 4096 -> 128 172 / 122;
// 3136 rows 64 -> 1024 14.7 / 11.4, 512 -> 1024 16.5 / 15.2, 2048 -> 1024 29.9 / 29.9, 1024 -> 128 13.7 / 17.9.  Beyond one round two columns go either way with the reduction's length and are left to two
// launches: 38400 rows 4096 -> 256 188 / 166, 1024 -> 256 50 / 54
bool fused(const AdapterKernelArgs& k)
{
    if (k.offsets || k.adapters == 0 || k.per < 127 || k.rp > 32) return false;
    const int64_t gn = (k.co + 127) / 128, tiles = (k.rows + 127) / 128 * gn;
    return gn == 1 ? tiles >= 96 : tiles >= 128 && tiles <= 256 && (gn == 2 || k.kp <= 512);
}

hipError_t launch_many_rows(const AdapterKernelArgs& k, hipStream_t s)
{
    auto tiles = [&](int bm, int bn) { return (int64_t)((k.rows + bm - 1) / bm) * ((k.co + bn - 1) / bn); };
    // The largest tile that gives every CU one: while there are fewer tiles than CUs the reduction is a chain, and smaller tiles with two groups of wavefronts make it shorter.  4096 -> 4096, us
    // with one adapter: 256 rows 64 x 64 tiles 26, 64 x 128 32, 128 x 128 37; 512 rows 42, 34, 39; 1024 rows 75, 60, 45
    if (tiles(64, 64) <= 256) return launch_form<1, 1, 2, 2, 2, 8>(k, s);
    if (tiles(64, 128) <= 256) return launch_form<1, 2, 2, 2, 2, 6>(k, s);
    if (tiles(128, 128) <= 256) return launch_form<2, 2, 2, 2, 2, 4>(k, s);
    // More: in units of a round of 256 tiles of 256 x 256, a round of 256 tiles of 128 x 128 takes 0.37.  4096 -> 4096: 2048 rows 88 and 81 us, 3000 rows 102 and 116, 8192 rows 218 and 266
    return (double)((tiles(256, 256) + 255) / 256) < 0.37 * (double)((tiles(128, 128) + 255) / 256) ? launch_form<4, 2, 2, 4, 1, 4>(k, s) : launch_form<2, 2, 2, 2, 1, 4>(k, s);
}

hipError_t pack(const void* src, int64_t ld, int rows, int cols, void* dst, int64_t blocks, int64_t steps, hipStream_t s, int* info = nullptr, int rank = 0, float* scale = nullptr, float factor = 0.f)
{
    EE_LAUNCH(adapter_pack_kernel, dim3(blocks_of(blocks * steps * 64)), dim3(256), 0, s, (const uint16_t*)src, ld, rows, cols, (uint16_t*)dst, (int)blocks, (int)steps, info, rank, scale, factor);
    return hipGetLastError();
}

}  // namespace

// packed weights: operands | bias | 256 zero bytes; adapters: first halves | second halves | factors | ranks
int64_t adapter_weight_bytes(const AdapterDims& d) { const AdapterSizes z(d); return z.w + z.bias + 256; }
int64_t adapter_pool_bytes(const AdapterDims& d) { const AdapterSizes z(d); return std::max<int64_t>(256, z.a + z.b + z.scale); }
// u | adapters of the rows | a padded copy of x where its rows are no whole 16-byte pieces
int64_t adapter_workspace(const AdapterDims& d, int64_t rows) { const AdapterSizes z(d); return up(u_bytes(rows) * rows * z.rp, 256) + up(4 * rows, 256) + (rows * z.kp * 2); }

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
    float* const factor = (float*)(p + z.a + z.b) + i;
    int* const info = (int*)(factor + d.adapters);
    const hipError_t e = pack(a, lda, rank, d.ci, p + z.a / d.adapters * i, z.ra / 32, z.kp / 16, s, info, rank, factor, scale);
    return e == hipSuccess ? pack(b, ldb, d.co, rank, p + z.a + z.b / d.adapters * i, z.np / 32, z.rp / 16, s, info, rank) : e;
}

hipError_t launch_adapter_project(const AdapterDims& d, const AdapterCall& c, hipStream_t s)
{
    const AdapterSizes z(d);
    AdapterKernelArgs k{};
    k.x = (const uint16_t*)c.x; k.ldx = c.ldx; k.y = c.y; k.ldy = c.ldy; k.out_f32 = c.out_f32;
    k.w = (const uint16_t*)c.packed; k.bias = (const float*)((const char*)c.packed + z.w); k.zeros = (const uint16_t*)((const char*)c.packed + z.w + z.bias);
    k.a = (const uint16_t*)c.pool; k.b = (const uint16_t*)((const char*)c.pool + z.a); k.scale = (const float*)((const char*)c.pool + z.a + z.b); k.info = (const int*)k.scale + d.adapters;
    k.ids = c.ids; k.offsets = c.offsets; k.rows = c.rows; k.slots = c.slots; k.per = c.per;
    k.ci = d.ci; k.co = d.co; k.kp = (int)z.kp; k.np = (int)z.np; k.rp = (int)z.rp; k.ra = (int)z.ra; k.adapters = d.adapters; k.parts = few_rows(k) ? 0 : c.out_f32 ? 3 : 2;
    k.splits = splits_of(k);
    char* ws = (char*)c.workspace;
    k.u = (uint16_t*)ws; ws += up(u_bytes(c.rows) * c.rows * z.rp, 256);
    k.row_ids = (int*)ws; ws += up(4ll * c.rows, 256);
    if (((uintptr_t)c.x & 15) || c.ldx % 8 || d.ci % 8 || c.ldx > 1 << 21) {
        EE_LAUNCH(adapter_rows_kernel, dim3(blocks_of((int64_t)c.rows * z.kp)), dim3(256), 0, s, k.x, k.ldx, c.rows, d.ci, (uint16_t*)ws, k.kp);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        k.x = (const uint16_t*)ws; k.ldx = k.kp; k.ci = k.kp;
    }
    if (k.parts && fused(k)) return launch_form<2, 2, 2, 2, 1, 6, true>(k, s);
    if (d.adapters == 0 && !c.offsets) k.row_ids = nullptr;           // every row has none
    else if (const hipError_t e = launch_shrink(k, s); e != hipSuccess) return e;
    return few_rows(k) ? launch_few_rows(k, s) : launch_many_rows(k, s);
}

}  // namespace ee
