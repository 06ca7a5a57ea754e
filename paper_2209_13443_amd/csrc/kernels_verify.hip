// Verification of drafted tokens against a target's probabilities, from given random numbers, for gfx950.
//
// Per sequence: draft i is accepted while u_i q_i(x_i) < p_i(x_i) (the product of two floats is exact in 64 bits); n: the number accepted.  One more token is
// drawn: weights w_j = max(p_n(j) - q_n(j), 0) behind a refusal (p_n where those are all zero), p_n where everything was accepted; the first j with
// w_0 + .. + w_j > u_K (w_0 + .. + w_{V-1}).  Entries that are not finite and positive weigh nothing.  Sums are held in 64 bits and added in one fixed order.
//
// Bound by reading two rows of V entries per sequence, of which only the decision above says which: every workgroup makes it again (K gathers).  Rows are cut into chunks so that
// a few sequences fill the chip: the first launch sums the chunks, the second finds the chunk in which the number lies and looks inside.
#include <algorithm>

#include "ee_internal.hpp"
#include "igemm_device.hpp"

namespace ee {
namespace {

struct VerifyArgs {
    VerifyCall c;
    int chunk, chunks;               // entries of a chunk
    double2* sums;                   // [b][chunks]: of the refusal's weights, of p
};

__device__ __forceinline__ double weight_of(double w) { return w > 0.0 && w < __builtin_inf() ? w : 0.0; }
template <bool F32> __device__ __forceinline__ float prob(const void* base, int64_t at)
{
    if constexpr (F32) return ((const float*)base)[at];
    else return __uint_as_float((uint32_t)((const uint16_t*)base)[at] << 16);
}

// drafts accepted (by all lanes of the first wavefront, 64 drafts at a time), -1: an empty slot
template <bool F32>
__device__ __forceinline__ int accepted(const VerifyCall& c, int b, int drafts, int lane)
{
    for (int i0 = 0; i0 < drafts; i0 += 64) {
        const int i = i0 + lane;
        bool ok = i < drafts;
        if (ok) {
            const int x = c.draft[b * c.draft_row + i];
            ok = x >= 0 && x < c.v;
            if (ok) {
                const double u = c.u[b * c.u_row + i], p = prob<F32>(c.p, b * c.p_seq + i * c.p_row + x);
                const double q = c.q ? (double)prob<F32>(c.q, b * c.q_seq + i * c.q_row + x) : 1.0;
                ok = u * q < p;
            }
        }
        const unsigned long long good = __ballot(ok);
        if (~good) return min(drafts, i0 + (int)__builtin_ctzll(~good));
    }
    return drafts;
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) v += __shfl_xor(v, off);
    return v;
}

// the rows the extra token is drawn from
struct Rows { int64_t p, q; bool minus; int skip; };
__device__ __forceinline__ Rows rows_of(const VerifyCall& c, int b, int n, int drafts)
{
    Rows r{b * c.p_seq + n * c.p_row, 0, false, -1};
    if (n < drafts) {
        if (c.q) { r.minus = true; r.q = b * c.q_seq + n * c.q_row; }
        else r.skip = c.draft[b * c.draft_row + n];
    }
    return r;
}

template <bool F32>
__device__ __forceinline__ double2 weights_at(const VerifyCall& c, const Rows& r, int j)
{
    const double p = prob<F32>(c.p, r.p + j);
    const double w = r.minus ? p - (double)prob<F32>(c.q, r.q + j) : j == r.skip ? 0.0 : p;
    return double2{weight_of(w), weight_of(p)};
}

template <bool F32>
__global__ __launch_bounds__(256) void verify_sum_kernel(VerifyArgs a)
{
    __shared__ int l_n;
    __shared__ double2 l_part[4];
    const VerifyCall& c = a.c;
    const int b = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks, tid = threadIdx.x;
    const int drafts = c.lengths ? min(c.lengths[b], c.k) : c.k;
    if (tid < 64) {
        const int n = accepted<F32>(c, b, drafts, tid);
        if (tid == 0) l_n = n;
    }
    __syncthreads();
    if (drafts < 0) return;
    const Rows r = rows_of(c, b, l_n, drafts);
    double2 s{0.0, 0.0};
    const int j1 = min(c.v, (chunk + 1) * a.chunk);
    for (int j = chunk * a.chunk + tid; j < j1; j += 256) {
        const double2 w = weights_at<F32>(c, r, j);
        s.x += w.x;
        s.y += w.y;
    }
    s.x = wave_sum(s.x);
    s.y = wave_sum(s.y);
    if ((tid & 63) == 0) l_part[tid >> 6] = s;
    __syncthreads();
    if (tid == 0) a.sums[(int64_t)b * a.chunks + chunk] = double2{l_part[0].x + l_part[1].x + l_part[2].x + l_part[3].x, l_part[0].y + l_part[1].y + l_part[2].y + l_part[3].y};
}

template <bool F32>
__global__ __launch_bounds__(256) void verify_pick_kernel(VerifyArgs a)
{
    __shared__ int l_n, l_chunk, l_first;
    __shared__ double l_before, l_target;
    __shared__ bool l_use_p;
    __shared__ double l_scan[256];
    __shared__ int l_last;
    const VerifyCall& c = a.c;
    const int b = blockIdx.x, tid = threadIdx.x;
    const int drafts = c.lengths ? min(c.lengths[b], c.k) : c.k;
    if (tid < 64) {
        const int n = accepted<F32>(c, b, drafts, tid);
        if (tid == 0) {
            l_n = n;
            l_first = c.v;
            l_last = -1;
        }
    }
    __syncthreads();
    const int n = l_n;
    if (tid == 0 && drafts >= 0) {
        const double2* const s = a.sums + (int64_t)b * a.chunks;
        double2 all{0.0, 0.0};
        for (int k = 0; k < a.chunks; ++k) { all.x += s[k].x; all.y += s[k].y; }
        const bool use_p = !(all.x > 0.0);
        const double total = use_p ? all.y : all.x, target = (double)c.u[b * c.u_row + c.k] * total;
        double before = 0.0, at = 0.0;
        int chunk = -1;
        for (int k = 0; k < a.chunks; ++k) {
            const double v = use_p ? s[k].y : s[k].x;
            if (v > 0.0) { chunk = k; before = at; }
            at += v;
            if (at > target) break;
        }
        l_chunk = chunk;                                 // -1: nothing can be drawn
        l_before = before; l_target = target; l_use_p = use_p;
    }
    __syncthreads();
    int token = -1;
    if (drafts >= 0 && l_chunk >= 0) {
        const Rows r = rows_of(c, b, n, drafts);
        const int j0 = l_chunk * a.chunk, j1 = min(c.v, j0 + a.chunk), per = (a.chunk + 255) / 256;
        const int s0 = min(j1, j0 + tid * per), s1 = min(j1, s0 + per);
        double sum = 0.0;
        int last = -1;
        for (int j = s0; j < s1; ++j) {
            const double2 w = weights_at<F32>(c, r, j);
            const double v = l_use_p ? w.y : w.x;
            if (v > 0.0) last = j;
            sum += v;
        }
        l_scan[tid] = sum;
        if (last >= 0) atomicMax(&l_last, last);
        __syncthreads();
        for (int off = 1; off < 256; off <<= 1) {
            const double v = tid >= off ? l_scan[tid - off] : 0.0;
            __syncthreads();
            l_scan[tid] += v;
            __syncthreads();
        }
        double cum = l_before + (tid ? l_scan[tid - 1] : 0.0);
        if (l_before + l_scan[tid] > l_target)
            for (int j = s0; j < s1; ++j) {
                const double2 w = weights_at<F32>(c, r, j);
                const double v = l_use_p ? w.y : w.x;
                cum += v;
                if (v > 0.0 && cum > l_target) { atomicMin(&l_first, j); break; }
            }
        __syncthreads();
        token = l_first < c.v ? l_first : l_last;        // the number lies behind every sum (1, or by rounding): the last entry that can be drawn
    }
    if (tid == 0) c.accepted[b] = max(n, 0);
    for (int i = tid; i <= c.k; i += 256)
        c.tokens[b * (int64_t)(c.k + 1) + i] = drafts < 0 ? -1 : i < n ? c.draft[b * c.draft_row + i] : i == n ? token : -1;
}

void plan_verify(const VerifyCall& c, VerifyArgs& a)
{
    a.c = c;
    a.chunk = 4096;
    while ((c.v + (int64_t)a.chunk - 1) / a.chunk > 256) a.chunk *= 2;
    a.chunks = (int)((c.v + (int64_t)a.chunk - 1) / a.chunk);
}

}  // namespace

size_t verify_workspace(const VerifyCall& c)
{
    VerifyArgs a;
    plan_verify(c, a);
    return (size_t)c.b * a.chunks * sizeof(double2);
}

hipError_t launch_verify(const VerifyCall& c, void* workspace, hipStream_t s)
{
    VerifyArgs a;
    plan_verify(c, a);
    a.sums = (double2*)workspace;
    const dim3 grid((unsigned)((int64_t)c.b * a.chunks));
    if (c.f32) EE_LAUNCH(verify_sum_kernel<true>, grid, dim3(256), 0, s, a);
    else EE_LAUNCH(verify_sum_kernel<false>, grid, dim3(256), 0, s, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (c.f32) EE_LAUNCH(verify_pick_kernel<true>, dim3((unsigned)c.b), dim3(256), 0, s, a);
    else EE_LAUNCH(verify_pick_kernel<false>, dim3((unsigned)c.b), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace ee
