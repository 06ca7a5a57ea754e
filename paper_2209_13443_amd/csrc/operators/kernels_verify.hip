// Verification of drafted tokens against a target's probabilities, from given random numbers, for gfx950.
//
// Per sequence: draft i is accepted while u_i q_i(x_i) < p_i(x_i) (the product of two floats is exact in 64 bits); n: the number accepted.  One more token is
// drawn: weights w_j = max(p_n(j) - q_n(j), 0) behind a refusal (p_n where those are all zero), p_n where everything was accepted; the first j with
// w_0 + .. + w_j > u_K (w_0 + .. + w_{V-1}).  Entries that are not finite and positive weigh nothing.  Sums are held in 64 bits and added in one fixed order.
//
// Bound by reading two rows of V entries per sequence, of which only the decision above says which (K gathers, which every workgroup of a sequence makes).  Short rows are held by a workgroup
// of 256 threads; one of 1024 threads reads longer ones as long as one CU can; else rows are cut into chunks: the first launch sums them, the second finds the chunk in
// which the number lies and looks inside.
#include <algorithm>

#include "../ee_internal.hpp"
#include "../igemm_device.hpp"

namespace ee {
namespace {

struct VerifyArgs {
    VerifyCall c;
    int chunk, chunks, per;          // entries of a chunk (a multiple of 4096; 512), chunks of a row, chunks a workgroup of the first launch sums (0: no such launch, a workgroup per sequence)
    double* sums;                    // [b][chunks]
};

template <bool F32> __device__ __forceinline__ float prob(const void* base, int64_t at)
{
    if constexpr (F32) return ((const float*)base)[at];
    else return __uint_as_float((uint32_t)((const uint16_t*)base)[at] << 16);
}

__device__ __forceinline__ int drafts_of(const VerifyCall& c, int b) { return c.lengths ? min(c.lengths[b], c.k) : c.k; }

// drafts accepted, by all lanes of one wavefront, 64 drafts at a time; `drafts` itself where it is not above 0
template <bool F32>
__device__ __forceinline__ int accepted(const VerifyCall& c, int b, int drafts, int lane)
{
    for (int i0 = 0; i0 < drafts; i0 += 64) {
        const int i = i0 + lane;
        bool ok = i < drafts;
        if (ok) {
            const int x = c.draft[b * c.draft_row + i];
            const double u = c.u[b * c.u_row + i];
            ok = x >= 0 && x < c.v;
            if (ok) {
                const double p = prob<F32>(c.p, b * c.p_seq + i * c.p_row + x), q = c.q ? (double)prob<F32>(c.q, b * c.q_seq + i * c.q_row + x) : 1.0;
                ok = u * q < p;
            }
        }
        const unsigned long long good = __ballot(ok);
        if (~good) return min(drafts, i0 + (int)__builtin_ctzll(~good));
    }
    return drafts;
}

// the rows the extra token is drawn from: p, less q (minus) or without one entry (skip)
struct Rows { int64_t p, q; bool minus; int skip; };
template <bool F32>
__device__ __forceinline__ Rows rows_of(const VerifyCall& c, int b, int n, int drafts)
{
    Rows r{b * c.p_seq + n * c.p_row, 0, false, -1};
    if (n < drafts) {
        if (c.q) { r.minus = true; r.q = b * c.q_seq + n * c.q_row; }
        else r.skip = c.draft[b * c.draft_row + n];
    }
    return r;
}

// eight entries as loaded, from wherever a row starts: 16-byte loads need no alignment
template <bool F32> struct Raw8 {
    typedef float v4f __attribute__((ext_vector_type(4)));
    v4f a, b;
    __device__ __forceinline__ void load(const void* base, int64_t at)
    {
        const float* const p = (const float*)base + at;
        __builtin_memcpy(&a, p, 16);
        __builtin_memcpy(&b, p + 4, 16);
    }
    __device__ __forceinline__ void get(float (&o)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) { o[e] = a[e]; o[4 + e] = b[e]; }
    }
};
template <> struct Raw8<false> {
    v4i a;
    __device__ __forceinline__ void load(const void* base, int64_t at) { __builtin_memcpy(&a, (const uint16_t*)base + at, 16); }
    __device__ __forceinline__ void get(float (&o)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = __uint_as_float(e & 1 ? (uint32_t)a[e >> 1] & 0xFFFF0000u : (uint32_t)a[e >> 1] << 16);
    }
};

// entries j .. j + 7 of a row, 0 behind its end
template <bool F32>
__device__ __forceinline__ void load8(const void* base, int64_t row, int j, int v, float (&o)[8])
{
    if (j + 8 <= v) {
        Raw8<F32> raw;
        raw.load(base, row + j);
        raw.get(o);
    } else
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float last = prob<F32>(base, row + min(j + e, v - 1));          // all eight in flight: no branches
            o[e] = j + e < v ? last : 0.f;
        }
}

// weights of entries j .. j + 7, from p alone or from both; one that is not finite and positive is 0
template <bool P_ONLY>
__device__ __forceinline__ void weigh(const Rows& r, int j, const float (&p)[8], const float (&q)[8], double (&w)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        double t = (double)p[e];
        if (!P_ONLY && r.minus) t -= (double)q[e];
        if (!P_ONLY && j + e == r.skip) t = 0.0;
        t = fmax(t, 0.0);                                        // a NaN: 0
        w[e] = t < __builtin_inf() ? t : 0.0;
    }
}
// their sum where none is infinite and none is the one to skip: half the work of the above (a NaN counts as 0 here too)
template <bool P_ONLY>
__device__ __forceinline__ double sum8(const Rows& r, const float (&p)[8], const float (&q)[8])
{
    double w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = fmax(!P_ONLY && r.minus ? (double)p[e] - (double)q[e] : (double)p[e], 0.0);
    return ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
}
template <bool F32, bool P_ONLY>
__device__ __forceinline__ void weights8(const VerifyCall& c, const Rows& r, int j, double (&w)[8])
{
    float p[8], q[8];
    load8<F32>(c.p, r.p, j, c.v, p);
    if (!P_ONLY && r.minus) load8<F32>(c.q, r.q, j, c.v, q);
    weigh<P_ONLY>(r, j, p, q, w);
}

// v of the lane CTRL says (a data-parallel-primitive control word: shifts inside rows of 16 lanes, the last lane of a row to the next rows), 0 where there is none
template <int CTRL, int ROWS>
__device__ __forceinline__ double from_lane(double v)
{
    const long long bits = __builtin_bit_cast(long long, v);
    const int lo = __builtin_amdgcn_update_dpp(0, (int)bits, CTRL, ROWS, 0xF, false), hi = __builtin_amdgcn_update_dpp(0, (int)(bits >> 32), CTRL, ROWS, 0xF, false);
    return __builtin_bit_cast(double, (long long)(uint32_t)lo | (long long)hi << 32);
}
// the sum over the lanes up to this one
__device__ __forceinline__ double wave_scan(double v)
{
    v += from_lane<0x111, 0xF>(v);       // row_shr 1, 2, 4, 8: inside rows
    v += from_lane<0x112, 0xF>(v);
    v += from_lane<0x114, 0xF>(v);
    v += from_lane<0x118, 0xF>(v);
    v += from_lane<0x142, 0xA>(v);       // row_bcast 15: the last lane of rows 0 and 2 to rows 1 and 3
    v += from_lane<0x143, 0xC>(v);       // row_bcast 31: lane 31 to rows 2 and 3
    return v;
}
// the same over the threads of the workgroup (of NW wavefronts); all: over all of them.  Two uses of l have a barrier between them
template <int NW = 4>
__device__ __forceinline__ double block_scan(double v, double* l, double& all)
{
    const int wave = threadIdx.x >> 6;
    v = wave_scan(v);
    if ((threadIdx.x & 63) == 63) l[wave] = v;
    __syncthreads();
    double before = 0.0;
    for (int w = 0; w < wave; ++w) before += l[w];
    all = l[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) all += l[w];
    return before + v;
}

template <bool F32>
__global__ __launch_bounds__(256) void verify_sum_kernel(VerifyArgs a)
{
    __shared__ int l_n;
    __shared__ double l_sum[2][4];
    const VerifyCall& c = a.c;
    request_args<sizeof(VerifyArgs)>();
    const int share = (a.chunks + a.per - 1) / a.per, b = blockIdx.x / share, first = (blockIdx.x - b * share) * a.per, tid = threadIdx.x;
    const int drafts = drafts_of(c, b);
    if (tid < 64) {
        const int n = accepted<F32>(c, b, drafts, tid);
        if (tid == 0) {
            l_n = n;
            if (first == 0) c.accepted[b] = max(n, 0);
        }
    }
    if (drafts < 0) return;
    __syncthreads();
    const Rows r = rows_of<F32>(c, b, l_n, drafts);
    for (int k = first; k < min(first + a.per, a.chunks); ++k) {
        double s = 0.0;
        const int j0 = k * a.chunk, j1 = min(c.v, j0 + a.chunk);
#pragma unroll 2
        for (int j = j0 + tid * 8; j < j1; j += 2048) {
            double w[8];
            weights8<F32, false>(c, r, j, w);
            s += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
        }
        double all;
        block_scan(s, l_sum[k & 1], all);
        if (tid == 0) a.sums[(int64_t)b * a.chunks + k] = all;
    }
}

// ONE: the row is one chunk, nothing has been done before.  A chunk has 16 entries a thread, neighbours
template <bool F32, bool ONE>
__global__ __launch_bounds__(256) void verify_pick_kernel(VerifyArgs a)
{
    __shared__ int l_n, l_chunk, l_last_chunk, l_first, l_last;
    __shared__ double l_sum[4][4], l_before;
    const VerifyCall& c = a.c;
    request_args<sizeof(VerifyArgs)>();
    const int b = blockIdx.x, tid = threadIdx.x;
    const int drafts = drafts_of(c, b);
    const double u = c.u[b * c.u_row + c.k];
    double mine = 0.0;                                           // the thread's chunk (at most 256)
    if (!ONE && drafts >= 0 && tid < a.chunks) mine = a.sums[(int64_t)b * a.chunks + tid];
    if (tid < 64) {
        const int n = ONE ? accepted<F32>(c, b, drafts, tid) : drafts < 0 ? drafts : c.accepted[b];
        if (tid == 0) {
            l_n = n;
            if (ONE) c.accepted[b] = max(n, 0);
            l_first = l_chunk = 0x7FFFFFFF;
            l_last = l_last_chunk = -1;
        }
    }
    __syncthreads();
    const int n = l_n;
    int token = -1;
    if (drafts >= 0) {
        const Rows r = rows_of<F32>(c, b, n, drafts);
        auto entries = [&](int j, bool p_only, double (&w)[16]) {
            double lo[8], hi[8];
            if (p_only) { weights8<F32, true>(c, r, j, lo); weights8<F32, true>(c, r, j + 8, hi); }
            else { weights8<F32, false>(c, r, j, lo); weights8<F32, false>(c, r, j + 8, hi); }
#pragma unroll
            for (int e = 0; e < 8; ++e) { w[e] = lo[e]; w[8 + e] = hi[e]; }
        };
        auto sum16 = [](const double (&w)[16]) {
            double s = 0.0;
#pragma unroll
            for (int e = 0; e < 16; ++e) s += w[e];
            return s;
        };
        double w[16], total, before = 0.0, incl;
        int chunk = 0;
        bool p_only = false;
        if constexpr (ONE) {
            entries(tid * 16, false, w);
            incl = block_scan(sum16(w), l_sum[0], total);
            if (!(total > 0.0)) {                                // nothing is left of p without q: p itself
                p_only = true;
                entries(tid * 16, true, w);
                incl = block_scan(sum16(w), l_sum[1], total);
            }
        } else {
            incl = block_scan(mine, l_sum[0], total);
            if (!(total > 0.0)) {                                // the chunks of p have not been summed
                p_only = true;
                for (int k = 0; k < a.chunks; ++k) {
                    double s = 0.0, all;
                    for (int j = k * a.chunk + tid * 8; j < min(c.v, (k + 1) * a.chunk); j += 2048) {
                        double e[8];
                        weights8<F32, true>(c, r, j, e);
                        s += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
                    }
                    block_scan(s, l_sum[2 + (k & 1)], all);
                    if (tid == k) mine = all;
                }
                incl = block_scan(mine, l_sum[1], total);
            }
        }
        const double target = u * total;
        if (total > 0.0) {
            if constexpr (!ONE) {
                if (mine > 0.0 && incl > target) atomicMin(&l_chunk, tid);
                if (mine > 0.0) atomicMax(&l_last_chunk, tid);
                __syncthreads();
                chunk = min(l_chunk, l_last_chunk);              // behind all sums: the last that can be drawn from
                if (tid == chunk) l_before = incl - mine;
                __syncthreads();
                before = l_before;
            }
            // inside the chunk, 4096 entries at a time
            for (int j0 = chunk * a.chunk, turn = 2; j0 < min(c.v, (chunk + 1) * a.chunk); j0 += 4096, turn ^= 1) {
                const int j = j0 + tid * 16;
                double all = 0.0;
                if constexpr (!ONE) {
                    entries(j, p_only, w);
                    incl = before + block_scan(sum16(w), l_sum[turn], all);
                }
                if (incl > target) {
                    double cum = incl - sum16(w);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        cum += w[e];
                        if (w[e] > 0.0 && cum > target) { atomicMin(&l_first, j + e); break; }
                    }
                }
                int last = -1;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (w[e] > 0.0) last = j + e;
                if (last >= 0) atomicMax(&l_last, last);
                __syncthreads();
                if (l_first != 0x7FFFFFFF) break;
                before += all;
            }
            token = l_first != 0x7FFFFFFF ? l_first : l_last;    // behind every sum (the number is 1, or by rounding): the last entry that can be drawn
        }
    }
    for (int i = tid; i <= c.k; i += 256)
        c.tokens[b * (int64_t)(c.k + 1) + i] = drafts < 0 ? -1 : i < n ? c.draft[b * c.draft_row + i] : i == n ? token : -1;
}

// A workgroup per sequence, one launch.  Its wavefronts take segments of 512 entries (8 a lane) in turn; their sums are scanned, the segment the number lies in is read once more.  What bounds it is
// what one CU has under way: 256 KB of two rows take 6 us, 512 KB 25 us on all CUs at once, at 5.2 TB/s.
enum { SEGMENTS = 256 };
template <bool F32>
__global__ __launch_bounds__(1024) void verify_row_kernel(VerifyArgs a)
{
    constexpr int NW = 16, AHEAD = F32 ? 2 : 4;                  // AHEAD: segments whose loads a wavefront has in flight
    __shared__ int l_n, l_at, l_last;
    __shared__ double l_segment[SEGMENTS], l_sum[2][NW], l_before;
    const VerifyCall& c = a.c;
    request_args<sizeof(VerifyArgs)>();
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int drafts = drafts_of(c, b);
    const double u = c.u[b * c.u_row + c.k];
    if (wave == 0) {
        const int n = accepted<F32>(c, b, drafts, lane);
        if (lane == 0) {
            l_n = n;
            c.accepted[b] = max(n, 0);
            l_at = 0x7FFFFFFF;
            l_last = -1;
        }
    }
    __syncthreads();
    const int n = __builtin_amdgcn_readfirstlane(l_n);
    int token = -1;
    if (drafts >= 0) {
        const Rows r = rows_of<F32>(c, b, n, drafts);
        auto sums = [&](auto p_tag) {
            constexpr bool P = decltype(p_tag)::value;
            auto slow = [&](int k) {
                double w[8];
                weights8<F32, P>(c, r, k * 512 + lane * 8, w);
                return ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
            };
            auto add = [&](int k, double s) {
                s = wave_scan(s);
                if (lane == 63) l_segment[k] = s;
            };
            // whole segments: all loads, then the sums; the others entry by entry
            auto whole = [&](int k) { return k * 512 + 512 <= c.v && !(!P && r.skip >= k * 512 && r.skip < k * 512 + 512); };
            for (int k = wave; k < a.chunks; k += NW * AHEAD) {
                Raw8<F32> p[AHEAD], q[AHEAD];
#pragma unroll
                for (int e = 0; e < AHEAD; ++e)
                    if (whole(k + NW * e)) {
                        p[e].load(c.p, r.p + (k + NW * e) * 512 + lane * 8);
                        if (!P && r.minus) q[e].load(c.q, r.q + (k + NW * e) * 512 + lane * 8);
                    }
#pragma unroll
                for (int e = 0; e < AHEAD; ++e) {
                    const int at = k + NW * e;
                    if (at >= a.chunks) break;
                    double s = __builtin_inf();
                    if (whole(at)) {
                        float pf[8], qf[8];
                        p[e].get(pf);
                        if (!P && r.minus) q[e].get(qf);
                        s = sum8<P>(r, pf, qf);
                    }
                    if (!(s < __builtin_inf())) s = slow(at);                    // also where an entry of the lane's is infinite
                    add(at, s);
                }
            }
        };
        bool p_only = false;
        double total, mine, incl;
        sums(std::false_type{});
        __syncthreads();
        mine = tid < a.chunks ? l_segment[tid] : 0.0;
        incl = block_scan<NW>(mine, l_sum[0], total);
        if (!(total > 0.0)) {                                    // nothing is left of p without q: p itself
            p_only = true;
            sums(std::true_type{});
            __syncthreads();
            mine = tid < a.chunks ? l_segment[tid] : 0.0;
            incl = block_scan<NW>(mine, l_sum[1], total);
        }
        const double target = u * total;
        if (total > 0.0) {
            if (mine > 0.0 && incl > target) atomicMin(&l_at, tid);
            if (mine > 0.0) atomicMax(&l_last, tid);
            __syncthreads();
            const int at = min(l_at, l_last);                    // behind all sums: the last that can be drawn from
            if (tid == at) l_before = incl - mine;
            __syncthreads();
            if (wave > 0) return;
            const int j = at * 512 + lane * 8;
            double w[8];
            if (p_only) weights8<F32, true>(c, r, j, w);
            else weights8<F32, false>(c, r, j, w);
            const double s = ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7])), to = l_before + wave_scan(s);
            const unsigned long long past = __ballot(s > 0.0 && to > target), some = __ballot(s > 0.0);
            const int who = past ? (int)__builtin_ctzll(past) : 63 - (int)__builtin_clzll(some);
            double cum = to - s;
            int found = -1, behind = -1;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                cum += w[e];
                if (w[e] > 0.0) {
                    behind = j + e;
                    if (found < 0 && cum > target) found = behind;
                }
            }
            token = __builtin_amdgcn_readlane(found >= 0 ? found : behind, who);       // behind every sum (the number is 1, or by rounding): the last entry that can be drawn
        }
    }
    if (wave > 0) return;
    for (int i = lane; i <= c.k; i += 64)
        c.tokens[b * (int64_t)(c.k + 1) + i] = drafts < 0 ? -1 : i < n ? c.draft[b * c.draft_row + i] : i == n ? token : -1;
}

// Whether a workgroup per sequence is the way: rows that leave it little to do alone, longer ones the more CUs are at work; not for more sequences than CUs, which would wait for a second round.
// The kernel for up to 4096 entries / this, fp32, us: 128 x 256 5.7 / 5.8, 128 x 512 6.7 / 4.9, 128 x 4096 8.7 / 5.2, 512 x 4096 10.0 / 8.3, 512 x 256 6.4 / 9.0.  Two launches / this: 64 x 5000 12.0 / 6.0, 64 x 16000 12.3 / 8.0, 64 x 32000 13.2 / 11.1, 64 x 64000 15.8 / 16.0, 16 x 32000 12.3 / 12.2, 16 x 64000 12.9 / 14.8, 128 x 64000
// 22.9 / 18.1, 256 x 128256 53.7 / 45.9 (bf16 37.5 / 30.2), 300 x 16000 19.4 / 18.3, 300 x 32000 25.2 / 28.4
bool row_each(const VerifyCall& c) { return c.b <= 256 && c.v >= 512 && c.v <= std::max(24576, 512 * c.b); }

void plan_verify(const VerifyCall& c, VerifyArgs& a)
{
    a.c = c;
    a.chunk = 4096;
    if (row_each(c)) {
        a.chunk = 512;
        a.chunks = (c.v + 511) / 512;                            // at most SEGMENTS
        a.per = 0;
        return;
    }
    while ((c.v + (int64_t)a.chunk - 1) / a.chunk > 256) a.chunk *= 2;
    a.chunks = (int)((c.v + (int64_t)a.chunk - 1) / a.chunk);
    // 8 workgroups a CU are on the chip at once, so more than 2048 only repeat the decision: 256 rows of 50257, 3328 chunks, take 27.5 us with 2048, 28.8 with a chunk each
    a.per = (int)std::clamp<int64_t>((int64_t)c.b * a.chunks / 2048, 1, a.chunks);
}

}  // namespace

size_t verify_workspace(const VerifyCall& c)
{
    VerifyArgs a;
    plan_verify(c, a);
    return a.per && a.chunks > 1 ? (size_t)c.b * a.chunks * sizeof(double) : 0;
}

hipError_t launch_verify(const VerifyCall& c, void* workspace, hipStream_t s)
{
    VerifyArgs a;
    plan_verify(c, a);
    a.sums = (double*)workspace;
    const dim3 each((unsigned)c.b);
    if (!a.per) {
        if (c.f32) EE_LAUNCH(verify_row_kernel<true>, each, dim3(1024), 0, s, a);
        else EE_LAUNCH(verify_row_kernel<false>, each, dim3(1024), 0, s, a);
        return hipGetLastError();
    }
    if (a.chunks == 1) {
        if (c.f32) EE_LAUNCH((verify_pick_kernel<true, true>), each, dim3(256), 0, s, a);
        else EE_LAUNCH((verify_pick_kernel<false, true>), each, dim3(256), 0, s, a);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)((int64_t)c.b * ((a.chunks + a.per - 1) / a.per)));
    if (c.f32) EE_LAUNCH(verify_sum_kernel<true>, grid, dim3(256), 0, s, a);
    else EE_LAUNCH(verify_sum_kernel<false>, grid, dim3(256), 0, s, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (c.f32) EE_LAUNCH((verify_pick_kernel<true, false>), each, dim3(256), 0, s, a);
    else EE_LAUNCH((verify_pick_kernel<false, false>), each, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace ee
