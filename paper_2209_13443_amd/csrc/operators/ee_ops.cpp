// The C ABI of the operators that need no context: argument checks in front of their launches.
#include <algorithm>

#include "../ee_internal.hpp"

using namespace ee;

namespace {

bool aligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
int done(hipError_t e) { return e == hipSuccess ? EE_OK : EE_ERR_DEVICE; }

// Elements [samples][pixels][channels], strides and the channels' size in bytes
struct Elements { uintptr_t at; int64_t sample, pixel, channels; };

// Whether no byte belongs to both: they lie one behind the other, or take turns -- pixel by pixel (channel slices of one wider tensor) or sample by sample
bool apart(const Elements& p, const Elements& q, int64_t samples, int64_t pixels)
{
    typedef __int128 wide;
    auto first = [&](const Elements& e) { return (wide)e.at + std::min<wide>(0, (wide)(samples - 1) * e.sample); };
    auto extent = [&](const Elements& e) { return (wide)(samples - 1) * (e.sample < 0 ? -(wide)e.sample : e.sample) + (wide)(pixels - 1) * e.pixel + e.channels; };
    if (first(p) + extent(p) <= first(q) || first(q) + extent(q) <= first(p)) return true;
    // windows of lp and lq bytes, repeated every `pitch` bytes
    auto turns = [&](wide pitch, wide lp, wide lq) {
        const wide d = ((first(q) - first(p)) % pitch + pitch) % pitch;
        return d >= lp && d + lq <= pitch;
    };
    // what the samples take up of a pixel's pitch: one place, or places next to one another
    auto window = [&](const Elements& e) { return samples == 1 || e.sample % e.pixel == 0 ? (wide)e.channels : extent(e) - (wide)(pixels - 1) * e.pixel; };
    if (pixels > 1 && p.pixel == q.pixel && p.pixel > 0 && turns(p.pixel, window(p), window(q))) return true;
    const wide sample = p.sample < 0 ? -(wide)p.sample : p.sample;
    return samples > 1 && p.sample == q.sample && sample > 0 && turns(sample, (wide)(pixels - 1) * p.pixel + p.channels, (wide)(pixels - 1) * q.pixel + q.channels);
}

int check_norm(const ee_norm_desc* d, NormArgs& a)
{
    if (!d) return EE_ERR_ARG;
    if (d->dtype != EE_I8 && d->dtype != EE_BF16) return EE_ERR_UNSUPPORTED;
    if (d->b < 0 || d->pixels < 0 || d->c < 1 || d->groups < 1 || d->c % d->groups != 0) return EE_ERR_ARG;
    if (!(d->eps >= 0.f) || !std::isfinite(d->eps) || d->frac_bits < 0 || d->frac_bits > 7 || d->res_shift < -8 || d->res_shift > 8) return EE_ERR_ARG;
    if (d->act < EE_ACT_NONE || d->act > EE_ACT_SILU) return EE_ERR_ARG;
    if (d->dtype == EE_I8 && d->act == EE_ACT_SILU) return EE_ERR_UNSUPPORTED;
    if ((int64_t)d->pixels * d->c >= 1ll << 31 || (d->dtype == EE_I8 && (int64_t)d->pixels * (d->c / d->groups) >= 1 << 24)) return EE_ERR_OVERFLOW;
    const int64_t es = d->dtype == EE_I8 ? 1 : 2;
    if (d->pixels > 1) {
        for (const int64_t stride : {d->x_pixel, d->res_pixel, d->y_pixel})
            if (stride < 0) return EE_ERR_ARG;
        if (d->y_pixel < d->c) return EE_ERR_ARG;
        for (const int64_t stride : {d->x_pixel, d->res_pixel, d->y_pixel})
            if (stride >= 1 << 20 || ((d->pixels + 1024ll) * stride + d->c) * es >= 1ll << 31) return EE_ERR_OVERFLOW;
    }
    a = NormArgs{};
    a.dtype = d->dtype; a.act = d->act; a.b = d->b; a.pixels = d->pixels; a.c = d->c; a.groups = d->groups; a.frac_bits = d->frac_bits; a.res_shift = d->res_shift; a.eps = d->eps;
    a.x_sample = d->x_sample; a.x_pixel = d->x_pixel; a.res_sample = d->res_sample; a.res_pixel = d->res_pixel; a.y_sample = d->y_sample; a.y_pixel = d->y_pixel;
    if (a.pixels == 1) a.x_pixel = a.res_pixel = a.y_pixel = a.c;
    return EE_OK;
}

int check_dims(const ee_adapter_dims* d, AdapterDims& a)
{
    if (!d || d->ci < 1 || d->co < 1 || d->adapters < 0 || d->rank < 0 || (d->adapters > 0 && d->rank < 1)) return EE_ERR_ARG;
    if (d->ci > 1 << 18 || d->co > 1 << 18 || d->adapters > 65536 || d->rank > 256) return EE_ERR_OVERFLOW;
    a = AdapterDims{d->ci, d->co, d->adapters, d->rank};
    return EE_OK;
}

}  // namespace

extern "C" int ee_group_norm_workspace(const ee_norm_desc* desc, int64_t* bytes)
{
    NormArgs a;
    if (!bytes) return EE_ERR_ARG;
    if (const int rc = check_norm(desc, a)) return rc;
    *bytes = a.b && a.pixels ? (int64_t)group_norm_workspace(a) : 0;
    return EE_OK;
}

extern "C" int ee_group_norm(const ee_norm_desc* desc, const void* x, const float* weight, const float* bias, const void* res, void* y,
                             void* workspace, int64_t workspace_bytes, void* hip_stream)
{
    NormArgs a;
    if (const int rc = check_norm(desc, a)) return rc;
    if (a.b == 0 || a.pixels == 0) return EE_OK;
    const int64_t es = a.dtype == EE_I8 ? 1 : 2;
    if (!x || !y || !aligned(x, (unsigned)es) || !aligned(y, (unsigned)es) || !aligned(res, (unsigned)es) || !aligned(weight, 4) || !aligned(bias, 4)) return EE_ERR_ARG;
    a.x = x; a.res = res; a.y = y; a.weight = weight; a.bias = bias;
    if (const int rc = group_norm_check(a)) return rc;
    const size_t need = group_norm_workspace(a);
    if (need && (!workspace || !aligned(workspace, 256))) return EE_ERR_ARG;
    if (workspace_bytes < (int64_t)need) return EE_ERR_OVERFLOW;
    // y is x, or res, or shares nothing with it
    auto elements = [&](const void* at, int64_t sample, int64_t pixel) { return Elements{(uintptr_t)at, a.b == 1 ? 0 : es * sample, a.pixels == 1 ? 0 : es * pixel, (int64_t)es * a.c}; };
    const Elements of_y = elements(y, a.y_sample, a.y_pixel);
    for (const Elements& e : {elements(x, a.x_sample, a.x_pixel), res ? elements(res, a.res_sample, a.res_pixel) : of_y})
        if (!(e.at == of_y.at && e.sample == of_y.sample && e.pixel == of_y.pixel) && !apart(e, of_y, a.b, a.pixels)) return EE_ERR_ARG;
    return done(launch_group_norm(a, workspace, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int ee_adapter_bytes(const ee_adapter_dims* dims, int64_t* packed_bytes, int64_t* pool_bytes)
{
    AdapterDims d;
    if (!packed_bytes || !pool_bytes) return EE_ERR_ARG;
    if (const int rc = check_dims(dims, d)) return rc;
    *packed_bytes = adapter_weight_bytes(d);
    *pool_bytes = adapter_pool_bytes(d);
    return EE_OK;
}

extern "C" int ee_adapter_pack(const ee_adapter_dims* dims, const void* w, int64_t ldw, const float* bias, void* packed, void* hip_stream)
{
    AdapterDims d;
    if (const int rc = check_dims(dims, d)) return rc;
    if (!w || !packed || ldw < d.ci || !aligned(w, 2) || !aligned(bias, 4) || !aligned(packed, 256)) return EE_ERR_ARG;
    return done(launch_adapter_pack(d, w, ldw, bias, packed, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int ee_adapter_load(const ee_adapter_dims* dims, int i, int rank, const void* a, int64_t lda, const void* b, int64_t ldb, float scale, void* pool, void* hip_stream)
{
    AdapterDims d;
    if (const int rc = check_dims(dims, d)) return rc;
    if (i < 0 || i >= d.adapters || rank < 0 || rank > d.rank || !pool || !aligned(pool, 256)) return EE_ERR_ARG;
    if (rank > 0 && (!a || !b || lda < d.ci || ldb < rank || !aligned(a, 2) || !aligned(b, 2))) return EE_ERR_ARG;
    return done(launch_adapter_load(d, i, rank, a, lda, b, ldb, rank ? scale : 0.f, pool, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int ee_adapter_workspace(const ee_adapter_dims* dims, int rows, int64_t* bytes)
{
    AdapterDims d;
    if (!bytes || rows < 0) return EE_ERR_ARG;
    if (const int rc = check_dims(dims, d)) return rc;
    if (rows > 1 << 22) return EE_ERR_OVERFLOW;
    *bytes = adapter_workspace(d, rows);
    return EE_OK;
}

extern "C" int ee_adapter_project(const ee_adapter_dims* dims, const ee_adapter_call* call, void* hip_stream)
{
    AdapterDims d;
    if (const int rc = check_dims(dims, d)) return rc;
    if (!call || call->rows < 0 || call->slots < 0) return EE_ERR_ARG;
    const ee_adapter_call& q = *call;
    if (!q.offsets && (q.per < 0 || (int64_t)q.slots * q.per != q.rows)) return EE_ERR_ARG;
    if (q.rows == 0 || q.slots == 0) return EE_OK;
    if (q.rows > 1 << 22) return EE_ERR_OVERFLOW;
    if (!q.packed || !q.x || !q.y || q.ldx < d.ci || q.ldy < d.co || !aligned(q.packed, 256) || !aligned(q.x, 2) || !aligned(q.y, q.out_f32 ? 4 : 2)) return EE_ERR_ARG;
    if (d.adapters > 0 && (!q.pool || !q.ids || !aligned(q.pool, 256))) return EE_ERR_ARG;
    if (!aligned(q.ids, 4) || !aligned(q.offsets, 4) || !q.workspace || !aligned(q.workspace, 256)) return EE_ERR_ARG;
    if (q.workspace_bytes < adapter_workspace(d, q.rows)) return EE_ERR_OVERFLOW;
    if (!apart({(uintptr_t)q.x, 0, 2 * q.ldx, 2ll * d.ci}, {(uintptr_t)q.y, 0, (q.out_f32 ? 4 : 2) * q.ldy, (q.out_f32 ? 4ll : 2ll) * d.co}, 1, q.rows)) return EE_ERR_ARG;
    AdapterCall c{q.packed, q.pool, q.x, q.y, q.workspace, q.ids, q.offsets, q.ldx, q.ldy, q.rows, q.slots, q.per, q.out_f32};
    return done(launch_adapter_project(d, c, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int ee_verify_workspace(int b, int k, int v, int64_t* bytes)
{
    if (!bytes || b < 0 || k < 0 || v < 1) return EE_ERR_ARG;
    VerifyCall c{};
    c.b = b; c.k = k; c.v = v;
    if (v > 1 << 30) return EE_ERR_OVERFLOW;
    *bytes = (int64_t)verify_workspace(c);
    return EE_OK;
}

extern "C" int ee_verify_draft(const ee_verify_call* call, void* hip_stream)
{
    if (!call || call->b < 0 || call->k < 0 || call->v < 1) return EE_ERR_ARG;
    const ee_verify_call& q = *call;
    if (q.b == 0) return EE_OK;
    const unsigned es = q.f32 ? 4 : 2;
    if ((!q.draft && q.k) || !q.p || !q.u || !q.accepted || !q.tokens || !aligned(q.p, es) || !aligned(q.q, es)) return EE_ERR_ARG;
    if (!aligned(q.draft, 4) || !aligned(q.u, 4) || !aligned(q.lengths, 4) || !aligned(q.accepted, 4) || !aligned(q.tokens, 4)) return EE_ERR_ARG;
    VerifyCall c{q.draft, q.p, q.q, q.u, q.lengths, q.accepted, q.tokens, q.draft_row, q.u_row, q.p_seq, q.p_row, q.q_seq, q.q_row, q.b, q.k, q.v, q.f32};
    if (q.v > 1 << 30 || (int64_t)q.b * (q.k + 1ll) > 1 << 28 || (int64_t)q.b * 256 > 1ll << 31) return EE_ERR_OVERFLOW;
    const size_t need = verify_workspace(c);
    if (need && (!q.workspace || !aligned(q.workspace, 256))) return EE_ERR_ARG;
    if (q.workspace_bytes < (int64_t)need) return EE_ERR_OVERFLOW;
    return done(launch_verify(c, q.workspace, static_cast<hipStream_t>(hip_stream)));
}
