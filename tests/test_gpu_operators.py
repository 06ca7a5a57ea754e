"""The operators that are calls of their own (group norm with an activation, projection with per-request adapters, verification of
drafted tokens) against their definitions in 64 bits, at the sizes, strides and values where they can go wrong.

Tolerances: one rounding of the result (half a step, 2^-8 relative in bf16, 2^-24 in float32) plus what float sums of the given
length may lose (a step of 2^-24 of the sum of the terms' magnitudes per addition, at the most)."""
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
EPS = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
F32 = 2.0 ** -24


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


@pytest.fixture(scope="module")
def ee():
    import paper_2209_13443_amd as ee
    return ee


# ---- group norm -------------------------------------------------------------------------------------------------------------------
def over(t, f):
    """f ("sum", "amax") over pixels and a group's channels, the pixels on the CPU: the library's reductions of few results over many workgroups have given wrong ones here now and then (the
    same call again another value, the operator's result the same)."""
    return getattr(getattr(t, f)(3, keepdim=True).cpu(), f)(1, keepdim=True).to(t.device)


def norm_ref(torch, x, groups, w, b, eps, act, res, f=0, rs=0):
    """(result, bound) in 64 bits; x [b, p, c]"""
    n_b, pix, c = x.shape
    cpg = c // groups
    w = torch.ones(c, dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros(c, dtype=torch.float64, device=x.device) if b is None else b.double()
    if x.dtype == torch.int8:
        xi = x.long().view(n_b, pix, groups, cpg)
        n = pix * cpg
        s1, s2 = over(xi, "sum"), over(xi * xi, "sum")
        var = (n * s2 - s1 * s1).double() / float(n) ** 2
        t = (n * xi - s1).double() * (w.view(groups, cpg) * 2.0 ** f / (n * (var + np.float32(eps)).sqrt())) + (b.view(groups, cpg) * 2.0 ** f + 0.5)
        t = t.view(x.shape)
        if res is not None:
            t = t + res.double() * 2.0 ** rs
        lo, hi = {"none": (-128, 127), "relu": (0, 127), "relu6": (0, min(127, 6 * 2 ** f))}[act]
        return t.floor().clamp(lo, hi).to(torch.int8), None
    xd = x.double().view(n_b, pix, groups, cpg)
    mean = over(xd, "sum") / (pix * cpg)
    a = w.view(groups, cpg) / (over((xd - mean).square(), "sum") / (pix * cpg) + np.float32(eps)).sqrt()
    y = ((xd - mean) * a + b.view(groups, cpg)).view(x.shape)
    # the mean and the variance from at most a few dozen additions behind one another each, of numbers as large as the largest
    size = (((xd - mean).abs() + over(xd.abs(), "amax")) * a.abs()).view(x.shape) + b.abs()
    if res is not None:
        y = y + res.double()
        size = size + res.double().abs()
    y = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "relu6": lambda v: v.clamp(0, 6), "silu": lambda v: v * torch.sigmoid(v)}[act](y)
    return y, EPS["bf16"] * y.abs() + 128 * F32 * size + 1e-30


NORM_SHAPES = [  # b, h, w, c, groups
    (1, 1, 1, 8, 8), (1, 1, 1, 1, 1), (3, 1, 1, 64, 4), (2, 7, 7, 512, 32), (5, 3, 5, 24, 3), (2, 9, 11, 96, 12), (3, 5, 7, 33, 3), (2, 13, 13, 40, 20), (1, 56, 56, 64, 32),
    (2, 31, 33, 288, 24), (1, 100, 100, 16, 2), (1, 1, 1, 8192, 1), (2, 2, 3, 1030, 1030), (1, 130, 120, 64, 32), (1, 300, 260, 32, 4), (2, 70, 70, 1024, 1), (1, 67, 61, 7, 7), (3, 20, 20, 1000, 5),
    (2, 17, 19, 272, 16), (1, 90, 91, 80, 4), (1, 70, 60, 56, 2), (1, 65, 66, 2056, 4)]


@pytest.mark.parametrize("dtype", ["bf16", "int8"])
@pytest.mark.parametrize("shape", NORM_SHAPES)
def test_group_norm_shapes(torch, ee, shape, dtype):
    b, h, w, c, groups = shape
    g = torch.Generator(device="cuda").manual_seed(h * w + c)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    kind = torch.bfloat16 if dtype == "bf16" else torch.int8
    x = (rnd(b, h, w, c) * 2 + rnd(c)).to(kind) if dtype == "bf16" else (rnd(b, h, w, c) * 40 + 10 * rnd(c)).clamp(-128, 127).to(kind)
    res = rnd(b, h, w, c).mul_(30 if dtype == "int8" else 1).clamp(-128, 127).to(kind)
    wt, bs = 1 + 0.3 * rnd(c), 0.5 * rnd(c)
    for act, r, aff in (("none", None, False), ("relu", res, True), ("silu" if dtype == "bf16" else "relu6", None, True)):
        say(f"[case] norm {shape} {dtype} {act} residual {r is not None}")
        got = ee.group_norm(x, groups, wt if aff else None, bs if aff else None, act=act, residual=r, frac_bits=4, res_shift=-1)
        torch.cuda.synchronize()
        flat = lambda t: None if t is None else t.reshape(b, h * w, c)
        ref, tol = norm_ref(torch, flat(x), groups, wt if aff else None, bs if aff else None, 1e-5, act, flat(r), 4, -1)
        got = got.reshape(b, h * w, c)
        if tol is None:
            assert torch.equal(got, ref), f"{int((got != ref).sum())} of {ref.numel()} differ"
        else:
            off = (got.double() - ref).abs() - tol
            assert float(off.max()) <= 0, f"off by {float(off.max())} more than the bound"


@pytest.mark.parametrize("dtype", ["bf16", "int8"])
def test_group_norm_slices_strides_and_in_place(torch, ee, dtype):
    kind = torch.bfloat16 if dtype == "bf16" else torch.int8
    g = torch.Generator(device="cuda").manual_seed(3)
    wide = (torch.randn(4, 6, 5, 96, device="cuda", generator=g) * 20).to(kind)
    for c0, c1, groups in ((0, 32, 4), (32, 80, 3), (1, 34, 3), (90, 96, 2)):
        say(f"[case] slice {c0}:{c1} {dtype}")
        x = wide[:, :, :, c0:c1]
        ref, tol = norm_ref(torch, x.reshape(4, 30, c1 - c0), groups, None, None, 1e-5, "relu", None, 5)
        out = wide.clone()
        got = ee.group_norm(x, groups, act="relu", frac_bits=5, out=out[..., c0:c1])
        plain = ee.group_norm(x.contiguous(), groups, act="relu", frac_bits=5)
        here = wide.clone()
        ee.group_norm(here[..., c0:c1], groups, act="relu", frac_bits=5, out=here[..., c0:c1])
        torch.cuda.synchronize()
        assert (torch.equal(got.reshape(ref.shape), ref) if tol is None else bool(((got.reshape(ref.shape).double() - ref).abs() <= tol).all()))
        near = lambda a, b: torch.equal(a, b) if dtype == "int8" else bool(((a.double() - b.double()).abs() <= 2 * tol.view(a.shape)).all())
        assert near(plain, got) and near(here[..., c0:c1], got)
        keep = torch.ones(96, dtype=torch.bool, device="cuda")
        keep[c0:c1] = False
        assert torch.equal(out[..., keep], wide[..., keep]) and torch.equal(here[..., keep], wide[..., keep])     # the rest of the wide tensor is left alone
    # every other sample; a large tensor (two launches) in place
    x = (torch.randn(4, 90, 90, 64, device="cuda", generator=g) * 20).to(kind)
    ref, tol = norm_ref(torch, x[::2].reshape(2, 8100, 64), 8, None, None, 1e-5, "none", None, 5)
    got = x.clone()
    ee.group_norm(got[::2], 8, frac_bits=5, out=got[::2])
    assert (torch.equal(got[::2].reshape(ref.shape), ref) if tol is None else bool(((got[::2].reshape(ref.shape).double() - ref).abs() <= tol).all()))
    assert torch.equal(got[1::2], x[1::2])


@pytest.mark.parametrize("pixels", [1, 49, 4100, 40000])
def test_group_norm_values(torch, ee, pixels):
    """Constant groups, a mean far from zero, extreme int8 values, a NaN and an infinity that stay in their own group and sample."""
    c, groups = 32, 4
    bias = torch.linspace(-1, 1, c, device="cuda")
    const = torch.full((2, pixels, c), 3.0, device="cuda").to(torch.bfloat16)
    got = ee.group_norm(const, groups, None, bias)
    assert torch.equal(got, bias.to(torch.bfloat16).expand_as(got))
    q = torch.full((2, pixels, c), -128, dtype=torch.int8, device="cuda")
    half = torch.full((c,), 0.5, device="cuda")
    assert bool((ee.group_norm(q, groups, None, half, frac_bits=0) == 1).all())                  # floor(0.5 + 0.5): on the border, on every machine
    g = torch.Generator(device="cuda").manual_seed(pixels)
    ends = torch.where(torch.rand(2, pixels, c, device="cuda", generator=g) < 0.5, -128, 127).to(torch.int8)
    ref, _ = norm_ref(torch, ends, groups, None, bias, 1e-5, "none", None, 5)
    assert torch.equal(ee.group_norm(ends, groups, None, bias, frac_bits=5), ref)
    far = (300 + torch.randn(2, pixels, c, device="cuda", generator=g) * 4).to(torch.bfloat16)
    ref, tol = norm_ref(torch, far, groups, None, bias, 1e-5, "none", None)
    assert bool(((ee.group_norm(far, groups, None, bias).double() - ref).abs() <= tol).all())
    x = torch.randn(3, pixels, c, device="cuda", generator=g).to(torch.bfloat16)
    clean = ee.group_norm(x, groups, None, bias, act="silu")
    x[1, pixels // 2, 9] = float("nan")
    x[2, pixels - 1, 0] = float("inf")
    got = ee.group_norm(x, groups, None, bias, act="silu")
    assert bool(got[1, :, 8:16].isnan().all()) and bool(got[2, :, :8].isnan().all())
    same = torch.ones_like(got, dtype=torch.bool)
    same[1, :, 8:16] = False
    same[2, :, :8] = False
    assert torch.equal(got[same], clean[same])
    assert ee.group_norm(x[:0], groups).shape == (0, pixels, c)


def test_group_norm_bits_as_int16_and_refusals(torch, ee):
    x = torch.randn(2, 4, 4, 16, device="cuda").to(torch.bfloat16)
    got = ee.group_norm(x.view(torch.int16), 4, act="relu")
    assert got.dtype == torch.int16 and torch.equal(got.view(torch.bfloat16), ee.group_norm(x, 4, act="relu"))

    def refused(code, *a, **k):
        with pytest.raises(ee.EEError) as e:
            ee.group_norm(*a, **k)
        assert e.value.code == code, e.value
    refused(ee.EE_ERR_ARG, x, 3)
    refused(ee.EE_ERR_ARG, x, 0)
    refused(ee.EE_ERR_ARG, x, 4, act="gelu")
    refused(ee.EE_ERR_ARG, x, 4, eps=float("nan"))
    refused(ee.EE_ERR_ARG, x, 4, eps=-1.0)
    refused(ee.EE_ERR_UNSUPPORTED, x.to(torch.int8), 4, act="silu")
    refused(ee.EE_ERR_UNSUPPORTED, x.float(), 4)
    refused(ee.EE_ERR_ARG, x, 4, weight=torch.ones(8, device="cuda"))
    refused(ee.EE_ERR_ARG, x, 4, weight=torch.ones(16))
    refused(ee.EE_ERR_UNSUPPORTED, x, 4, weight=torch.ones(16, device="cuda", dtype=torch.bfloat16))
    refused(ee.EE_ERR_ARG, x, 4, residual=x[:1])
    refused(ee.EE_ERR_ARG, x.permute(0, 3, 1, 2), 4)
    refused(ee.EE_ERR_ARG, x.transpose(1, 2)[:, :, :3], 4)                     # pixels that are no one stride apart
    refused(ee.EE_ERR_UNSUPPORTED, torch.zeros(1, 1, 8200, device="cuda", dtype=torch.bfloat16), 1)


# ---- projection with adapters -----------------------------------------------------------------------------------------------------------
def project_ref(torch, x, w, bias, ad, rows_ids, out):
    """(result, bound) in 64 bits; ad: list of (a, b, scale); x [rows, ci]"""
    xd, wd = x.double(), w.double()
    y, size = xd @ wd.T, xd.abs() @ wd.abs().T
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    extra = torch.zeros_like(y)
    for i, (a, b, s) in enumerate(ad):
        at = (rows_ids == i).nonzero()[:, 0]
        if at.numel() and a is not None:
            y[at] += s * ((xd[at] @ a.double().T) @ b.double().T)
            extra[at] = abs(s) * ((xd[at].abs() @ a.double().abs().T) @ b.double().abs().T)
    ci = x.shape[1]
    # float sums of ci terms, of the rank's for the adapter (whose inner sums are rounded to 2^-18, or 2^-24 for float results)
    return y, EPS[out] * y.abs() + (ci + 8) * F32 * (size + extra) + ({"bf16": 2.0 ** -18, "fp32": F32}[out] + 520 * F32) * extra + 1e-30


def adapters_of(torch, g, n, r, ci, co):
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    return [((rnd(r, ci) / ci ** 0.5).bfloat16(), (rnd(co, r) / r ** 0.5).bfloat16(), 0.5 + i) for i in range(n)]


PROJECTIONS = [  # slots, per, ci, co, rank, adapters
    (1, 1, 8, 8, 1, 1), (1, 1, 1, 1, 1, 2), (3, 1, 33, 5, 4, 2), (12, 1, 512, 1000, 16, 5), (64, 1, 2048, 100, 8, 24), (70, 1, 100, 300, 10, 70), (5, 49, 256, 64, 32, 3), (7, 9, 72, 130, 128, 4),
    (2, 200, 320, 512, 64, 2), (40, 16, 96, 1001, 16, 7), (300, 1, 128, 257, 33, 9), (2, 1, 4096, 4096, 16, 2), (33, 4, 1000, 96, 256, 2), (4, 70, 64, 32, 16, 0), (16, 33, 513, 65, 5, 16),
    (17, 1, 256, 2048, 16, 17), (130, 3, 64, 640, 40, 30)]


@pytest.mark.parametrize("case", PROJECTIONS)
def test_adapter_projection_shapes(torch, ee, case):
    slots, per, ci, co, r, n = case
    g = torch.Generator(device="cuda").manual_seed(ci * 7 + co)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    w, bias, ad = (rnd(co, ci) / ci ** 0.5).bfloat16(), rnd(co), adapters_of(torch, g, n, r, ci, co)
    proj = ee.AdapterProjection(w, bias, adapters=n, rank=r)
    for i, (a, b, s) in enumerate(ad):
        proj.load(i, a, b, s)
    x = rnd(slots, per, ci).bfloat16()
    ids = torch.randint(-2, n + 2, (slots,), device="cuda", generator=g, dtype=torch.int32)            # some in front of and behind the adapters: none
    for out in ("bf16", "fp32"):
        say(f"[case] project {case} {out}")
        got = proj(x, ids if n else None, dtype=torch.bfloat16 if out == "bf16" else torch.float32)
        torch.cuda.synchronize()
        ref, tol = project_ref(torch, x.view(-1, ci), w, bias, ad, ids.repeat_interleave(per), out)
        off = (got.view(-1, co).double() - ref).abs() - tol
        assert got.shape == (slots, per, co) and float(off.max()) <= 0, f"off by {float(off.max())} more than the bound"


@pytest.mark.parametrize("ci,co,r", [(64, 96, 16), (72, 33, 8), (45, 200, 64)])
@pytest.mark.parametrize("lengths", [(0, 5, 0, 1, 40, 0), (1,), (0, 0), (200, 1, 1, 130), (3,) * 50])
def test_adapter_projection_packed_rows(torch, ee, ci, co, r, lengths):
    """Runs of different lengths, empty ones too; rows in front of the first and behind the last slot are left as they were and may hold anything."""
    g = torch.Generator(device="cuda").manual_seed(sum(lengths) + ci)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    n, front, behind = 4, 3, 37
    w, ad = (rnd(co, ci) / ci ** 0.5).bfloat16(), adapters_of(torch, g, n, r, ci, co)
    proj = ee.AdapterProjection(w, None, adapters=n, rank=r)
    for i, (a, b, s) in enumerate(ad):
        proj.load(i, a, b, s)
    rows = front + sum(lengths) + behind
    x = rnd(rows, ci).bfloat16()
    x[:front] = float("nan")
    x[rows - behind:] = float("inf")
    offsets = torch.tensor([front + sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32, device="cuda")
    ids = torch.randint(-1, n, (len(lengths),), device="cuda", generator=g, dtype=torch.int32)
    out = torch.full((rows, co), 7.0, device="cuda").bfloat16()
    say(f"[case] packed {lengths} {ci} {co} {r}")
    assert proj(x, ids, offsets=offsets, out=out) is out
    torch.cuda.synchronize()
    mine = slice(front, rows - behind)
    assert bool((out[:front] == 7).all()) and bool((out[rows - behind:] == 7).all())
    if sum(lengths):
        ref, tol = project_ref(torch, x[mine], w, None, ad, ids.repeat_interleave(torch.tensor(lengths, device="cuda")), "bf16")
        assert bool(((out[mine].double() - ref).abs() <= tol).all())


def test_adapter_projection_strides_loading_and_rows_apart(torch, ee):
    g = torch.Generator(device="cuda").manual_seed(11)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    ci, co, n = 120, 72, 3
    wide = rnd(co, ci + 9).bfloat16()
    w, ad = wide[:, 3:3 + ci], adapters_of(torch, g, n, 8, ci, co)
    proj = ee.AdapterProjection(w, None, adapters=n, rank=12)
    ids = torch.arange(20, device="cuda", dtype=torch.int32) % (n + 1)
    base = proj(rnd(20, ci).bfloat16(), ids)                                   # nothing loaded: no adapter adds anything
    assert bool(base.isfinite().all())
    for i, (a, b, s) in enumerate(ad):
        proj.load(i, a, b, s)
    for lead, step in ((0, ci), (0, ci + 8), (8, ci + 24), (1, ci + 5)):
        big = rnd(20, lead + step + 8).bfloat16()
        x = big[:, lead:lead + ci]
        out = torch.full((20, co + 11), 5.0, device="cuda")
        say(f"[case] rows {lead} {step}")
        proj(x, ids, out=out[:, 4:4 + co], dtype=torch.float32)
        ref, tol = project_ref(torch, x, w, None, ad, ids, "fp32")
        assert bool(((out[:, 4:4 + co].double() - ref).abs() <= tol).all()) and bool((out[:, :4] == 5).all()) and bool((out[:, 4 + co:] == 5).all())
    # a smaller adapter in place of a larger one, one taken out, between calls
    a, b, _ = adapters_of(torch, g, 1, 2, ci, co)[0]
    proj.load(1, a, b, -3.0)
    proj.unload(2)
    now = [ad[0], (a, b, -3.0), (None, None, 0.0)]
    x = rnd(20, ci).bfloat16()
    ref, tol = project_ref(torch, x, w, None, now, ids, "bf16")
    assert bool(((proj(x, ids).double() - ref).abs() <= tol).all())
    # a row that is not finite stays alone, whatever adapter it has
    clean = proj(x, ids)
    for row in (0, 1, 19):
        bad = x.clone()
        bad[row, 5] = float("nan")
        got = proj(bad, ids)
        rest = torch.arange(20, device="cuda") != row
        assert bool(got[row].isnan().all()) and torch.equal(got[rest], clean[rest])


def test_adapter_projection_refusals(torch, ee):
    w = torch.zeros(32, 16, device="cuda", dtype=torch.bfloat16)
    proj = ee.AdapterProjection(w, adapters=2, rank=4)
    x = torch.zeros(6, 16, device="cuda", dtype=torch.bfloat16)
    ids = torch.zeros(6, device="cuda", dtype=torch.int32)

    def refused(code, f, *a, **k):
        with pytest.raises(ee.EEError) as e:
            f(*a, **k)
        assert e.value.code == code, e.value
    refused(ee.EE_ERR_ARG, proj, x)                                            # adapters, and no ids
    refused(ee.EE_ERR_ARG, proj, x, ids[:5])
    refused(ee.EE_ERR_UNSUPPORTED, proj, x, ids.long())
    refused(ee.EE_ERR_ARG, proj, x[:, :8], ids)
    refused(ee.EE_ERR_UNSUPPORTED, proj, x.float(), ids)
    refused(ee.EE_ERR_UNSUPPORTED, proj, x, ids, dtype=torch.float16)
    refused(ee.EE_ERR_ARG, proj, x, ids, out=torch.zeros(6, 31, device="cuda", dtype=torch.bfloat16))
    refused(ee.EE_ERR_ARG, proj, x, ids, offsets=torch.zeros(6, device="cuda", dtype=torch.int32))
    refused(ee.EE_ERR_ARG, proj, x.cpu(), ids)
    refused(ee.EE_ERR_ARG, proj.load, 2, x[:4], w[:, :4])
    refused(ee.EE_ERR_ARG, proj.load, 0, x[:5], w[:, :5])
    refused(ee.EE_ERR_ARG, proj.load, 0, x[:4], w[:, :3])
    refused(ee.EE_ERR_OVERFLOW, ee.AdapterProjection, w, adapters=2, rank=300)
    assert proj(x[:0], ids[:0]).shape == (0, 32)


# ---- verification -----------------------------------------------------------------------------------------------------------------------
def verify_ref(draft, p, q, u, lengths):
    """numpy, 64 bits; p [b, k + 1, v] float64"""
    b, k = draft.shape
    v = p.shape[2]
    accepted, tokens = np.zeros(b, np.int32), np.full((b, k + 1), -1, np.int32)
    fine = lambda w: np.where((w > 0) & np.isfinite(w), w, 0.0)
    for i in range(b):
        m = k if lengths is None else min(int(lengths[i]), k)
        if m < 0:
            continue
        n = 0
        while n < m and 0 <= draft[i, n] < v and float(u[i, n]) * (1.0 if q is None else q[i, n, draft[i, n]]) < p[i, n, draft[i, n]]:
            tokens[i, n] = draft[i, n]
            n += 1
        w = p[i, n]
        if n < m:
            less = np.zeros(v) if q is None else q[i, n]
            w = fine(w - less)
            if q is None and 0 <= draft[i, n] < v:
                w[draft[i, n]] = 0.0
            if not w.sum() > 0:
                w = p[i, n]
        w = fine(w)
        accepted[i] = n
        if w.sum() > 0:
            cum = np.cumsum(w)
            over = np.nonzero((cum > float(u[i, k]) * cum[-1]) & (w > 0))[0]
            tokens[i, n] = over[0] if over.size else np.nonzero(w > 0)[0][-1]
    return accepted, tokens


def check_verify(torch, ee, draft, p, q, u, lengths, what):
    say(f"[case] verify {what}")
    got = ee.verify_draft(draft, p, u, draft_probs=q, lengths=lengths)
    again = ee.verify_draft(draft, p, u, draft_probs=q, lengths=lengths)
    torch.cuda.synchronize()
    host = lambda t: None if t is None else t.double().cpu().numpy()
    ref = verify_ref(draft.cpu().numpy(), host(p), host(q), u.cpu().numpy(), None if lengths is None else lengths.cpu().numpy())
    assert np.array_equal(got[0].cpu().numpy(), ref[0]), what
    bad = np.nonzero(got[1].cpu().numpy() != ref[1])
    assert bad[0].size == 0, f"{what}: {[(int(i), int(j), int(got[1][i, j]), int(ref[1][i, j])) for i, j in zip(*bad)][:5]}"
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    return got


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("b,k,v", [(1, 0, 1), (1, 1, 1), (4, 3, 2), (7, 4, 100), (16, 5, 1000), (3, 70, 37), (9, 2, 4096), (9, 2, 4097), (5, 8, 33001), (2, 1, 128256), (1, 2, 1100000)])
def test_verify_draft_shapes(torch, ee, b, k, v, dtype):
    kind = torch.float32 if dtype == "fp32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(b * 100 + k * 10 + v)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    logits = 2 * rnd(b, k + 1, v)
    p = torch.softmax(logits, -1).to(kind)
    weak = logits[:, :k] + 0.5 * rnd(b, k, v)
    q = torch.softmax(weak, -1).to(kind)
    draft = (weak - torch.empty_like(weak).exponential_(generator=g).log_()).argmax(-1).int() if k else torch.zeros(b, 0, dtype=torch.int32, device="cuda")
    u = torch.rand(b, k + 1, device="cuda", generator=g)
    lengths = torch.randint(-1, k + 2, (b,), device="cuda", generator=g, dtype=torch.int32)
    for qq in (q, None):
        for ll in (None, lengths):
            check_verify(torch, ee, draft, p, qq, u, ll, f"{b} {k} {v} {dtype} q {qq is not None} lengths {ll is not None}")


def test_verify_draft_strange_values(torch, ee):
    """Rows of zeros, NaN and infinities, residuals with nothing in them, drafts outside the vocabulary, random numbers at both ends, views."""
    g = torch.Generator(device="cuda").manual_seed(5)
    b, k, v = 12, 3, 5000
    p = torch.softmax(torch.randn(b, k + 1, v, device="cuda", generator=g), -1)
    q = torch.softmax(torch.randn(b, k, v, device="cuda", generator=g), -1)
    draft = torch.randint(0, v, (b, k), device="cuda", generator=g, dtype=torch.int32)
    u = torch.rand(b, k + 1, device="cuda", generator=g)
    p[0] = 0
    p[1] = float("nan")
    p[2, :, 100] = float("inf")
    p[3, :, 7] = float("nan")
    q[4] = p[4, :k]                      # refused only where u is 1: nothing is left, p is drawn from
    u[4, :k] = 1.0
    q[5] = float("nan")
    draft[6, 0], draft[7, 1], draft[8, 2] = -1, v, 2 ** 31 - 1
    u[9] = 0.0
    u[10] = 1.0
    p[11] = 0
    p[11, :, 4321] = 0.25                # one entry, behind the first chunk
    for qq in (q, None):
        check_verify(torch, ee, draft, p, qq, u, None, f"strange {qq is not None}")
        check_verify(torch, ee, draft, p, qq, torch.full_like(u, float("nan")), None, f"no numbers {qq is not None}")
    # views: rows of wider tensors, odd starts
    for kind in (torch.float32, torch.bfloat16):
        wide_p, wide_q = torch.rand(b, k + 3, v + 13, device="cuda", generator=g).to(kind), torch.rand(b, k + 3, v + 13, device="cuda", generator=g).to(kind)
        wide_u, wide_d = torch.rand(b, k + 5, device="cuda", generator=g), torch.randint(0, v, (b, k + 5), device="cuda", generator=g, dtype=torch.int32)
        check_verify(torch, ee, wide_d[:, 2:2 + k], wide_p[:, 1:k + 2, 3:3 + v], wide_q[:, 2:k + 2, 5:5 + v], wide_u[:, 1:k + 2], None, f"views {kind}")
        check_verify(torch, ee, wide_d[:, 2:2 + k], wide_p[:1, 1:2, 3:3 + v].expand(b, k + 1, v), None, wide_u[:, 1:k + 2], None, f"one row for all {kind}")


def test_verify_draft_gives_the_targets_distribution(torch, ee):
    """Whatever the draft, the first token that comes out has the target's probabilities: 400,000 sequences, each count within 6 standard deviations."""
    n, v = 400_000, 6
    g = torch.Generator(device="cuda").manual_seed(1)
    p1 = torch.tensor([0.4, 0.05, 0.25, 0.0, 0.2, 0.1], device="cuda")
    q1 = torch.tensor([0.1, 0.3, 0.25, 0.2, 0.15, 0.0], device="cuda")
    draft = torch.multinomial(q1, n, replacement=True, generator=g).int()[:, None]
    u = torch.rand(n, 2, device="cuda", generator=g)
    _, tokens = ee.verify_draft(draft, p1.expand(n, 2, v), u, draft_probs=q1.expand(n, 1, v))
    count = torch.bincount(tokens[:, 0].long(), minlength=v).double().cpu().numpy()
    p = p1.double().cpu().numpy()
    assert np.all(np.abs(count - n * p) <= 6 * np.sqrt(n * p * (1 - p)))


def test_verify_draft_refusals(torch, ee):
    p, q = torch.zeros(2, 4, 9, device="cuda"), torch.zeros(2, 3, 9, device="cuda")
    d, u = torch.zeros(2, 3, device="cuda", dtype=torch.int32), torch.zeros(2, 4, device="cuda")

    def refused(code, *a, **k):
        with pytest.raises(ee.EEError) as e:
            ee.verify_draft(*a, **k)
        assert e.value.code == code, e.value
    refused(ee.EE_ERR_UNSUPPORTED, d.long(), p, u)
    refused(ee.EE_ERR_UNSUPPORTED, d, p.half(), u)
    refused(ee.EE_ERR_UNSUPPORTED, d, p, u, draft_probs=q.bfloat16())
    refused(ee.EE_ERR_ARG, d, p[:, :3], u)
    refused(ee.EE_ERR_ARG, d, p, u[:, :3])
    refused(ee.EE_ERR_ARG, d, p, u, draft_probs=p)
    refused(ee.EE_ERR_ARG, d, p, u, lengths=torch.zeros(3, device="cuda", dtype=torch.int32))
    refused(ee.EE_ERR_ARG, d.cpu(), p, u)
    a, t = ee.verify_draft(d[:0], p[:0], u[:0])
    assert a.shape == (0,) and t.shape == (0, 4)


# ---- streams, graphs, all together --------------------------------------------------------------------------------------------------------
def chain(ee, s):
    """The end of a step: features normalised, an early and a last head with each request's adapter, the early exit's tokens verified by the last one."""
    f = ee.group_norm(s["x"], 8, s["gw"], s["gb"], act="silu")
    early, last = s["early"](f[:, :-1].contiguous(), s["ids"], dtype=s["torch"].float32), s["last"](f, s["ids"], dtype=s["torch"].float32)
    q, p = s["torch"].softmax(early, -1), s["torch"].softmax(last, -1)
    accepted, tokens = ee.verify_draft(s["draft"], p, s["u"], draft_probs=q, lengths=s["lengths"])
    return f, early, last, p, q, accepted, tokens


def chain_state(torch, ee, seed, b=9, k=4, c=128, v=700):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    s = dict(torch=torch, x=(2 * rnd(b, k + 1, c)).bfloat16(), gw=1 + 0.2 * rnd(c), gb=0.1 * rnd(c), ids=torch.randint(-1, 3, (b,), device="cuda", generator=g, dtype=torch.int32),
             draft=torch.randint(0, v, (b, k), device="cuda", generator=g, dtype=torch.int32), u=torch.rand(b, k + 1, device="cuda", generator=g) ** 4,
             lengths=torch.randint(0, k + 1, (b,), device="cuda", generator=g, dtype=torch.int32))
    w = (rnd(v, c) / c ** 0.5).bfloat16()
    for name, noise in (("early", 0.1), ("last", 0.0)):
        wn = (w.float() + noise * rnd(v, c) / c ** 0.5).bfloat16()
        s[name] = ee.AdapterProjection(wn, rnd(v), adapters=3, rank=8)
        s[name + "_w"], s[name + "_ad"] = wn, adapters_of(torch, g, 3, 8, c, v)
        for i, (a, bb, sc) in enumerate(s[name + "_ad"]):
            s[name].load(i, a, bb, sc)
    return s


def test_chain_of_the_three_and_compaction(torch, ee):
    """Norm, heads with adapters and verification as a step uses them, then the library's compaction takes out the sequences whose drafts were all accepted."""
    import workloads as W
    s = chain_state(torch, ee, 21)
    f, early, last, p, q, accepted, tokens = chain(ee, s)
    ref, tol = norm_ref(torch, s["x"], 8, s["gw"], s["gb"], 1e-5, "silu", None)
    assert bool(((f.double() - ref).abs() <= tol).all())
    want = verify_ref(s["draft"].cpu().numpy(), p.double().cpu().numpy(), q.double().cpu().numpy(), s["u"].cpu().numpy(), s["lengths"].cpu().numpy())
    assert np.array_equal(accepted.cpu().numpy(), want[0]) and np.array_equal(tokens.cpu().numpy(), want[1])
    blob = W.load_net("tiny_bf16")
    eng = ee.Engine(blob, 16)
    act = torch.randint(0, 100, (9,) + blob.stage_out_shape(0), device="cuda", dtype=torch.int16)
    flags = (accepted == s["lengths"]).to(torch.uint8)
    left, ids, b_rem, _ = eng.compact_refill(0, flags, act, s["ids"])
    keep = flags == 0
    assert b_rem == int(keep.sum()) and torch.equal(left, act[keep]) and torch.equal(ids, s["ids"][keep])
    eng.close()


def test_operators_on_another_stream_and_in_graphs(torch, ee):
    """Two graphs captured from the same handles, replayed in turn with eager work between, equal to eager results on new inputs every time; another stream than the default."""
    states = [chain_state(torch, ee, seed, b=b) for seed, b in ((1, 9), (2, 40))]
    big = [torch.randn(2, 96, 96, 64, device="cuda").bfloat16() for _ in states]                      # two launches and a workspace
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    with torch.cuda.stream(side):
        for s, x in zip(states, big):
            chain(ee, s)
            ee.group_norm(x, 32)
    torch.cuda.synchronize()
    for s, x in zip(states, big):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(chain(ee, s) + (ee.group_norm(x, 32),))
        graphs.append(graph)
    for turn in range(4):
        g = torch.Generator(device="cuda").manual_seed(100 + turn)
        for s, x in zip(states, big):
            s["x"].copy_(2 * torch.randn(s["x"].shape, device="cuda", generator=g))
            s["u"].copy_(torch.rand(s["u"].shape, device="cuda", generator=g))
            s["ids"].copy_(torch.randint(-1, 3, s["ids"].shape, device="cuda", generator=g))
            x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        for n in ((0, 1), (1, 0))[turn % 2]:
            graphs[n].replay()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            eager = [chain(ee, s) + (ee.group_norm(x, 32),) for s, x in zip(states, big)]
        torch.cuda.synchronize()
        for got, want in zip(outs, eager):
            for a, b in zip(got, want):
                assert torch.equal(a, b), f"turn {turn}"


@pytest.mark.parametrize("c,groups", [(32, 16), (64, 8), (6, 3), (10, 2)])
def test_group_norm_int8_products_between_whole_numbers(torch, ee, c, groups):
    """Two values a group, without eps: the deviation is a whole number over n, and factors of a quarter put products on halves, where a product that is not rounded before it is added, or a
    reciprocal in the place of a division, ends one lower."""
    cpg = c // groups
    for pixels in (1, 2, 4, 5, 12):
        n = pixels * cpg
        x = torch.zeros(20 * (n - 1), n, dtype=torch.int8, device="cuda")
        w = torch.tensor([0.25, 0.5, 0.75, 1.0, 1.5, 2.0, 2.5, 3.0], device="cuda").repeat((c + 7) // 8)[:c].contiguous()
        for ones in range(1, n):
            for i, v in enumerate((1, 2, 3, 5, 7)):
                for turn in range(4):
                    x[20 * (ones - 1) + 4 * i + turn, torch.arange(ones, device="cuda").add(turn * 3).remainder(n)] = v
        x = x.view(-1, pixels, 1, cpg).expand(-1, pixels, groups, cpg).reshape(-1, pixels, c).contiguous()
        for f in (0, 2, 5):
            say(f"[case] {c} channels {groups} groups {pixels} pixels frac_bits {f}")
            ref = norm_ref(torch, x.cpu(), groups, w.cpu(), None, 0.0, "none", None, f)[0].cuda()      # on the CPU, where a division by a number is one
            got = ee.group_norm(x, groups, w, None, eps=0.0, frac_bits=f)
            assert torch.equal(got, ref), f"{(got != ref).sum().item()} of {ref.numel()} differ"


@pytest.mark.parametrize("rows,ci,co", [(9, 72, 40), (40, 264, 1000), (200, 512, 200), (512, 1088, 512), (2048, 1088, 1000), (4096, 1088, 1000), (8192, 1088, 1000), (16384, 1088, 1024)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_adapter_projection_infinities_stay_with_their_rows(torch, ee, rows, ci, co, dtype):
    """An adapter with infinities and NaN in both halves beside others: rows of other adapters and of none are what the formula says, its own too.  A row of x with
    an infinity: the formula's infinities and NaN, in that row only."""
    g = torch.Generator(device="cuda").manual_seed(rows + co)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    say(f"[case] {rows} rows {ci} -> {co} {dtype}")
    w = (rnd(co, ci) / ci ** 0.5).bfloat16()
    proj = ee.AdapterProjection(w, None, adapters=4, rank=16)
    ranks = (16, 1, 5, 16)
    ab = [((rnd(r, ci) / ci ** 0.5).bfloat16(), (rnd(co, r) / r ** 0.5).bfloat16()) for r in ranks]
    a0, b0 = ab[0]
    b0[5, 2], b0[7, 0], b0[co - 1, 15] = float("inf"), float("nan"), -float("inf")
    ab[3][0][4, 3] = float("nan")                                          # a first half: its rows are NaN throughout
    for i, (a, b) in enumerate(ab):
        proj.load(i, a, b, 0.5)
    ids = torch.randint(-1, 3, (rows,), device="cuda", generator=g, dtype=torch.int32)
    ids[rows // 2] = 3
    ids[0], ids[rows - 1] = 0, 1
    x = rnd(rows, ci).bfloat16()
    out = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    bits = lambda t: t.view(torch.int16 if dtype == "bf16" else torch.int32)
    got = proj(x, ids, dtype=out)
    def near(rows_, cols, i):
        """rows_ of adapter i (-1: none) against 64 bits; the sums are as long as in the other tests"""
        xd, wd = x[rows_].double(), w.double()[cols].t()
        ref, size = xd @ wd, xd.abs() @ wd.abs()
        if i >= 0:
            a, b = ab[i][0].double().t(), ab[i][1].double()[cols].t()
            ref, size = ref + 0.5 * (xd @ a) @ b, size + 0.5 * (xd.abs() @ a.abs()) @ b.abs()
        return ((got[rows_][:, cols].double() - ref).abs() <= EPS[dtype] * ref.abs() + (ci + 64) * F32 * size).all()
    for i in (-1, 1, 2):
        assert near(ids == i, list(range(co)), i), i
    assert got[ids == 3].isnan().all()
    own = ids == 0
    sign = torch.sign(x[own].double() @ a0.double().t())
    assert torch.equal(got[own][:, 5].double(), sign[:, 2] * float("inf")) and got[own][:, 7].isnan().all() and torch.equal(got[own][:, co - 1].double(), -sign[:, 15] * float("inf"))
    assert near(own, [o for o in range(co) if o not in (5, 7, co - 1)], 0)
    # the infinity in x: rank 1, so that the formula's sum is not NaN everywhere
    x2 = x.clone()
    x2[rows - 1, 3] = float("inf")
    got2 = proj(x2, ids, dtype=out)
    assert torch.equal(bits(got2)[:rows - 1], bits(got)[:rows - 1])
    inf = float("inf")
    one = torch.sign(w[:, 3].double()) * inf + torch.sign(ab[1][0][0, 3].double()) * inf * torch.sign(ab[1][1][:, 0].double())
    assert torch.equal(got2[rows - 1].double().nan_to_num(nan=3.0, posinf=1.0, neginf=-1.0), one.nan_to_num(nan=3.0, posinf=1.0, neginf=-1.0))
    proj.load(0, *(t.nan_to_num(0, 0, 0) for t in ab[0]), 0.5)              # a sound adapter in its place, none in the other's
    proj.unload(3)
    assert proj(x, ids, dtype=out).isfinite().all()


@pytest.mark.parametrize("dtype,b,h,c,groups", [("bf16", 301, 56, 128, 32), ("int8", 601, 56, 128, 8), ("bf16", 5, 250, 400, 5), ("bf16", 70001, 1, 64, 4)])
def test_group_norm_large_batches_in_place(torch, ee, dtype, b, h, c, groups):
    """Batches that are worked through in parts, results that are written past the caches, y that is x or the residual, as many samples as no part of them divides."""
    g = torch.Generator(device="cuda").manual_seed(b)
    shape = (b, h, h, c)
    if dtype == "int8":
        x, res = (torch.randint(-128, 128, shape, device="cuda", generator=g, dtype=torch.int8) for _ in range(2))
    else:
        x, res = ((torch.randn(shape, device="cuda", generator=g) * 2 + 1).bfloat16() for _ in range(2))
    w, bias = torch.randn(c, device="cuda", generator=g), torch.randn(c, device="cuda", generator=g)
    kw = dict(act="relu", frac_bits=4, res_shift=0) if dtype == "int8" else dict(act="relu")
    say(f"[case] {dtype} {shape}")
    apart = ee.group_norm(x, groups, w, bias, residual=res, **kw)
    for first in range(0, b, max(1, b // 7)):
        part = slice(first, min(b, first + max(1, b // 7)))
        ref, bound = norm_ref(torch, x[part].reshape(-1, h * h, c), groups, w, bias, 1e-5, "relu", res[part].reshape(-1, h * h, c), 4 if dtype == "int8" else 0)
        got = apart[part].reshape(ref.shape)
        assert torch.equal(got, ref) if bound is None else bool(((got.double() - ref).abs() <= bound).all())
    for target in ("x", "res"):
        xx, rr = x.clone(), res.clone()
        out = xx if target == "x" else rr
        assert ee.group_norm(xx, groups, w, bias, residual=rr, out=out, **kw) is out
        assert torch.equal(out, apart), target
        assert torch.equal(rr if target == "x" else xx, res if target == "x" else x)


def test_verify_draft_many_sequences_share_their_rows(torch, ee):
    """As many sequences as chunks are no longer shared out, over one row of probabilities (stride 0)."""
    g = torch.Generator(device="cuda").manual_seed(5)
    b, v = 40000, 9001
    p = torch.softmax(torch.randn(1, 2, v, device="cuda", generator=g), -1).expand(b, 2, v)
    q = torch.softmax(torch.randn(1, 1, v, device="cuda", generator=g), -1).expand(b, 1, v)
    draft = torch.randint(0, v, (b, 1), device="cuda", generator=g, dtype=torch.int32)
    u = torch.rand(b, 2, device="cuda", generator=g)
    accepted, tokens = ee.verify_draft(draft, p, u, draft_probs=q)
    pd, qd = p[0].double(), q[0, 0].double()
    x = draft[:, 0].long()
    ok = u[:, 0].double() * qd[x] < pd[0][x]
    assert torch.equal(accepted.long(), ok.long()) and 0 < ok.sum() < b
    for rows, w, first in ((~ok, (pd[0] - qd).clamp(min=0), 0), (ok, pd[1], 1)):
        cum = w.cpu().cumsum(0)
        target = u[rows, 1].double().cpu() * cum[-1]
        want = torch.searchsorted(cum, target, right=True).clamp(max=v - 1)
        got = tokens[rows, first].long().cpu()
        near = (cum[got] - target).abs().minimum((cum[got] - w.cpu()[got] - target).abs()) <= v * 2.0 ** -53 * cum[-1]      # sums in another order
        assert bool(((got == want) | near).all()) and bool((w.cpu()[got] > 0).all())
    assert torch.equal(tokens[ok, 0], draft[ok, 0]) and bool((tokens[~ok, 1] == -1).all())


def test_results_must_not_share_elements(torch, ee):
    x = torch.ones(4, 3, 8, device="cuda").bfloat16()
    wide = torch.zeros(4, 3, 8, device="cuda").bfloat16()
    for out in (wide[:1].expand(4, 3, 8), wide.view(-1).as_strided((4, 3, 8), (8, 8, 1)), wide.view(-1).as_strided((4, 3, 8), (4, 32, 1)), wide.view(-1).as_strided((4, 3, 8), (8, 31, 1))):
        with pytest.raises(ee.EEError):
            ee.group_norm(x, 2, out=out)
    turns = torch.zeros(3, 4, 8, device="cuda").bfloat16().transpose(0, 1)            # the pixels of the samples take turns
    assert torch.equal(ee.group_norm(x, 2, out=turns), ee.group_norm(x, 2))
    proj = ee.AdapterProjection(torch.ones(16, 8, device="cuda").bfloat16())
    for out in (torch.zeros(16, device="cuda").bfloat16().expand(12, 16), torch.zeros(12 * 16, device="cuda").bfloat16().as_strided((12, 16), (8, 1))):
        with pytest.raises(ee.EEError):
            proj(x.view(12, 8), out=out)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("b,v", [(12, 999), (40, 20001), (70, 35003), (13, 24576), (13, 24577), (12, 60001), (256, 5001), (257, 5000)])
def test_verify_draft_strange_values_in_every_form(torch, ee, b, v, dtype):
    """Rows of zeros, NaN and infinities, residuals with nothing in them, single entries at every place of a piece, drafts at the ends, numbers at both ends: on both sides of where one workgroup
    takes a row and where it is cut up."""
    kind = torch.float32 if dtype == "fp32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(b + v)
    k = 2
    p = torch.softmax(2 * torch.randn(b, k + 1, v, device="cuda", generator=g), -1).to(kind)
    q = torch.softmax(2 * torch.randn(b, k, v, device="cuda", generator=g), -1).to(kind)
    draft = torch.randint(0, v, (b, k), device="cuda", generator=g, dtype=torch.int32)
    u = torch.rand(b, k + 1, device="cuda", generator=g)
    p[0] = 0
    p[1] = float("nan")
    p[2, :, v // 2], p[2, :, v - 1] = float("inf"), float("inf")
    p[3, :, 7], q[3, :, 9] = float("nan"), -float("inf")
    q[4] = p[4, :k]                      # nothing is left
    u[4, :k] = 1.0
    q[5] = float("inf")
    draft[6, 0], draft[7, 0] = -1, v
    u[8, k], u[9, k] = 0.0, 1.0
    p[10] = 0
    p[10, :, v - 1] = 0.25
    draft[11, 0], u[11, 0] = v - 1, 1.0
    for i in range(12, min(b, 40)):      # a single entry
        at = [0, 7, 8, 511, 512, 513, 8191, v - 9, v - 8][i % 9] % v
        p[i] = 0
        p[i, :, at] = 0.5
    lengths = torch.randint(-1, k + 1, (b,), device="cuda", generator=g, dtype=torch.int32)
    for qq in (q, None):
        check_verify(torch, ee, draft, p, qq, u, None, f"{b} x {v} {dtype} strange {qq is not None}")
        check_verify(torch, ee, draft, p, qq, u, lengths, f"{b} x {v} {dtype} strange, lengths {qq is not None}")


def test_group_norm_widest_groups(torch, ee):
    g = torch.Generator(device="cuda").manual_seed(8)
    for dtype, c in ((torch.int8, 8192), (torch.bfloat16, 8192), (torch.int8, 4096), (torch.int8, 1023), (torch.bfloat16, 1023)):
        for pixels in (1, 3, 40):
            say(f"[case] {dtype} {pixels} x {c}")
            x = torch.randint(-128, 128, (2, pixels, c), device="cuda", generator=g, dtype=torch.int8).to(dtype)
            w, b = torch.randn(c, device="cuda", generator=g), torch.randn(c, device="cuda", generator=g)
            f = 5 if dtype == torch.int8 else 0
            ref, bound = norm_ref(torch, x, 1, w, b, 1e-5, "none", None, f)
            got = ee.group_norm(x, 1, w, b, frac_bits=f)
            assert torch.equal(got, ref) if bound is None else bool(((got.double() - ref).abs() <= bound).all())
    for dtype, c in ((torch.int8, 8208), (torch.bfloat16, 8200), (torch.int8, 1025), (torch.bfloat16, 1025)):
        with pytest.raises(ee.EEError) as e:
            ee.group_norm(torch.zeros(1, 2, c, device="cuda", dtype=dtype), 1)
        assert e.value.code == ee.EE_ERR_UNSUPPORTED


def test_group_norm_int8_values_near_whole_numbers_everywhere(torch, ee):
    """One factor for all channels and few different values: a value near a whole number is one in all of a group."""
    g = torch.Generator(device="cuda").manual_seed(9)
    for pixels, c, groups in ((2000, 128, 8), (49, 512, 32), (9, 48, 16), (700, 64, 2)):
        x = torch.randint(-2, 3, (6, pixels, c), device="cuda", generator=g, dtype=torch.int8)
        res = torch.randint(-128, 128, x.shape, device="cuda", generator=g, dtype=torch.int8)
        for scale, f, rs in ((1.0, 0, 0), (0.5, 4, -1), (3.0, 7, -8), (2.0 ** -20, 0, 0)):
            w, b = torch.full((c,), scale, device="cuda"), torch.full((c,), 2 * scale, device="cuda")
            for r in (None, res):
                say(f"[case] {pixels} {c} {groups} scale {scale} f {f} rs {rs} residual {r is not None}")
                ref, _ = norm_ref(torch, x, groups, w, b, 1e-5, "none", r, f, rs)
                assert torch.equal(ee.group_norm(x, groups, w, b, frac_bits=f, residual=r, res_shift=rs), ref)


@pytest.mark.parametrize("rows,ci,co", [(9, 72, 40), (200, 2080, 1000), (512, 1096, 512), (2048, 1096, 1000), (4096, 1096, 1000), (8192, 1096, 1000), (16384, 1064, 1024)])
def test_adapter_projection_infinite_weights(torch, ee, rows, ci, co):
    """Infinities in the shared weight, at its first, last and a middle column: the formula's infinities in those outputs, the others as they were.  Reductions of an odd number of slabs."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    say(f"[case] {rows} rows {ci} -> {co}")
    w = (rnd(co, ci) / ci ** 0.5).bfloat16()
    a, b = (rnd(16, ci) / ci ** 0.5).bfloat16(), (rnd(co, 16) / 4).bfloat16()
    odd = w.clone()
    odd[3, 0], odd[5, ci - 1], odd[co - 1, ci // 2] = float("inf"), -float("inf"), float("inf")
    x = rnd(rows, ci).bfloat16()
    ids = torch.randint(-1, 2, (rows,), device="cuda", generator=g, dtype=torch.int32)
    out = []
    for weight in (w, odd):
        proj = ee.AdapterProjection(weight, None, adapters=2, rank=16)
        proj.load(0, a, b)
        proj.load(1, b[:ci, :].t().contiguous() if co == ci else a, b, 0.25)
        out.append(proj(x, ids, dtype=torch.float32))
    keep = [o for o in range(co) if o not in (3, 5, co - 1)]
    assert torch.equal(out[0][:, keep], out[1][:, keep]) and out[0].isfinite().all()
    inf = float("inf")
    for o, c, sign in ((3, 0, 1.0), (5, ci - 1, -1.0), (co - 1, ci // 2, 1.0)):
        assert torch.equal(out[1][:, o], sign * inf * torch.sign(x[:, c].float()))


@pytest.mark.parametrize("rows,ci,co", [(9, 72, 40), (12, 4096, 64), (300, 520, 200), (1500, 1096, 72)])
def test_adapter_projection_infinite_first_halves(torch, ee, rows, ci, co):
    """An infinity in an adapter's first half, at its first, last and a middle column: the formula's infinities in its rows."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    w = (rnd(co, ci) / ci ** 0.5).bfloat16()
    x = rnd(rows, ci).bfloat16()
    ids = (torch.arange(rows, device="cuda") % 3).int() - 1
    b = rnd(co, 2).bfloat16()
    for col in (0, ci // 2, ci - 1):
        say(f"[case] {rows} rows {ci} -> {co} column {col}")
        a = (rnd(2, ci) / ci ** 0.5).bfloat16()
        a[0, col] = float("inf")
        proj = ee.AdapterProjection(w, None, adapters=2, rank=16)
        proj.load(0, a, b)
        for dtype in (torch.float32, torch.bfloat16):
            y = proj(x, ids, dtype=dtype)
            own = ids == 0
            want = torch.sign(x[own][:, col].float())[:, None] * torch.sign(b[:, 0].float())[None, :] * float("inf")
            assert torch.equal(y[own].float(), want) and y[~own].isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("slots,per,ci,co,r", [(40, 127, 1096, 250, 32), (33, 128, 520, 256, 16), (9, 333, 2088, 136, 20), (64, 196, 1024, 256, 32), (7, 1001, 264, 72, 1), (30, 150, 1024, 130, 17),
                                              (3, 5000, 40, 129, 8), (24, 255, 1032, 1000, 32)])
def test_adapter_projection_long_slots(torch, ee, slots, per, ci, co, r, dtype):
    """Slots of many rows each, tiles with the end of one and the start of the next, slots without an adapter, adapters of lower rank and with infinities beside sound ones."""
    g = torch.Generator(device="cuda").manual_seed(slots * per)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    say(f"[case] {slots} x {per} {ci} -> {co} rank {r} {dtype}")
    w, bias = (rnd(co, ci) / ci ** 0.5).bfloat16(), rnd(co)
    n = 5
    proj = ee.AdapterProjection(w, bias, adapters=n, rank=r)
    ranks = [r, max(1, r // 2), r, 1, r]
    ab = [((rnd(k, ci) / ci ** 0.5).bfloat16(), (rnd(co, k) / k ** 0.5).bfloat16()) for k in ranks]
    ab[4][1][co // 2, 0] = float("inf")
    for i, (a, b) in enumerate(ab):
        proj.load(i, a, b, 0.5 + i)
    ids = torch.randint(-1, n, (slots,), device="cuda", generator=g, dtype=torch.int32)
    ids[0], ids[1] = 4, 2
    x = rnd(slots, per, ci).bfloat16()
    out = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    y = proj(x, ids, dtype=out)
    assert torch.equal(y, proj(x, ids, dtype=out)) or ids.eq(4).any()
    xd, wd = x.double(), w.double().t()
    ref, size = xd @ wd + bias.double(), xd.abs() @ wd.abs() + bias.double().abs()
    for s in range(slots):
        i = int(ids[s])
        if i >= 0:
            a, b = ab[i][0].double().t(), ab[i][1].double().t()
            ref[s] += (0.5 + i) * (xd[s] @ a) @ b
            size[s] += (0.5 + i) * (xd[s].abs() @ a.abs()) @ b.abs()
    wild = torch.zeros(slots, 1, co, dtype=torch.bool, device="cuda")
    wild[ids == 4, :, co // 2] = True
    wild = wild.expand(slots, per, co)
    assert torch.equal(y[wild].double(), ref[wild])
    # the sum of a first half's parts is off by 2^-18 (2^-24) of it
    part = {"bf16": 2.0 ** -18, "fp32": 2.0 ** -24}[dtype]
    bad = ((y.double() - ref).abs() > EPS[dtype] * ref.abs() + ((ci + 2 * r + 8) * F32 + part) * size) & ~wild
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}"


def test_adapter_projection_single_rows_and_columns(torch, ee):
    """Dimensions of one element have any stride."""
    g = torch.Generator(device="cuda").manual_seed(12)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g).bfloat16()
    for ci, co, r in ((24, 40, 1), (1, 5, 1), (9, 1, 3), (1, 1, 1)):
        say(f"[case] {ci} -> {co} rank {r}")
        w, a, b, x = rnd(co, ci), rnd(r, ci), rnd(co, r), rnd(3, ci)
        odd = lambda t: t.as_strided(t.shape, tuple(7 if n == 1 else s for n, s in zip(t.shape, t.stride())))
        proj = ee.AdapterProjection(odd(w), None, adapters=1, rank=4)
        proj.load(0, odd(a), odd(b), 2.0)
        ids = torch.tensor([0, -1, 0], device="cuda", dtype=torch.int32)
        y = proj(x, ids, dtype=torch.float32).double()
        ref = x.double() @ w.double().t()
        ref[[0, 2]] += 2.0 * ((x.double() @ a.double().t()) @ b.double().t())[[0, 2]]
        size = x.double().abs() @ w.double().t().abs() + 2.0 * (x.double().abs() @ a.double().t().abs()) @ b.double().t().abs()
        assert bool(((y - ref).abs() <= (ci + r + 8) * F32 * size + 1e-30).all())


def test_expanded_pixels(torch, ee):
    """A dimension repeated by a stride of zero is not one stride apart from the next; all of them repeated are."""
    x = torch.randn(2, 3, 1, 16, device="cuda").bfloat16()
    y = torch.randn(2, 3, 1, 5, 16, device="cuda").bfloat16()
    for bad in (x.expand(2, 3, 4, 16), y.expand(2, 3, 4, 5, 16)):
        with pytest.raises(ee.EEError) as e:
            ee.group_norm(bad, 2)
        assert e.value.code == ee.EE_ERR_ARG
    proj = ee.AdapterProjection(torch.ones(8, 16, device="cuda").bfloat16())
    with pytest.raises(ee.EEError):
        proj(x.expand(2, 3, 4, 16))
    one = x[:, :1]
    whole = one.expand(2, 3, 4, 16)
    assert torch.equal(ee.group_norm(whole, 2), ee.group_norm(whole.contiguous(), 2))
    res = x.expand(2, 3, 4, 16).contiguous()
    assert torch.equal(ee.group_norm(res, 2, residual=whole), ee.group_norm(res, 2, residual=whole.contiguous()))
    samples = x[:1].expand(5, 3, 1, 16)
    assert torch.equal(ee.group_norm(samples, 2), ee.group_norm(samples.contiguous(), 2))


@pytest.mark.parametrize("h,w,c,groups", [(1, 1, 40, 5), (1, 3, 40, 5), (7, 7, 40, 5), (13, 11, 48, 48), (35, 35, 33, 3), (9, 11, 96, 12), (100, 100, 40, 20), (300, 301, 40, 5), (300, 301, 24, 24), (211, 199, 33, 3)])
def test_group_norm_of_constant_groups_is_the_bias(torch, ee, h, w, c, groups):
    """Every partial mean of a constant group is the constant and every partial variance 0, whatever the number of values and their size: the result is the bias, not a rounding of it."""
    bias = torch.linspace(-1, 1, c, device="cuda")
    say(f"[case] {h}x{w}x{c} groups {groups}")
    for value in (3.0, -57.25, 1003.0, 65537.0, 1e6, -1.5e10, 1e20, 3e38, 1e-30):
        x = torch.full((2, h, w, c), value, device="cuda").to(torch.bfloat16)
        for act in ("none", "relu"):
            want = (bias if act == "none" else bias.clamp(min=0)).to(torch.bfloat16).expand_as(x)
            got = ee.group_norm(x, groups, None, bias, act=act)
            assert torch.equal(got, want), f"{value}: off by {float((got.double() - want.double()).abs().max())}"


@pytest.mark.parametrize("h,w,c", [(64, 64, 64), (300, 301, 40), (512, 512, 256), (512, 512, 512), (1024, 1024, 256), (2048, 2048, 64), (700, 701, 33)])
@pytest.mark.parametrize("cpg", [8, 2, 1])
def test_group_norm_of_a_constant_and_one_pixel_apart(torch, ee, h, w, c, cpg):
    """One pixel is 0, all others one value v: the variance is that pixel's alone, v^2 (n - 1) / n^2 with n pixels, wherever it lies.  Bound of the result: half a step of bf16, and half of what the
    variance may be off by: 64 values are added from a pivot that is v off at most, 63 additions of up to 64 v^2 each within 2^-24, 2^-12 of v^2; twice that for the mean's part and the merges."""
    groups = c // cpg if c % cpg == 0 else c // 3
    n = h * w
    say(f"[case] {h}x{w}x{c} groups {groups}")
    for value in (57.25, 100.5, 3.3125):
        for at in (0, 1, n // 2, n - 1):
            x = torch.full((1, n, c), value, device="cuda", dtype=torch.bfloat16)
            x[0, at] = 0
            y = ee.group_norm(x.view(1, h, w, c), groups, eps=0.0).view(n, c)
            a = n / (value * (n - 1) ** 0.5)
            apart, others = (1 / n - 1) * value * a, value / n * a
            mean = 128 * F32 * 2 * value * a
            assert float((y[at].double() - apart).abs().max()) <= (2.0 ** -8 + 2.0 ** -11) * abs(apart) + mean, (value, at, float(y[at, 0]), apart)
            y[at] = others
            assert float((y.float() - others).abs().max()) <= (2.0 ** -8 + 2.0 ** -11) * others + mean, (value, at)


def test_group_norm_of_large_maps_against_64_bits(torch, ee):
    """Long lanes over values that drift from the first pixel to the last and are far from zero: every part's mean is another one."""
    g = torch.Generator(device="cuda").manual_seed(3)
    for h, w, c, groups, level, drift in ((512, 512, 256, 32, 0.0, 0.0), (700, 511, 64, 32, 200.0, 50.0), (1024, 1024, 64, 8, -1000.0, 300.0), (513, 512, 33, 3, 5.0, 40.0)):
        say(f"[case] {h}x{w}x{c} groups {groups} level {level} drift {drift}")
        x = (torch.randn(1, h * w, c, device="cuda", generator=g) * 4 + level + drift * torch.linspace(0, 1, h * w, device="cuda").view(1, -1, 1)).bfloat16()
        x[0, 0] = 0
        ref, tol = norm_ref(torch, x, groups, None, None, 1e-5, "none", None)
        got = ee.group_norm(x.view(1, h, w, c), groups).view(x.shape)
        off = (got.double() - ref).abs() - tol
        assert float(off.max()) <= 0, f"off by {float(off.max())} more than the bound"


@pytest.mark.parametrize("dtype", ["bf16", "int8"])
def test_group_norm_more_samples_than_a_launch_has_workgroups(torch, ee, dtype):
    """2^24 workgroups of 256 threads are as many threads as a launch may not have."""
    b, c, groups = (1 << 24) + 5, 16, 4
    g = torch.Generator(device="cuda").manual_seed(24)
    x = torch.randint(-100, 100, (b, c), device="cuda", generator=g, dtype=torch.int8)
    x = x if dtype == "int8" else x.bfloat16()
    say(f"[case] {b} samples {dtype}")
    got = ee.group_norm(x, groups, frac_bits=4)
    for first in list(range(0, b, 1 << 21)) + [b - 9]:
        part = slice(first, first + (1 << 21))
        ref, bound = norm_ref(torch, x[part, None], groups, None, None, 1e-5, "none", None, 4)
        assert torch.equal(got[part, None], ref) if bound is None else bool(((got[part, None].double() - ref).abs() <= bound).all()), first


def test_adapter_projection_copies_more_elements_than_a_launch_has_threads(torch, ee):
    """Rows that are no whole 16-byte pieces, more than 2^32 elements with their padding: all of them are copied and projected."""
    rows, ci, co = (1 << 21) + 77, 2047, 8
    g = torch.Generator(device="cuda").manual_seed(32)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    x = torch.empty(rows, ci, device="cuda", dtype=torch.bfloat16)
    for first in range(0, rows, 1 << 18):
        x[first:first + (1 << 18)] = rnd(min(1 << 18, rows - first), ci)
    w, ad = (rnd(co, ci) / ci ** 0.5).bfloat16(), adapters_of(torch, g, 1, 4, ci, co)
    proj = ee.AdapterProjection(w, None, adapters=1, rank=4)
    proj.load(0, *ad[0])
    ids = (torch.arange(rows, device="cuda", dtype=torch.int32) % 2) - 1
    say(f"[case] {rows} x {ci} -> {co}")
    got = proj(x, ids, dtype=torch.float32)
    for first in (0, (1 << 20) - 9, rows - (1 << 14)):
        part = slice(first, first + (1 << 14))
        ref, tol = project_ref(torch, x[part], w, None, ad, ids[part], "fp32")
        assert bool(((got[part].double() - ref).abs() <= tol).all()), first


def test_adapter_projection_next_to_its_input(torch, ee):
    """Results in front of, behind and beside the rows they are of, in one tensor; over them they are refused."""
    g = torch.Generator(device="cuda").manual_seed(41)
    ci = co = 64
    proj = ee.AdapterProjection((torch.randn(co, ci, device="cuda", generator=g) / 8).bfloat16())
    x = torch.randn(700, ci, device="cuda", generator=g).bfloat16()
    for rows in (1, 12, 700):
        for dtype in (torch.bfloat16, torch.float32):
            want = proj(x[:rows], dtype=dtype)
            wide = torch.zeros(2 * rows, 3 * ci, device="cuda", dtype=torch.bfloat16)
            n = 1 if dtype == torch.bfloat16 else 2
            results = lambda t: t if n == 1 else t.view(dtype)
            for src, dst in ((wide[:rows, :ci], wide[:rows, ci:ci + n * co]), (wide[:rows, 2 * ci:], wide[:rows, :n * co]), (wide[:rows, :ci], wide[rows:, :n * co]), (wide[rows:, ci:2 * ci], wide[:rows, ci:ci + n * co])):
                src.copy_(x[:rows])
                say(f"[case] {rows} rows {dtype}")
                assert torch.equal(proj(src, out=results(dst), dtype=dtype), want)
                assert torch.equal(src, x[:rows])
            src = wide[:rows, :ci]
            for dst in (wide[:rows, :n * co], wide[:rows, ci // 2:ci // 2 + n * co]):
                with pytest.raises(ee.EEError) as e:
                    proj(src, out=results(dst), dtype=dtype)
                assert e.value.code == ee.EE_ERR_ARG


def test_group_norm_next_to_its_input(torch, ee):
    """Results beside, between, in front of and behind what they are of, in one tensor, or over it; over a part of it they are refused."""
    g = torch.Generator(device="cuda").manual_seed(42)
    for b, p, c in ((1, 1, 32), (3, 1, 32), (1, 20, 32), (3, 20, 32), (2, 5000, 32), (2, 20, 33)):
        x0, r0 = ((torch.randn(b, p, c, device="cuda", generator=g) * 3).bfloat16() for _ in range(2))
        groups = c // 8 if c % 8 == 0 else 3
        plain, with_res = ee.group_norm(x0, groups, act="relu"), ee.group_norm(x0, groups, act="relu", residual=r0)
        new = lambda *s: torch.zeros(s, device="cuda", dtype=torch.bfloat16)
        wide, samples, turns, line = new(b, p, 3 * c), new(3 * b, p, c), new(p, 3 * b, c), new(3, b, p, c)
        for views in ([wide[..., i * c:(i + 1) * c] for i in range(3)], [samples[i::3] for i in range(3)], [samples[i * b:(i + 1) * b] for i in range(3)], [turns[:, i * b:(i + 1) * b].transpose(0, 1) for i in range(3)],
                      [turns[:, i::3].transpose(0, 1) for i in range(3)] if b == 1 else [line[i] for i in range(3)]):
            for i, j, k in ((0, 1, 2), (2, 0, 1), (1, 2, 0)):
                x, out, res = views[i], views[j], views[k]
                x.copy_(x0)
                res.copy_(r0)
                say(f"[case] {b} x {p} x {c}")
                near = lambda a, w: bool(((a.double() - w.double()).abs() <= 2.0 ** -6 * w.double().abs() + 2.0 ** -14).all())      # alignment chooses the order of sums
                assert near(ee.group_norm(x, groups, act="relu", out=out), plain) and near(ee.group_norm(x, groups, act="relu", residual=res, out=out), with_res)
                assert torch.equal(x, x0) and torch.equal(res, r0)
                assert near(ee.group_norm(x, groups, act="relu", residual=res, out=res), with_res) and torch.equal(x, x0)
                assert near(ee.group_norm(x, groups, act="relu", out=x), plain)
        flat = new(b * p * c + c)
        for at in (1, 8, c):
            with pytest.raises(ee.EEError) as e:
                ee.group_norm(flat[:b * p * c].view(b, p, c), groups, out=flat[at:at + b * p * c].view(b, p, c)) if b * p * c > at else ee.group_norm(flat[:c].view(1, 1, c), groups, out=flat[1:1 + c].view(1, 1, c))
            assert e.value.code == ee.EE_ERR_ARG


@pytest.mark.parametrize("slots,per,ci,co,r,n", [(40, 127, 1096, 250, 32, 5), (64, 196, 1024, 256, 32, 16), (3, 5000, 40, 129, 8, 5), (24, 255, 1032, 1000, 32, 5), (12, 1, 4096, 4096, 16, 8), (64, 1, 2048, 1000, 16, 24),
                                                 (300, 1, 2048, 512, 16, 24), (200, 7, 1096, 1000, 64, 9), (24, 333, 4096, 4096, 64, 16)])
def test_adapter_projection_repeats_its_bits(torch, ee, slots, per, ci, co, r, n):
    """The same call gives the same bits, of infinities and NaN too, with other work in the caches between the calls."""
    g = torch.Generator(device="cuda").manual_seed(slots + co)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    say(f"[case] {slots} x {per} {ci} -> {co} rank {r}")
    proj = ee.AdapterProjection((rnd(co, ci) / ci ** 0.5).bfloat16(), rnd(co), adapters=n, rank=r)
    for i, (a, b, s) in enumerate(adapters_of(torch, g, n, r, ci, co)):
        if i == n - 1:
            b[co // 2, 0] = float("inf")
        proj.load(i, a, b, s)
    ids = torch.randint(-1, n, (slots,), device="cuda", generator=g, dtype=torch.int32)
    ids[0] = n - 1
    x = rnd(slots, per, ci).bfloat16()
    for dtype, bits in ((torch.bfloat16, torch.int16), (torch.float32, torch.int32)):
        first = proj(x, ids, dtype=dtype)
        for turn in range(6):
            other = torch.full((1 << (18 + turn),), float(turn), device="cuda")
            assert torch.equal(proj(x, ids, dtype=dtype).view(bits), first.view(bits)), turn
            assert bool((other == turn).all())


@pytest.mark.parametrize("b,p,c,groups", [(1, 49, 512, 32), (64, 3136, 256, 32), (37, 1225, 96, 12), (2, 40000, 64, 32), (9, 400, 33, 3)])
def test_group_norm_repeats_its_bits(torch, ee, b, p, c, groups):
    g = torch.Generator(device="cuda").manual_seed(p)
    x = (torch.randn(b, p, c, device="cuda", generator=g) * 3 + 1).bfloat16()
    x[0, 0, 0] = float("nan")
    say(f"[case] {b} x {p} x {c}")
    first = ee.group_norm(x, groups, act="silu", residual=x)
    for turn in range(6):
        other = torch.full((1 << (18 + turn),), float(turn), device="cuda")
        assert torch.equal(ee.group_norm(x, groups, act="silu", residual=x).view(torch.int16), first.view(torch.int16)), turn
        assert bool((other == turn).all())


@pytest.mark.parametrize("h,w,c,groups", [(1, 1, 32, 4), (1, 2, 32, 4), (2, 2, 32, 32), (7, 7, 64, 8), (20, 20, 33, 3), (35, 35, 96, 12), (100, 101, 64, 32)])
def test_group_norm_of_lowest_values(torch, ee, h, w, c, groups):
    """A value whose deviation has no square in float, as masks have them: its group is NaN wherever it lies, never a bias that looks sound; the other groups are as they were."""
    g = torch.Generator(device="cuda").manual_seed(h * c)
    x = torch.randn(2, h, w, c, device="cuda", generator=g).bfloat16()
    cpg = c // groups
    bias = torch.ones(c, device="cuda")
    clean = ee.group_norm(x, groups, None, bias)
    for value in (torch.finfo(torch.bfloat16).min, torch.finfo(torch.bfloat16).max, float("inf"), -float("inf"), float("nan")):
        for pixel in sorted({0, 1, h * w // 2, h * w - 1} & set(range(h * w))):
            say(f"[case] {h}x{w}x{c} groups {groups} {value} at {pixel}")
            bad = x.clone()
            bad.view(2, h * w, c)[1, pixel, 2 * cpg] = value
            got = ee.group_norm(bad, groups, None, bias)
            mine = torch.zeros(2, h, w, c, dtype=torch.bool, device="cuda")
            mine[1, :, :, 2 * cpg:3 * cpg] = True
            if h * w * cpg > 1 or value != value or abs(value) == float("inf"):
                assert bool(got[mine].isnan().all()), float(got[mine].float().abs().max())
            assert torch.equal(got[~mine], clean[~mine])


@pytest.mark.parametrize("dtype", ["bf16", "int8"])
@pytest.mark.parametrize("pixels", [300, 700, 1023, 1025, 1800, 2047, 2049, 2500, 4095, 4097])
def test_group_norm_on_both_sides_of_every_form(torch, ee, dtype, pixels):
    """Numbers of pixels around where 256, 512 and 1,024 threads hold a sample, groups of one channel, of three, of a column's sixteenth, fourth and whole, with few and with many samples."""
    g = torch.Generator(device="cuda").manual_seed(pixels)
    for c, groups in ((16, 16), (32, 32), (48, 16), (48, 48), (64, 16), (64, 8), (80, 8), (96, 3), (112, 7), (33, 11), (272, 16)):
        for b in (1, 3, 90):
            x = torch.randint(-100, 101, (b, pixels, c), device="cuda", generator=g, dtype=torch.int8)
            x = x if dtype == "int8" else (x.float() / 7).bfloat16()
            say(f"[case] {dtype} {b} x {pixels} x {c} groups {groups}")
            ref, bound = norm_ref(torch, x, groups, None, None, 1e-5, "none", None, 5)
            got = ee.group_norm(x, groups, frac_bits=5)
            assert torch.equal(got, ref) if bound is None else bool(((got.double() - ref).abs() <= bound).all())


@pytest.mark.parametrize("rows,ci,co,r", [(12, 1, 16, 256), (64, 1, 76, 256), (400, 1, 65, 100), (1302, 1, 76, 256), (5000, 1, 9, 128), (33, 8, 100, 256)])
def test_adapter_projection_small_adapters_beside_large_outputs(torch, ee, rows, ci, co, r):
    """Many small terms of an adapter beside a bias a thousand times as large, whose float they are added to once: the bound has ci + 8 roundings of the large one, and those of the small ones among themselves."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    w, bias, ad = (rnd(co, ci) / ci ** 0.5).bfloat16(), 1000 * (1 + rnd(co).abs()), adapters_of(torch, g, 3, r, ci, co)
    proj = ee.AdapterProjection(w, bias, adapters=3, rank=r)
    for i, (a, b, s) in enumerate(ad):
        proj.load(i, a, b, s)
    for turn in range(8):
        x = rnd(rows, ci).bfloat16()
        ids = torch.randint(-1, 3, (rows,), device="cuda", generator=g, dtype=torch.int32)
        say(f"[case] {rows} rows {ci} -> {co} rank {r}")
        got = proj(x, ids, dtype=torch.float32)
        ref, tol = project_ref(torch, x, w, bias, ad, ids, "fp32")
        off = ((got.double() - ref).abs() / tol).cpu()
        assert float(off.max()) <= 1, f"{float(off.max())} times the bound"
