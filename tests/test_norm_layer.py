"""Group norm as a layer of a network: the oracle's against its definition, what the two readers of a network refuse, and the library's segments and stream against the oracle.

int8: equal.  bf16, a layer alone: one rounding to bf16 (half a step, 2^-8 relative) on each side's own value, and what float sums lose in front of it (128 steps of 2^-24 of the values'
size); whole segments: 2e-2 of a sample's largest value, as for other bf16 networks."""
import sys

import numpy as np
import pytest

import workloads as W
from workloads.blob import bf16_bits_to_f32, f32_to_bf16_bits

ACTS = ("none", "relu", "relu6", "silu")


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def plain_i8(x, groups, weight, bias, eps, act, frac_bits, res, res_shift):
    n, c = x.shape[0], x.shape[-1]
    xi = x.reshape(n, -1, groups, c // groups).astype(np.int64)
    cnt = xi.shape[1] * xi.shape[3]
    s1, s2 = xi.sum((1, 3), keepdims=True), (xi * xi).sum((1, 3), keepdims=True)
    m = weight.astype(np.float64).reshape(groups, -1) * 2.0 ** frac_bits / (cnt * np.sqrt((cnt * s2 - s1 * s1) / float(cnt) ** 2 + np.float64(np.float32(eps))))
    t = (cnt * xi - s1) * m + (bias.astype(np.float64).reshape(groups, -1) * 2.0 ** frac_bits + 0.5)
    t = t.reshape(x.shape)
    if res is not None:
        t = t + res * 2.0 ** res_shift
    return np.clip(np.floor(t), 0 if act else -128, min(127, 6 * 2 ** frac_bits) if act == 2 else 127).astype(np.int8)


def plain_f64(x, groups, weight, bias, eps, act, res):
    """(values, their size)"""
    n, c = x.shape[0], x.shape[-1]
    xd = x.astype(np.float64).reshape(n, -1, groups, c // groups)
    d = xd - xd.mean((1, 3), keepdims=True)
    a = weight.astype(np.float64).reshape(groups, -1) / np.sqrt((d * d).mean((1, 3), keepdims=True) + np.float64(np.float32(eps)))
    t = (d * a + bias.astype(np.float64).reshape(groups, -1)).reshape(x.shape)
    size = ((np.abs(d) + np.abs(xd).max((1, 3), keepdims=True)) * np.abs(a)).reshape(x.shape) + np.abs(np.tile(bias, x.size // c).reshape(x.shape))
    if res is not None:
        t, size = t + res, size + np.abs(res)
    t = [t, np.maximum(t, 0), np.clip(t, 0, 6), t / (1 + np.exp(-t))][act]
    return t, size


def inputs(shape, groups, i8, seed=0):
    r = np.random.default_rng(seed)
    c = shape[-1]
    w, b = (1 + 0.3 * r.standard_normal(c)).astype(np.float32), (0.3 * r.standard_normal(c)).astype(np.float32)
    if i8:
        return r.integers(-128, 128, shape).astype(np.int8), w, b, r.integers(-128, 128, shape).astype(np.int8)
    return tuple(f32_to_bf16_bits((4 + 2 * r.standard_normal(shape)).astype(np.float32)) if i in (0, 3) else (w, b)[i - 1] for i in range(4))


@pytest.mark.parametrize("shape,groups", [((3, 1, 1, 8), 8), ((2, 5, 7, 24), 3), ((1, 9, 4, 33), 11), ((4, 2, 2, 64), 1)])
@pytest.mark.parametrize("act", range(3))
def test_oracle_int8_against_its_definition(orc, shape, groups, act):
    x, w, b, res = inputs(shape, groups, True, act)
    for f, use, rs in ((0, None, 0), (5, res, 0), (7, res, 3), (3, None, 0)):
        assert np.array_equal(orc.groupnorm(x, groups, w, b, 1e-3, act, f, use, rs), plain_i8(x, groups, w, b, 1e-3, act, f, use, rs))
    const = np.full(shape, -77, np.int8)                                   # no variance: the bias, rounded half up
    lo, hi = (0 if act else -128), (127 if act < 2 else 6)
    assert np.array_equal(orc.groupnorm(const, groups, w, b, 1e-3, act, 0), np.broadcast_to(np.clip(np.floor(b.astype(np.float64) + 0.5), lo, hi).astype(np.int8), shape))


def test_oracle_int8_rounds_every_operation(orc):
    """Two values a group: products halfway between whole numbers (5 and 0: the deviation is 2.5, a product of -5 * 0.5 / 5 = -0.5 rounds up to 0)."""
    x = np.array([[[[5, 0, 0, 5, 7, 0]]]], np.int8)
    w = np.array([0.5, 0.5, 1.5, 1.5, 2.5, 2.5], np.float32)
    got = orc.groupnorm(x, 3, w, np.zeros(6, np.float32), 0.0, 0, 0)
    assert got.ravel().tolist() == [1, 0, -1, 2, 3, -2]
    assert np.array_equal(got, plain_i8(x, 3, w, np.zeros(6, np.float32), 0.0, 0, 0, None, 0))


@pytest.mark.parametrize("shape,groups", [((3, 1, 1, 8), 4), ((2, 5, 7, 24), 3), ((1, 9, 4, 33), 11)])
@pytest.mark.parametrize("act", range(4))
def test_oracle_bf16_against_its_definition(orc, shape, groups, act):
    x, w, b, res = inputs(shape, groups, False, act)
    for use in (None, res):
        t, size = plain_f64(bf16_bits_to_f32(x), groups, w, b, 1e-5, act, None if use is None else bf16_bits_to_f32(use).astype(np.float64))
        got = bf16_bits_to_f32(orc.groupnorm(x, groups, w, b, 1e-5, act, 0, use)).astype(np.float64)
        assert np.all(np.abs(got - t) <= 2.0 ** -8 * np.abs(t) + 2.0 ** -24 * size + 1e-30)       # the last term: the rounding to float in between


@pytest.fixture(params=[W.DT_I8, W.DT_BF16], ids=["i8", "bf16"])
def net(request):
    return W.norm_net(10, 12, 16, 8, request.param)


def test_readers_accept_and_refuse_alike(orc, net):
    import paper_2209_13443_amd as ee
    check = lambda blob: (orc.blob_check(blob), ee.blob_check(blob.tobytes()))
    assert check(net) == (0, 0)
    norms = [i for i, op in enumerate(net.ops) if int(op["kind"]) == W.OP_GROUPNORM]
    assert len(norms) >= 6
    first = norms[0]
    i8 = net.dtype == W.DT_I8
    for field, value in [("aux", 0), ("aux", 7), ("aux", 8 | 4 << 16), ("aux", 8 | -1 << 16), ("kh", 3), ("stride", 2), ("pad", 1), ("f_lo", -1.0), ("f_lo", np.nan), ("f_lo", np.inf),
                         ("w_off", 4), ("w_off", int(net.ops[first]["w_off"]) + 2), ("b_off", net.raw.size), ("b_off", -64), ("c_out", 32)] + \
                        ([("shift", 8), ("shift", -1), ("res_shift", 9), ("aux", 8 | 3 << 16)] if i8 else []):
        bad = W.Blob(net.tobytes())
        bad.ops[first][field] = value
        assert check(bad) == (-2, -2), (field, value)
    bad = W.Blob(net.tobytes())
    bad.ops[first]["kind"] = 5
    assert check(bad) == (-3, -3)
    bad = W.Blob(net.tobytes())
    bad.ops[first]["res"] = 0                                              # the image: another shape
    assert check(bad) == (-2, -2)


def test_oracle_segments_are_their_layers(orc):
    """A segment of the oracle equals its layers one after the other, through residuals and slices."""
    net = W.norm_net(10, 12, 16, 8, W.DT_I8)
    x = W.input_pool(net, 3)
    kinds = set()
    for s in range(net.n_stages):
        tens = {0: x}
        for op in net.stage_ops(s):
            src, kind = tens[int(op["src"])], int(op["kind"])
            res = tens[int(op["res"])] if int(op["res"]) >= 0 else None
            w, b = net.op_weights(op)
            if kind == W.OP_GROUPNORM:
                kinds.add((int(op["aux"]) >> 16, res is not None, int(op["c_tot"]) != int(op["c_out"])))
                y = plain_i8(src, int(op["aux"]) & 0xFFFF, w, b, float(op["f_lo"]), int(op["aux"]) >> 16, int(op["shift"]), res, int(op["res_shift"]))
            elif kind == W.OP_MAXPOOL:
                y = orc.maxpool_i8(src, int(op["kh"]), int(op["stride"]), int(op["pad"]))
            else:
                acc = orc.conv_acc_i8(src, w.reshape(int(op["c_out"]), int(op["kh"]), int(op["kw"]), int(op["c_in"])), b, int(op["stride"]), int(op["pad"]))
                y = orc.requant_i8(acc, res, int(op["shift"]), int(op["res_shift"]), int(op["lo"]), int(op["hi"]))
            dst, c_off, co, c_tot = int(op["dst"]), int(op["c_off"]), int(op["c_out"]), int(op["c_tot"])
            if c_tot == co:
                tens[dst] = y
            else:
                tens.setdefault(dst, np.full(y.shape[:3] + (c_tot,), 99, np.int8))[..., c_off:c_off + co] = y
        out = orc.stage_forward(net, s, x)
        assert np.array_equal(out, tens[int(net.stages[s]["out_tensor"])])
        assert len(np.unique(out)) > 20
        x = out
    assert {(1, False, False), (2, False, False), (1, True, False), (1, False, True), (0, False, False)} <= kinds


@pytest.mark.parametrize("dtype", [W.DT_I8, W.DT_BF16], ids=["i8", "bf16"])
def test_calibration_of_a_network_with_norms(orc, monkeypatch, dtype):
    """The oracle's calibration goes through the norms, whose scale is the network's own: it stays."""
    import oracle.calibrate as cal
    from workloads import nets
    monkeypatch.setitem(nets.CONFIGS, "norms", (lambda dt: nets._norm_layers(dt, 6, 8, 16, 4, 32), dtype, 0x99))
    monkeypatch.setitem(cal.SPLITS, "norms", (0.5, 0.5))
    rec, blob = cal.calibrate("norms", 24)
    fresh = W.build_net("norms")
    for op, was, entry in zip(blob.ops, fresh.ops, rec["ops"]):
        if int(op["kind"]) == W.OP_GROUPNORM:
            assert entry == dict(shift=int(was["shift"]), res_shift=int(was["res_shift"]))
        elif int(op["kind"]) == W.OP_CONV and dtype == W.DT_I8:
            assert entry["shift"] > 0
    assert np.array_equal(W.apply_calibration(fresh, rec).ops, blob.ops)
    exited = [e["exited"] for e in rec["exits"]]
    assert 6 <= exited[0] <= 18 and sum(exited) == 24
    x = W.input_pool(blob, 24, seed_off=cal.CAL_SEED_OFF)
    flags = orc.exit_head(blob, 0, orc.stage_forward(blob, 0, x), float(blob.exits[0]["thr"]))[3]
    assert int(np.count_nonzero(flags)) == exited[0]


# ---- on the GPU -------------------------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


@pytest.fixture(scope="module")
def ee():
    import paper_2209_13443_amd as ee
    return ee


def dev(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a.view(np.int16) if a.dtype == np.uint16 else a)).cuda()


def host(t, like):
    a = t.cpu().numpy()
    return a.view(np.uint16) if like.dtype == np.uint16 else a


def close(ref, got, what):
    if ref.dtype == np.int8:
        assert np.array_equal(ref, got), f"{what}: {np.count_nonzero(ref != got)} of {ref.size} differ"
    else:
        r, g = bf16_bits_to_f32(ref).astype(np.float64), bf16_bits_to_f32(got).astype(np.float64)
        scale = np.abs(r).reshape(r.shape[0], -1).max(axis=1).reshape(-1, 1, 1, 1) + 1e-30
        assert np.all(np.abs(g - r) <= 2e-2 * scale), f"{what}: {np.max(np.abs(g - r) / scale)}"


@pytest.mark.gpu
@pytest.mark.parametrize("h,w,ci,groups,mid", [(10, 12, 16, 8, 64), (1, 1, 32, 64, 64), (7, 5, 16, 3, 48), (33, 31, 16, 4, 128)])
def test_segments_match_the_oracle(torch, ee, orc, h, w, ci, groups, mid):
    for dtype in (W.DT_I8, W.DT_BF16):
        blob = W.norm_net(h, w, ci, groups, dtype, mid=mid)
        eng = ee.Engine(blob, 16)
        act = W.input_pool(blob, 13)
        for s in range(blob.n_stages):
            for b in (1, 13, 6):
                say(f"[case] {h}x{w}x{ci} groups {groups} dtype {dtype} segment {s} b={b}")
                ref = orc.stage_forward(blob, s, act[:b])
                close(ref, host(eng.stage_forward(s, dev(torch, act[:b]), ref.shape[1:]), ref), f"segment {s} b={b}")
            act = orc.stage_forward(blob, s, act)
        eng.close()


@pytest.mark.gpu
@pytest.mark.parametrize("act", range(4))
def test_one_bf16_layer_within_its_rounding(torch, ee, orc, act):
    """A segment that is one norm (and its exit): the value itself against 64 bits."""
    blob = W.norm_net(10, 12, 16, 8, W.DT_BF16)
    keep = W.Blob(blob.tobytes())
    op, st, e = keep.ops[0:1], keep.stages, keep.exits
    norm = next(o for o in blob.ops if int(o["kind"]) == W.OP_GROUPNORM)
    op[0] = norm
    for k, v in (("src", 0), ("dst", 1), ("res", -1), ("h_in", 10), ("w_in", 12), ("c_in", 16), ("h_out", 10), ("w_out", 12), ("c_out", 16), ("c_off", 0), ("c_tot", 16), ("aux", 4 | act << 16)):
        op[0][k] = v
    keep.header[0]["n_stages"] = 1
    for k, v in (("n_ops", 1), ("n_tensors", 2), ("out_tensor", 1), ("out_h", 10), ("out_w", 12), ("out_c", 16)):
        st[0][k] = v
    for k, v in (("h", 10), ("w", 12), ("c", 16)):
        e[0][k] = v
    assert orc.blob_check(keep) == 0
    x = W.input_pool(keep, 9)
    eng = ee.Engine(keep, 9)
    ref = orc.stage_forward(keep, 0, x)
    got = bf16_bits_to_f32(host(eng.stage_forward(0, dev(torch, x), ref.shape[1:]), ref)).astype(np.float64)
    w, b = keep.op_weights(op[0])
    t, size = plain_f64(bf16_bits_to_f32(x), 4, w, b, float(op[0]["f_lo"]), act, None)
    bound = 2.0 ** -8 * np.abs(t) + 128 * 2.0 ** -24 * size + 1e-30
    assert np.all(np.abs(got - t) <= bound), np.max(np.abs(got - t) / bound)
    assert np.all(np.abs(bf16_bits_to_f32(ref) - t) <= bound)
    eng.close()


@pytest.mark.gpu
def test_large_images_take_two_launches(torch, ee, orc):
    """A norm whose sample no workgroup holds: the workspace of the context, also where the batch changes from call to call."""
    blob = W.norm_net(70, 66, 16, 2, W.DT_I8, mid=64)
    eng = ee.Engine(blob, 5)
    x = W.input_pool(blob, 5)
    for b in (5, 1, 3, 5):
        say(f"[case] 70x66 b={b}")
        ref = orc.stage_forward(blob, 0, x[:b])
        close(ref, host(eng.stage_forward(0, dev(torch, x[:b]), ref.shape[1:]), ref), f"b={b}")
    eng.close()


@pytest.mark.gpu
@pytest.mark.parametrize("lanes,refill", [(1, 1), (2, 2)])
def test_stream_of_a_network_with_norms(torch, ee, orc, lanes, refill):
    """Batches that are compacted and refilled: the statistics are a sample's own, so what a request gets does not depend on the batch it is in."""
    blob = W.norm_net(10, 12, 16, 8, W.DT_I8)
    n, b_max = 48, 8
    x = W.input_pool(blob, n)
    conf = orc.exit_head(blob, 0, orc.stage_forward(blob, 0, x), 2.0)[1]
    blob.exits[0]["thr"] = np.float32(np.median(conf))
    lut = np.array([[100 + 10 * b for b in range(b_max)] for _ in range(2)], np.int64) * 1000
    arrivals = (np.arange(n) * 20000).astype(np.int64)
    ref, rst, rev = orc.serve_stream(blob, arrivals, x, b_max, lut, refill=refill, lanes=lanes, max_events=5000)
    assert np.all(np.bincount(ref["exit_idx"], minlength=2) > 5)
    eng = ee.Engine(blob, b_max)
    assert not eng.zero_copy_supported()                                   # the norm at the border reads packed samples
    assert eng.set_lanes(lanes) == lanes
    for rep in range(2):
        got, gst, gev = eng.serve_stream(arrivals, dev(torch, x), lut, clock=1, refill=refill, lanes=lanes, max_events=5000)
        for f in ("exit_idx", "label", "score", "latency_ns"):
            assert np.array_equal(got[f], ref[f]), (f, rep)
        assert gst == rst and np.array_equal(gev, rev)
    eng.autotune()                                                         # the other layers' tables; nothing changes
    got = eng.serve_stream(arrivals, dev(torch, x), lut, clock=1, refill=refill, lanes=lanes, max_events=5000)[0]
    assert all(np.array_equal(got[f], ref[f]) for f in ("exit_idx", "label", "score"))
    eng.close()


@pytest.mark.gpu
def test_norms_are_timed_in_their_class(torch, ee, orc):
    blob = W.norm_net(10, 12, 16, 8, W.DT_BF16)
    eng = ee.Engine(blob, 4)
    x = dev(torch, W.input_pool(blob, 4))
    eng.stage_forward(0, x, blob.stage_out_shape(0))
    eng.profile(1)
    eng.stage_forward(0, x, blob.stage_out_shape(0))
    cls = eng.profile_read()
    cls = cls[0] if isinstance(cls, tuple) else cls
    assert cls["group_norm"]["launches"] == 3 and cls["group_norm"]["ms"] > 0 and cls["group_norm"]["bytes"] > 0
    us = eng.time_layer(1, 4)
    assert (us[0] if isinstance(us, tuple) else us) > 0
    eng.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [W.DT_I8, W.DT_BF16], ids=["i8", "bf16"])
def test_segments_captured_in_a_graph(torch, ee, orc, dtype):
    """Both segments as one graph, norms of one and of two launches among them: every replay, with the program's own work between them, gives the eager results."""
    blob = W.norm_net(70, 66, 16, 2, dtype, mid=64)
    eng = ee.Engine(blob, 3)
    pool = W.input_pool(blob, 12)
    x = dev(torch, pool[:3])
    shapes = [blob.stage_out_shape(0), blob.stage_out_shape(1)]
    want = []
    for k in range(4):
        mid = eng.stage_forward(0, dev(torch, pool[3 * k:3 * k + 3]), shapes[0])
        want.append(eng.stage_forward(1, mid, shapes[1]).clone())
    torch.cuda.synchronize()
    eng.close()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        eng = ee.Engine(blob, 3, stream=s)
        eng.stage_forward(1, eng.stage_forward(0, x, shapes[0]), shapes[1])
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            out = eng.stage_forward(1, eng.stage_forward(0, x, shapes[0]), shapes[1])
        for k in (0, 1, 2, 3, 1, 0):
            x.copy_(dev(torch, pool[3 * k:3 * k + 3]))
            g.replay()
            s.synchronize()
            assert torch.equal(out, want[k]), k
            torch.ones(1 << 20, device="cuda").sum().item()
        del g
    eng.close()


@pytest.mark.gpu
@pytest.mark.parametrize("h,c,b", [(10, 64, 4), (96, 64, 40), (112, 64, 256)])
def test_timed_norms_cover_all_their_launches(torch, ee, orc, h, c, b):
    """A layer of one launch, of two, and of two for each of two parts of the batch: the profile's time is from the first one's begin to the last one's end, so no less than seven tenths of what the layer
    takes among others like it, where the last launch alone is at most six tenths of two and a third of four."""
    blob = W.norm_net(10, 12, 16, 8, W.DT_BF16)
    keep = W.Blob(blob.tobytes())
    keep.ops[0] = next(o for o in blob.ops if int(o["kind"]) == W.OP_GROUPNORM)
    for k, v in (("src", 0), ("dst", 1), ("res", -1), ("h_in", h), ("w_in", h), ("c_in", c), ("h_out", h), ("w_out", h), ("c_out", c), ("c_off", 0), ("c_tot", c), ("aux", 8)):
        keep.ops[0][k] = v
    keep.header[0]["n_stages"] = 1
    for k, v in (("in_h", h), ("in_w", h), ("in_c", c)):
        keep.header[0][k] = v
    for k, v in (("n_ops", 1), ("n_tensors", 2), ("out_tensor", 1), ("out_h", h), ("out_w", h), ("out_c", c)):
        keep.stages[0][k] = v
    for k, v in (("h", h), ("w", h), ("c", c)):
        keep.exits[0][k] = v
    assert orc.blob_check(keep) == 0
    eng = ee.Engine(keep, b)
    x = torch.randn(b, h, h, c, device="cuda").bfloat16().view(torch.int16)
    eng.stage_forward(0, x, (h, h, c))
    alone = eng.time_layer(0, b)[0]
    eng.profile(1)
    reps = 20
    for _ in range(reps):
        eng.stage_forward(0, x, (h, h, c))
    cls, layers = eng.profile_read(len(keep.ops))
    say(f"[case] {b} x {h}x{h}x{c}: {alone:.1f} us a layer, profile {1e3 * layers[0]['ms'] / reps:.1f}")
    assert cls["group_norm"]["launches"] == layers[0]["launches"] == reps
    assert 1e3 * layers[0]["ms"] / reps >= (0.7 if h > 10 else 0.2) * alone
    eng.close()
