"""What the operators that need no context refuse, and the sizes they ask for: through the C ABI, without a GPU."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def ee():
    import paper_2209_13443_amd as ee
    return ee


def norm(ee, **k):
    d = dict(dtype=ee.EE_BF16, act=0, b=2, pixels=49, c=64, groups=8, frac_bits=0, res_shift=0, eps=1e-5, pad_=0, x_sample=49 * 64, x_pixel=64, res_sample=0, res_pixel=0,
             y_sample=49 * 64, y_pixel=64)
    d.update(k)
    return ee.NormDesc(**d)


P = 4096        # stands for device memory: these calls end before they use it


def test_group_norm_refuses(ee):
    lib, n = ee.raw(), C.c_int64(-1)
    bytes_of = lambda d: lib.ee_group_norm_workspace(C.byref(d), C.byref(n))
    assert lib.ee_group_norm_workspace(None, C.byref(n)) == ee.EE_ERR_ARG and lib.ee_group_norm_workspace(C.byref(norm(ee)), None) == ee.EE_ERR_ARG
    assert bytes_of(norm(ee)) == ee.EE_OK and n.value == 0
    assert bytes_of(norm(ee, pixels=1 << 20)) == ee.EE_OK and n.value > 0
    assert bytes_of(norm(ee, pixels=1 << 20, b=0)) == ee.EE_OK and n.value == 0
    for code, bad in [(ee.EE_ERR_ARG, dict(groups=0)), (ee.EE_ERR_ARG, dict(groups=7)), (ee.EE_ERR_ARG, dict(c=0)), (ee.EE_ERR_ARG, dict(b=-1)), (ee.EE_ERR_ARG, dict(pixels=-1)),
                      (ee.EE_ERR_ARG, dict(eps=-1e-5)), (ee.EE_ERR_ARG, dict(eps=float("nan"))), (ee.EE_ERR_ARG, dict(eps=float("inf"))), (ee.EE_ERR_ARG, dict(act=4)),
                      (ee.EE_ERR_ARG, dict(act=-1)), (ee.EE_ERR_ARG, dict(frac_bits=8)), (ee.EE_ERR_ARG, dict(frac_bits=-1)), (ee.EE_ERR_ARG, dict(res_shift=9)),
                      (ee.EE_ERR_UNSUPPORTED, dict(dtype=2)), (ee.EE_ERR_UNSUPPORTED, dict(dtype=ee.EE_I8, act=3)), (ee.EE_ERR_OVERFLOW, dict(pixels=1 << 25)),
                      (ee.EE_ERR_OVERFLOW, dict(dtype=ee.EE_I8, pixels=1 << 21))]:
        d = norm(ee, **bad)
        assert bytes_of(d) == code, bad
        assert lib.ee_group_norm(C.byref(d), P, None, None, None, P, None, 0, None) == code, bad
    d = norm(ee)
    assert lib.ee_group_norm(C.byref(d), None, None, None, None, P, None, 0, None) == ee.EE_ERR_ARG
    assert lib.ee_group_norm(C.byref(d), P, None, None, None, None, None, 0, None) == ee.EE_ERR_ARG
    assert lib.ee_group_norm(C.byref(d), P + 1, None, None, None, P, None, 0, None) == ee.EE_ERR_ARG
    assert lib.ee_group_norm(C.byref(d), P, P + 2, None, None, P, None, 0, None) == ee.EE_ERR_ARG
    d = norm(ee, c=8200, groups=1, x_pixel=8200, y_pixel=8200)
    assert lib.ee_group_norm(C.byref(d), P, None, None, None, P, None, 0, None) == ee.EE_ERR_UNSUPPORTED
    d = norm(ee, pixels=1 << 20)
    assert bytes_of(d) == ee.EE_OK
    assert lib.ee_group_norm(C.byref(d), P, None, None, None, P, None, 0, None) == ee.EE_ERR_ARG
    assert lib.ee_group_norm(C.byref(d), P, None, None, None, P, P, n.value - 1, None) == ee.EE_ERR_OVERFLOW
    assert lib.ee_group_norm(C.byref(d), P, None, None, None, P, P + 16, n.value, None) == ee.EE_ERR_ARG
    assert lib.ee_group_norm(C.byref(norm(ee, b=0)), None, None, None, None, None, None, 0, None) == ee.EE_OK
    assert lib.ee_group_norm(C.byref(norm(ee, pixels=0)), None, None, None, None, None, None, 0, None) == ee.EE_OK


def test_adapter_projection_refuses(ee):
    lib, n, m = ee.raw(), C.c_int64(-1), C.c_int64(-1)
    dims = lambda ci=64, co=32, adapters=4, rank=8: ee.AdapterDims(ci, co, adapters, rank)
    size = lambda d: lib.ee_adapter_bytes(C.byref(d), C.byref(n), C.byref(m))
    assert size(dims()) == ee.EE_OK and n.value >= 2 * 64 * 32 and m.value >= 2 * 4 * 8 * (64 + 32)
    assert size(dims(adapters=0, rank=0)) == ee.EE_OK
    for code, d in [(ee.EE_ERR_ARG, dims(ci=0)), (ee.EE_ERR_ARG, dims(co=0)), (ee.EE_ERR_ARG, dims(adapters=-1)), (ee.EE_ERR_ARG, dims(rank=0)), (ee.EE_ERR_ARG, dims(rank=-1)),
                    (ee.EE_ERR_OVERFLOW, dims(ci=1 << 19)), (ee.EE_ERR_OVERFLOW, dims(co=1 << 19)), (ee.EE_ERR_OVERFLOW, dims(adapters=1 << 17)), (ee.EE_ERR_OVERFLOW, dims(rank=257))]:
        assert size(d) == code
        assert lib.ee_adapter_pack(C.byref(d), P, 1 << 20, None, P, None) == code
        assert lib.ee_adapter_workspace(C.byref(d), 5, C.byref(n)) == code
    d = dims()
    assert lib.ee_adapter_pack(C.byref(d), None, 64, None, P, None) == ee.EE_ERR_ARG
    assert lib.ee_adapter_pack(C.byref(d), P, 63, None, P, None) == ee.EE_ERR_ARG
    assert lib.ee_adapter_pack(C.byref(d), P, 64, None, P + 16, None) == ee.EE_ERR_ARG
    load = lambda i=0, r=8, a=P, lda=64, b=P, ldb=8, pool=P: lib.ee_adapter_load(C.byref(d), i, r, a, lda, b, ldb, 1.0, pool, None)
    assert [load(i=4), load(i=-1), load(r=9), load(r=-1), load(a=None), load(b=None), load(lda=63), load(ldb=7), load(pool=None), load(pool=P + 128)] == [ee.EE_ERR_ARG] * 10
    assert lib.ee_adapter_workspace(C.byref(d), -1, C.byref(n)) == ee.EE_ERR_ARG
    assert lib.ee_adapter_workspace(C.byref(d), (1 << 22) + 1, C.byref(n)) == ee.EE_ERR_OVERFLOW
    assert lib.ee_adapter_workspace(C.byref(d), 12, C.byref(n)) == ee.EE_OK

    def call(**k):
        c = dict(packed=P, pool=P, x=P, y=P, ids=P, offsets=None, ldx=64, ldy=32, rows=12, slots=4, per=3, out_f32=0, workspace=P, workspace_bytes=n.value)
        c.update(k)
        return lib.ee_adapter_project(C.byref(d), C.byref(ee.AdapterCall(**c)), None)
    for bad in [dict(packed=None), dict(pool=None), dict(x=None), dict(y=None), dict(ids=None), dict(ldx=63), dict(ldy=31), dict(rows=13), dict(rows=-1), dict(slots=-1), dict(per=-3, slots=-4),
                dict(workspace=None), dict(workspace=P + 8), dict(x=P + 1), dict(y=P + 2, out_f32=1), dict(ids=P + 2), dict(offsets=P + 1)]:
        assert call(**bad) == ee.EE_ERR_ARG, bad
    assert call(workspace_bytes=n.value - 1) == ee.EE_ERR_OVERFLOW
    assert call(rows=0, slots=0) == ee.EE_OK and call(rows=0, slots=5, per=0) == ee.EE_OK
    assert lib.ee_adapter_project(C.byref(d), None, None) == ee.EE_ERR_ARG


def test_verify_draft_refuses(ee):
    lib, n = ee.raw(), C.c_int64(-1)
    assert lib.ee_verify_workspace(3, 4, 1000, C.byref(n)) == ee.EE_OK
    assert [lib.ee_verify_workspace(-1, 4, 9, C.byref(n)), lib.ee_verify_workspace(1, -1, 9, C.byref(n)), lib.ee_verify_workspace(1, 1, 0, C.byref(n)), lib.ee_verify_workspace(1, 1, 1, None)] == \
        [ee.EE_ERR_ARG] * 4
    assert lib.ee_verify_workspace(1, 1, (1 << 30) + 1, C.byref(n)) == ee.EE_ERR_OVERFLOW
    assert lib.ee_verify_workspace(3, 4, 100000, C.byref(n)) == ee.EE_OK and n.value > 0

    def call(**k):
        c = dict(draft=P, p=P, q=P, u=P, lengths=P, accepted=P, tokens=P, draft_row=4, u_row=5, p_seq=500000, p_row=100000, q_seq=400000, q_row=100000, b=3, k=4, v=100000, f32=1, workspace=P,
                 workspace_bytes=n.value)
        c.update(k)
        return lib.ee_verify_draft(C.byref(ee.VerifyCall(**c)), None)
    for bad in [dict(draft=None), dict(p=None), dict(u=None), dict(accepted=None), dict(tokens=None), dict(b=-1), dict(k=-1), dict(v=0), dict(p=P + 2), dict(q=P + 2), dict(q=P + 1, f32=0),
                dict(draft=P + 1), dict(u=P + 2), dict(lengths=P + 3), dict(accepted=P + 2), dict(tokens=P + 2), dict(workspace=None), dict(workspace=P + 16)]:
        assert call(**bad) == ee.EE_ERR_ARG, bad
    assert call(workspace_bytes=n.value - 1) == ee.EE_ERR_OVERFLOW
    assert call(v=(1 << 30) + 1) == ee.EE_ERR_OVERFLOW and call(b=1 << 24) == ee.EE_ERR_OVERFLOW and call(b=1 << 20, k=1 << 10) == ee.EE_ERR_OVERFLOW
    assert call(b=0) == ee.EE_OK
    assert lib.ee_verify_draft(None, None) == ee.EE_ERR_ARG


def test_group_norm_refuses_layouts(ee):
    lib, n = ee.raw(), C.c_int64(-1)

    def both(code, **k):
        d = norm(ee, **k)
        assert lib.ee_group_norm_workspace(C.byref(d), C.byref(n)) == code, k
        if code:
            assert lib.ee_group_norm(C.byref(d), P, None, None, P, P, P, 1 << 40, None) == code, k
    for k in [dict(x_pixel=-64), dict(res_pixel=-1), dict(y_pixel=-64), dict(y_pixel=63)]:
        both(ee.EE_ERR_ARG, **k)
    for k in [dict(x_pixel=1 << 20), dict(res_pixel=1 << 20), dict(y_pixel=1 << 20), dict(pixels=1 << 22, x_pixel=512), dict(pixels=1 << 22, y_pixel=512)]:
        both(ee.EE_ERR_OVERFLOW, **k)
    for k in [dict(y_sample=-49 * 64), dict(y_sample=64, y_pixel=128), dict(b=1, y_sample=0), dict(pixels=1, y_sample=64, y_pixel=0, x_pixel=-5), dict(x_sample=0), dict(x_pixel=0, res_pixel=0),
              dict(b=0, y_sample=0), dict(pixels=0, y_sample=0)]:
        both(ee.EE_OK, **k)


def test_group_norm_refuses_samples_of_2_gib(ee):
    """Up to the last number of pixels: what a sample spans is counted in 64 bits."""
    lib, n = ee.raw(), C.c_int64(-1)
    for pixels in (1 << 30, (1 << 31) - 1024, (1 << 31) - 500, (1 << 31) - 1):
        d = norm(ee, b=1, pixels=pixels, c=1, groups=1, x_sample=pixels, x_pixel=1, res_pixel=1, y_sample=pixels, y_pixel=1)
        assert lib.ee_group_norm_workspace(C.byref(d), C.byref(n)) == ee.EE_ERR_OVERFLOW, pixels
        assert lib.ee_group_norm(C.byref(d), P, None, None, None, P, P, 1 << 40, None) == ee.EE_ERR_OVERFLOW, pixels


def test_binding_refuses_sizes_past_32_bits(ee):
    """Sizes, numbers of adapters and places that an int32 cannot hold, of tensors that a GPU's memory may hold: refused, not cut down to what their lower bits say."""
    import torch
    big, key = 1 << 32, lambda shape, dtype=torch.bfloat16: (shape, tuple(torch.Size(shape[i + 1:]).numel() for i in range(len(shape))), dtype, 0)

    def refused(f, *a):
        with pytest.raises(ee.EEError) as e:
            f(*a)
        assert e.value.code == ee.EE_ERR_OVERFLOW
    plan = lambda x, groups=4, frac=0, rs=0: ee._norm_plan(x, None, None, None, None, groups, 1e-5, "none", frac, rs)
    assert plan(key((5, 7, 8)))[0] == 0
    for call in [(key((big + 5, 1, 8)),), (key((1, big + 7, 8)),), (key((1, 1, big + 8)),), (key((5, 7, 8)), big + 4), (key((5, 7, 8)), 4 - big), (key((5, 7, 8)), 4, big), (key((5, 7, 8)), 4, 0, -big)]:
        refused(plan, *call)
    project = lambda x, ids, offsets=None: ee._adapter_plan(0, 8, 16, 2, 4, torch.bfloat16, x, ids, offsets, None)
    ints = torch.int32
    assert project(key((5, 8)), key((5,), ints))[0] == 5
    refused(project, key((big + 5, 8)), key((big + 5,), ints))
    refused(project, key((3, big, 8)), key((3,), ints))
    refused(project, key((5, 8)), key((big + 1,), ints), key((big + 2,), ints))
    verify = lambda b, k, v: ee._verify_plan(key((b, k + 1, v), torch.float32), key((b, k), ints), key((b, k + 1), torch.float32), None, None)
    assert verify(2, 3, 9)[1:4] == (2, 3, 9)
    for sizes in [(big + 2, 3, 9), (2, big + 3, 9), (2, 3, big + 9)]:
        refused(verify, *sizes)
    held = object.__new__(ee.AdapterProjection)                       # a handle without device memory
    held.device, held.ci, held.co, held._dims, held._pool = torch.device("cuda", 0), 8, 16, ee.AdapterDims(8, 16, 2, 4), torch.zeros(1)
    refused(held.unload, big)
    refused(held.unload, big + 1)


def test_adapter_projection_refuses_results_over_its_input(ee):
    lib, n = ee.raw(), C.c_int64(-1)
    d = ee.AdapterDims(64, 64, 0, 0)
    assert lib.ee_adapter_workspace(C.byref(d), 12, C.byref(n)) == ee.EE_OK
    x = 1 << 20

    def call(y, **k):
        c = dict(packed=P, pool=None, x=x, y=y, ids=None, offsets=None, ldx=64, ldy=64, rows=12, slots=12, per=1, out_f32=0, workspace=P, workspace_bytes=n.value)
        c.update(k)
        return lib.ee_adapter_project(C.byref(d), C.byref(ee.AdapterCall(**c)), None)
    last = 2 * (11 * 64 + 64)                                             # bytes of x
    for bad in [dict(y=x), dict(y=x + 2), dict(y=x - 2), dict(y=x + last - 2), dict(y=x - last + 2), dict(y=x, out_f32=1), dict(y=x - 2 * last + 4, out_f32=1), dict(y=x + 64, ldx=128, ldy=128),
                dict(y=x - 130, ldx=192, ldy=192, rows=1, slots=1, per=1, x=x - 4), dict(y=x + 128, ldx=127, ldy=127), dict(y=x + 128, ldx=128, ldy=192), dict(y=x + 128, ldx=128, ldy=96, out_f32=1),
                dict(y=x, rows=1, slots=1), dict(y=x + 126, rows=1, slots=1, ldx=4096, ldy=4096)]:
        assert call(**bad) == ee.EE_ERR_ARG, bad


def test_group_norm_refuses_results_over_a_part_of_its_input(ee):
    lib, n = ee.raw(), C.c_int64(-1)
    x = 1 << 20
    whole = 2 * 2 * 49 * 64                                               # bytes of a dense x
    for k, y, res in [({}, x + 2, None), ({}, x - 2, None), ({}, x + 2 * 64, None), ({}, x + whole - 2, None), ({}, x - whole + 2, None), ({}, x - whole, x - 2), ({}, x + 2 * whole, x + 2 * whole + 16),
                      (dict(y_pixel=96, y_sample=49 * 96), x, None), (dict(x_pixel=128, y_pixel=128, x_sample=49 * 128, y_sample=49 * 128), x + 64, None),
                      (dict(x_sample=49 * 64, y_sample=2 * 49 * 64), x, None), (dict(x_sample=0), x, None), (dict(pixels=1, x_sample=64, y_sample=128), x, None), (dict(b=1), x + 2, None)]:
        d = norm(ee, res_sample=49 * 64, res_pixel=64)
        for name, v in k.items():
            setattr(d, name, v)
        assert lib.ee_group_norm(C.byref(d), x, None, None, res, y, None, 0, None) == ee.EE_ERR_ARG, (k, y, res)
