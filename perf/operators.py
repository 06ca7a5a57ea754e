"""The operators over a batch of in-flight requests that the library offers as calls of their own: group norm with an activation
(channels last), a shared projection with each request's low-rank adapter beside it, and the verification of drafted tokens.

A case is a dict of plain values, `prepare` makes what a program holds before the call, `run` is one pass, `work` says what a
pass cannot do without, `exact` computes it in 64 bits from the definition.  With `own` false `run` is the plain form: elementary
torch operations in 32 bits (64 where a result is a whole number next to a border), rounded once at the end.

Kinds of cases
  norm     group_norm on activations [slot][H][W][C], bf16 or int8, alone or as a channel slice of a wider (concatenated) tensor
  adapt    AdapterProjection on rows of slots: `per` rows a slot (1: decoding, or a head on pooled features; H*W: a 1x1 layer),
           or runs of different lengths packed one behind the other (per = 0)
  verify   verify_draft on the probabilities of a draft and a target
"""
import math

import torch

own = False

_ACTS = ("none", "relu", "silu")


def _norm(name, dtype, b, h, w, c, groups, act, res=False, c_tot=0):
    return dict(name=name, kind="norm", dtype=dtype, b=b, h=h, w=w, c=c, groups=groups, act=act, res=res, c_tot=c_tot or c)


def _adapt(name, slots, per, rows, ci, co, rank, adapters, out, bias):
    return dict(name=name, kind="adapt", slots=slots, per=per, rows=rows, ci=ci, co=co, rank=rank, adapters=adapters, out=out, bias=bias)


def _verify(name, b, k, v, dtype, certain=False, ragged=False):
    return dict(name=name, kind="verify", b=b, k=k, v=v, dtype=dtype, certain=certain, ragged=ragged)


def listed():
    return [
        # the smallest call: the last feature map of one image
        _norm("norm_one_7x7", "bf16", 1, 7, 7, 512, 32, "relu"),
        # the end of a bottleneck block of the 56 x 56 group, 64 slots: norm, shortcut and activation
        _norm("norm_block_56_res", "bf16", 64, 56, 56, 256, 32, "relu", res=True),
        # the first layer's output in the large-batch bf16 stream, two channels to a group
        _norm("norm_stem_112", "bf16", 256, 112, 112, 64, 32, "silu"),
        # an int8 network's 14 x 14 group with its shortcut, 64 slots
        _norm("norm_block_14_i8", "int8", 64, 14, 14, 1024, 32, "relu", res=True),
        # one branch of a concatenating block on a ragged batch: a slice of 96 of 288 channels
        _norm("norm_slice_35", "bf16", 37, 35, 35, 96, 12, "none", c_tot=288),
        # exit heads of a full batch: pooled features to float logits, every slot with its own user's adapter
        _adapt("adapt_head_64", 64, 1, 64, 2048, 1000, 16, 24, "fp32", True),
        # decoding: one token each of a few requests through a square projection
        _adapt("adapt_decode_12", 12, 1, 12, 4096, 4096, 16, 8, "bf16", False),
        # a 1x1 layer of the 14 x 14 group over 64 slots
        _adapt("adapt_layer_14", 64, 196, 64 * 196, 1024, 256, 32, 16, "bf16", True),
        # packed prompts of very different lengths
        _adapt("adapt_prompts", 24, 0, 8000, 4096, 4096, 64, 16, "bf16", False),
        # one sequence, few classes: latency
        _verify("verify_one", 1, 4, 1000, "fp32"),
        # a serving batch, sequences that drafted fewer tokens than others among them
        _verify("verify_64", 64, 5, 32000, "fp32", ragged=True),
        # the largest: many sequences, long drafts, a large vocabulary in bf16
        _verify("verify_256", 256, 8, 128256, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "adapt", "adapt", "verify"))
    if kind == "norm":
        per = rng.choice((1, 2, 3, 4, 6, 8, 8, 16, 16, 24, 32, 40, 64))
        groups = rng.choice((1, 2, 3, 8, 12, 16, 32, 32, 32))
        c, h, w = per * groups, _log_int(rng, 1, 128), _log_int(rng, 1, 128)
        b = _log_int(rng, 1, max(1, min(256, 256 * 112 * 112 * 64 // (2 * c * h * w))))
        dtype = rng.choice(("bf16", "bf16", "int8"))
        case = _norm("", dtype, b, h, w, c, groups, rng.choice(_ACTS if dtype == "bf16" else _ACTS[:2]), rng.random() < 0.4,
                     c * rng.choice((1, 1, 1, 2, 3)))
    elif kind == "adapt":
        ci, co = (_log_int(rng, 8, 512) * rng.choice((1, 8, 8, 8)) for _ in range(2))
        slots = _log_int(rng, 1, 256)
        per = rng.choice((1, 1, 0, _log_int(rng, 1, 3136)))
        most = max(1, min(1 << 15, (8000 * 4096 * 4096) // (2 * ci * co)))
        slots = min(slots, most)
        rows = slots * min(per, max(1, most // slots)) if per else _log_int(rng, slots, max(slots, most))
        per = rows // slots if per else 0
        case = _adapt("", slots, per, rows, ci, co, rng.choice((1, 4, 8, 10, 16, 16, 32, 64, 128)), _log_int(rng, 1, 32),
                      rng.choice(("bf16", "fp32")), rng.random() < 0.5)
    else:
        dtype = rng.choice(("fp32", "bf16"))
        case = _verify("", _log_int(rng, 1, 256), rng.randint(1, 8), _log_int(rng, 10, 128000 if dtype == "bf16" else 64000), dtype,
                       rng.random() < 0.25, rng.random() < 0.5)
    del case["name"]
    return case


def _prepare_norm(case, gen):
    shape = (case["b"], case["h"], case["w"])
    c, tot = case["c"], case["c_tot"]
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)
    weight, bias = 1.0 + 0.25 * rand(c), 0.25 * rand(c)
    # activations of a channel lie around a level of its own; the input of an int8 layer uses most of its range
    level = 0.5 * rand(tot)
    x = torch.empty(shape + (tot,), dtype=torch.bfloat16 if case["dtype"] == "bf16" else torch.int8, device="cuda")
    res = torch.empty(shape + (c,), dtype=x.dtype, device="cuda") if case["res"] else None
    for i in range(0, case["b"], 32):
        part, r = rand(min(32, case["b"] - i), case["h"], case["w"], tot) + level, None
        if res is not None:
            r = rand(part.shape[0], case["h"], case["w"], c)
        if case["dtype"] == "int8":
            part, r = (30.0 * part).round_().clamp_(-128, 127), None if r is None else (25.0 * r).round_().clamp_(-128, 127)
        x[i:i + 32] = part
        if r is not None:
            res[i:i + 32] = r
    return dict(case=case, x=x[..., tot - c:], weight=weight, bias=bias, res=res)


def _prepare_adapt(case, gen):
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)
    m, ci, co, r, n = (case[k] for k in ("rows", "ci", "co", "rank", "adapters"))
    x = rand(m, ci).to(torch.bfloat16)
    weight = (rand(co, ci) / math.sqrt(ci)).to(torch.bfloat16)
    a, b = (rand(n, r, ci) / math.sqrt(ci)).to(torch.bfloat16), (rand(n, co, r) / math.sqrt(r)).to(torch.bfloat16)
    scale = 0.5 + torch.rand(n, device="cuda", generator=gen)
    ids = torch.randint(0, n, (case["slots"],), device="cuda", generator=gen, dtype=torch.int32)
    ids[torch.rand(case["slots"], device="cuda", generator=gen) < 0.2] = -1          # requests without an adapter
    state = dict(case=case, weight=weight, a=a, b=b, scale=scale, ids=ids, bias=rand(co) if case["bias"] else None, offsets=None)
    if case["per"]:
        x = x.view(case["slots"], case["per"], ci)
    else:                                                                             # cuts anywhere: runs of no row among them
        cuts = torch.randint(0, m + 1, (case["slots"] - 1,), device="cuda", generator=gen).sort().values
        state["offsets"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), m)]).to(torch.int32)
    if own:                                                                           # what a serving program keeps: the weights, laid out once
        import paper_2209_13443_amd as ee
        state["proj"] = ee.AdapterProjection(weight, state["bias"], adapters=n, rank=r)
        for i, s in enumerate(scale.tolist()):
            state["proj"].load(i, a[i], b[i], s)
    return dict(state, x=x)


def _prepare_verify(case, gen):
    b, k, v = case["b"], case["k"], case["v"]
    dtype = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    p = torch.empty(b, k + 1, v, dtype=dtype, device="cuda")
    q = None if case["certain"] else torch.empty(b, k, v, dtype=dtype, device="cuda")
    draft = torch.empty(b, k, dtype=torch.int32, device="cuda")
    for i in range(0, b, 16):
        n = min(16, b - i)
        logits = 2.5 * torch.randn(n, k + 1, v, device="cuda", generator=gen)
        p[i:i + n] = torch.softmax(logits, -1)
        # the draft is a weaker model of the same thing; its tokens are drawn from its own probabilities
        weak = logits[:, :k] + 0.5 * torch.randn(n, k, v, device="cuda", generator=gen)
        if q is not None:
            q[i:i + n] = torch.softmax(weak, -1)
            weak = weak - torch.empty_like(weak).exponential_(generator=gen).log_()
        draft[i:i + n] = weak.argmax(-1)
    lengths = torch.randint(0, k + 1, (b,), device="cuda", generator=gen, dtype=torch.int32) if case["ragged"] else None
    return dict(case=case, draft=draft, p=p, q=q, u=torch.rand(b, k + 1, device="cuda", generator=gen), lengths=lengths)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"norm": _prepare_norm, "adapt": _prepare_adapt, "verify": _prepare_verify}[case["kind"]](case, gen)


FRAC_BITS, RES_SHIFT, EPS = 5, 0, 1e-5


def _plain_norm(s):
    case, x, res = s["case"], s["x"], s["res"]
    b, c, g = case["b"], case["c"], case["groups"]
    if case["dtype"] == "int8":
        xg = x.reshape(b, -1, g, c // g).double()
        n = xg.shape[1] * xg.shape[3]
        s1, s2 = xg.sum((1, 3), keepdim=True), xg.square().sum((1, 3), keepdim=True)
        mult = s["weight"].double().view(g, c // g) * 2.0 ** FRAC_BITS / torch.sqrt((n * s2 - s1 * s1) / float(n) ** 2 + EPS) / n
        y = ((n * xg - s1) * mult + (s["bias"].double().view(g, c // g) * 2.0 ** FRAC_BITS + 0.5)).view(x.shape)
        if res is not None:
            y = y + res.double() * 2.0 ** RES_SHIFT
        return y.floor().clamp(-128 if case["act"] == "none" else 0, 127).to(torch.int8)
    xg = x.reshape(b, -1, g, c // g).float()
    d = xg - xg.mean((1, 3), keepdim=True)
    y = d * torch.rsqrt(d.square().mean((1, 3), keepdim=True) + EPS)
    y = (y * s["weight"].view(g, c // g) + s["bias"].view(g, c // g)).view(x.shape)
    if res is not None:
        y = y + res.float()
    if case["act"] == "relu":
        y = y.clamp(min=0)
    if case["act"] == "silu":
        y = y * torch.sigmoid(y)
    return y.to(torch.bfloat16)


def _row_ids(s):
    """The adapter of every row."""
    case, ids = s["case"], s["ids"].long()
    rows = torch.arange(case["rows"], device="cuda")
    return ids[rows // case["per"]] if case["per"] else ids[torch.searchsorted(s["offsets"].long(), rows, right=True) - 1]


def _plain_adapt(s):
    case = s["case"]
    x = s["x"].reshape(case["rows"], case["ci"]).float()
    n, r, co = case["adapters"], case["rank"], case["co"]
    y = x @ s["weight"].float().T
    # every row through every adapter's first half, the other adapters' results are cleared
    u = (x @ s["a"].float().view(n * r, -1).T).view(-1, n, r)
    mine = _row_ids(s)[:, None] == torch.arange(n, device="cuda")
    u = torch.where(mine[:, :, None], u * s["scale"][:, None], u.new_zeros(()))
    y = y + u.view(-1, n * r) @ s["b"].float().transpose(0, 1).reshape(co, n * r).T
    if s["bias"] is not None:
        y = y + s["bias"]
    y = y.to(torch.bfloat16 if case["out"] == "bf16" else torch.float32)
    return y.view(s["x"].shape[:-1] + (co,))


def _plain_verify(s):
    case, p, q, u = s["case"], s["p"], s["q"], s["u"].double()
    b, k = case["b"], case["k"]
    every, at = torch.arange(b, device="cuda"), s["draft"].long()
    length = s["lengths"].long() if s["lengths"] is not None else at.new_full((b,), k)
    px = p[:, :k].gather(2, at[..., None])[..., 0].double()
    qx = q.gather(2, at[..., None])[..., 0].double() if q is not None else torch.ones_like(px)
    ok = (u[:, :k] * qx < px) & (torch.arange(k, device="cuda") < length[:, None])
    n = ok.long().cumprod(1).sum(1)
    row = p[every, n].double()
    last = n.clamp(max=k - 1)
    if q is not None:
        less = q[every, last].double()
    else:
        less = torch.zeros_like(row).scatter_(1, at[every, last][:, None], 2.0)
    refused = (n < length)[:, None]
    w = (row - torch.where(refused, less, less.new_zeros(()))).clamp(min=0)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, row)
    cum = w.cumsum(1)
    token = (cum > u[:, k:] * cum[:, -1:]).long().argmax(1)
    places = torch.arange(k + 1, device="cuda")
    drafted = torch.cat([at, at.new_zeros(b, 1)], 1)
    tokens = torch.where(places < n[:, None], drafted, torch.where(places == n[:, None], token[:, None], -1))
    return dict(accepted=n.int(), tokens=tokens.int())


def run(state):
    case = state["case"]
    if not own:
        return {"norm": _plain_norm, "adapt": _plain_adapt, "verify": _plain_verify}[case["kind"]](state)
    import paper_2209_13443_amd as ee
    if case["kind"] == "norm":
        return ee.group_norm(state["x"], case["groups"], state["weight"], state["bias"], eps=EPS, act=case["act"], residual=state["res"],
                             frac_bits=FRAC_BITS, res_shift=RES_SHIFT)
    if case["kind"] == "adapt":
        return state["proj"](state["x"], state["ids"], offsets=state["offsets"], dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32)
    accepted, tokens = ee.verify_draft(state["draft"], state["p"], state["u"], draft_probs=state["q"], lengths=state["lengths"])
    return dict(accepted=accepted, tokens=tokens)


def work(case):
    if case["kind"] == "norm":
        n = case["b"] * case["h"] * case["w"] * case["c"]
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 1) * (3 if case["res"] else 2) + 8 * case["c"], "flops": 8.0 * n}
    if case["kind"] == "adapt":
        m, ci, co, r = case["rows"], case["ci"], case["co"], case["rank"]
        used = min(case["adapters"], case["slots"])
        return {"bytes": 2 * (m * ci + co * ci) + (2 if case["out"] == "bf16" else 4) * m * co + 2 * used * r * (ci + co) + (4 * co if case["bias"] else 0),
                "flops": 2.0 * m * ci * co + 2.0 * m * r * (ci + co)}
    es, rows = (4 if case["dtype"] == "fp32" else 2), 1 if case["certain"] else 2
    b, k, v = case["b"], case["k"], case["v"]
    return {"bytes": b * (rows * es * v + k * (rows * es + 4) + 8 * (k + 1) + 4), "flops": 3.0 * b * v}


def _exact_norm(s):
    case = s["case"]
    b, c, g = case["b"], case["c"], case["groups"]
    if case["dtype"] == "bf16" and b * case["h"] * case["w"] * c > 1 << 28:
        return None
    out = torch.empty(s["x"].shape, dtype=torch.float64 if case["dtype"] == "bf16" else torch.int8, device="cuda")
    for i in range(b):
        x = s["x"][i].double().reshape(-1, c)
        n = x.shape[0] * (c // g)
        mean = (x.sum(0).view(g, -1).sum(1) / n).repeat_interleave(c // g)
        var = ((x - mean).square().sum(0).view(g, -1).sum(1) / n).repeat_interleave(c // g)
        y = (x - mean) / (var + EPS).sqrt() * s["weight"].double() + s["bias"].double()
        r = 0.0 if s["res"] is None else s["res"][i].double().reshape(-1, c)
        if case["dtype"] == "int8":
            y = (y * 2 ** FRAC_BITS + r * 2 ** RES_SHIFT + 0.5).floor().clamp(0 if case["act"] == "relu" else -128, 127)
        else:
            y = y + r
            y = torch.relu(y) if case["act"] == "relu" else y / (1 + (-y).exp()) if case["act"] == "silu" else y
        out[i] = y.view(out[i].shape)
    return out


def _exact_adapt(s):
    case = s["case"]
    m, ci, co = case["rows"], case["ci"], case["co"]
    x, rows = s["x"].reshape(m, ci).double(), _row_ids(s)
    y = torch.matmul(x, s["weight"].double().t())
    if s["bias"] is not None:
        y += s["bias"].double()
    for i in range(case["adapters"]):
        at = (rows == i).nonzero()[:, 0]
        y[at] += torch.matmul(torch.matmul(x[at], s["a"][i].double().t()), s["b"][i].double().t()) * s["scale"][i].double()
    return y.view(s["x"].shape[:-1] + (co,))


def _exact_verify(s):
    case = s["case"]
    k = case["k"]
    draft, u = s["draft"].tolist(), s["u"].tolist()
    lengths = [k] * case["b"] if s["lengths"] is None else s["lengths"].tolist()
    accepted, tokens = [], []
    for i in range(case["b"]):
        got = []
        for j in range(lengths[i]):
            p, q = s["p"][i, j, draft[i][j]].item(), 1.0 if s["q"] is None else s["q"][i, j, draft[i][j]].item()
            if not u[i][j] * q < p:
                break
            got.append(draft[i][j])
        n = len(got)
        w = s["p"][i, n].double()
        if n < lengths[i]:
            less = w.clone()
            if s["q"] is None:
                less[draft[i][n]] = 0
            else:
                less -= s["q"][i, n].double()
            less = torch.where(less > 0, less, torch.zeros_like(less))
            w = less if less.sum().item() > 0 else w
        steps = torch.cumsum(w, 0)
        got.append(int((steps <= u[i][k] * steps[-1]).sum().item()))
        accepted.append(n)
        tokens.append(got + [-1] * (k - n))
    return dict(accepted=torch.tensor(accepted, dtype=torch.int32), tokens=torch.tensor(tokens, dtype=torch.int32))


def exact(case, seed):
    return {"norm": _exact_norm, "adapt": _exact_adapt, "verify": _exact_verify}[case["kind"]](prepare(case, seed))
