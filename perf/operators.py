"""Performance cases of the operators around the attention: norms, rotary positions
and the paged cache.

Each case is one call path through paper_2504_06949_amd.ops:

  norm     norm_forward(), and for training norm_backward(): the layer's input norm
           (one weight row), or the QK-norm of head-split rows (a weight row per head)
  rotary   Rotary.forward() on queries and keys, and for training Rotary.backward()
  append   PagedCache.append(): new tokens' keys, values and gates into the pages
  attend   PagedCache.attend(): attention of the new tokens over the pages

`own` selects between those calls and the plain form of the same operators in
elementary torch operations.  Inputs are synthetic, drawn on the GPU: N(0, 1) rows,
QK-normed queries and keys where the cache's pruning bound needs them, gate logits
a ~ N(mu_h, 0.5) with the heads' means spread evenly over [1, 10].
"""
import math

import numpy as np
import torch

own = False

EPS = math.exp(-10.0)    # bound of the pruned mass
PAGE = 64                # positions per page
L_MAX = 131072           # longest sequence the cache's threshold is sized for


def listed():
    return [
        # QK-norm of one new token per sequence: the smallest call of a serving step.
        _norm("norm_token", B=8, H=12, L=1, n=64, groups=True, train=False),
        # QK-norm of a training step of the 125M layer (32k tokens), read from a fused
        # projection's [B, L, H, d] rows, with its backward pass.
        _norm("norm_qk_train", B=8, H=12, L=4096, n=64, groups=True, train=True, strided=True),
        # The layer's input norm of the same step, with mean and bias.
        _norm("norm_layer_train", B=1, H=1, L=32768, n=768, center=True, train=True),
        # float32, a width that no vector load divides: gradient checks, odd models.
        _norm("norm_f32_odd", B=1, H=1, L=1000, n=1537, dtype="f32", center=True, train=True),
        # Rotary positions of one new token for each of 16 sequences.
        _rotary("rotary_token", B=16, H=12, Hk=12, L=1, d=64, rot=64),
        # Queries and keys of the 125M layer's training step, with the backward pass.
        _rotary("rotary_train", B=8, H=12, Hk=12, L=4096, d=64, rot=64, train=True),
        # A long prompt: part of the head, neighbouring pairs, frequencies scaled by
        # ramp, shared key heads, ragged length, far positions.
        _rotary("rotary_long", B=1, H=16, Hk=4, L=30001, d=128, rot=96, layout="interleaved",
                scaling="ramp", start=900000),
        # One token each for 64 sequences.
        _paged("append_token", "append", H=12, Hk=12, d=64, new=[1] * 64,
               past=[37 * i % 4099 for i in range(64)]),
        # Prompts of a ragged batch, 32k tokens in all, one of them continued.
        _paged("append_prompts", "append", H=12, Hk=12, d=64,
               new=[8192, 5001, 77, 16384, 1, 2500, 613], past=[0, 0, 64, 0, 0, 1001, 3]),
        # Generation: one token each after 4k to 64k tokens.
        _paged("attend_token", "attend", H=12, Hk=12, d=64, new=[1] * 8,
               past=[4096, 65535, 20000, 8191, 33333, 5000, 12345, 50001]),
        # Chunks of new tokens beside single ones (a serving step of mixed requests).
        _paged("attend_mixed", "attend", H=12, Hk=12, d=64, new=[512, 1, 1, 300, 1, 1, 17, 1],
               past=[16000, 4000, 9999, 0, 30000, 64, 1000, 2047]),
        # A long prompt in one chunk, head dimension 128, four query heads per key head.
        _paged("attend_prompt", "attend", H=16, Hk=4, d=128, new=[8000], past=[8150]),
    ]


def _named(name, c):
    return {"name": name, **c} if name else c


def _norm(name, B, H, L, n, dtype="bf16", center=False, groups=False, train=False, strided=False):
    return _named(name, {"kind": "norm", "B": B, "H": H, "L": L, "n": n, "dtype": dtype, "center": center,
                         "groups": groups, "train": train, "strided": strided})


def _rotary(name, B, H, Hk, L, d, rot, dtype="bf16", layout="half", scaling="none", start=0,
            train=False):
    return _named(name, {"kind": "rotary", "B": B, "H": H, "Hk": Hk, "L": L, "d": d, "rot": rot,
                         "dtype": dtype, "layout": layout, "scaling": scaling, "start": start,
                         "train": train})


def _paged(name, kind, H, Hk, d, new, past, dtype="bf16"):
    return _named(name, {"kind": kind, "H": H, "Hk": Hk, "d": d, "dtype": dtype,
                         "new": " ".join(map(str, new)), "past": " ".join(map(str, past))})


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "rotary", "rotary", "append", "append", "token", "chunk"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "norm":
        train = rng.random() < 0.6
        if rng.random() < 0.5:
            B, H, n = rng.randint(1, 8), rng.choice([1, 3, 4, 8, 12, 16, 24]), rng.choice([64, 64, 128])
            L = _log_int(rng, 1, max(1, 25000000 // (B * H * n)))
            return _norm("", B, H, L, n, dtype, False, True, train, rng.random() < 0.5)
        n = _log_int(rng, 33, 8192)
        if rng.random() < 0.6:
            n = max(64, n // 64 * 64)
        return _norm("", 1, 1, _log_int(rng, 1, 25000000 // n), n, dtype, rng.random() < 0.6, False, train)
    if kind == "rotary":
        d = rng.choice([64, 64, 80, 128])
        Hk = rng.choice([1, 2, 4, 8, 12])
        H = Hk * rng.choice([1, 1, 2, 3])
        B = rng.randint(1, 8)
        L = _log_int(rng, 1, max(1, 50000000 // (B * (H + Hk) * d)))
        rot = rng.choice([d, d, d // 2, 2 * rng.randint(3, d // 2)])
        return _rotary("", B, H, Hk, L, d, rot, dtype, rng.choice(["half", "interleaved"]),
                       rng.choice(["none", "linear", "base", "ramp"]),
                       rng.choice([0, 0, _log_int(rng, 1, 1000000)]), rng.random() < 0.5)
    d = rng.choice([64, 64, 128])
    Hk = rng.choice([1, 2, 4, 8, 12])
    H = Hk * rng.choice([1, 1, 2, 4, 8])
    if H > 32:
        H = Hk
    N = _log_int(rng, 1, 32)
    if kind == "append":
        most = max(1, min(16384, 25000000 // (N * Hk * d)))
        single = rng.random() < 0.4
        return _paged("", "append", H, Hk, d, [1 if single else _log_int(rng, 1, most) for _ in range(N)],
                      [rng.choice([0, rng.randint(1, 3000)]) for _ in range(N)], dtype)
    keys = 200000000 // (Hk * d)          # positions that all sequences hold together
    if kind == "token":
        most = max(2, min(65536, keys // N))
        return _paged("", "attend", H, Hk, d, [1] * N, [_log_int(rng, 1, most) - 1 for _ in range(N)], dtype)
    N = min(N, 8)
    new = [1 if rng.random() < 0.3 else _log_int(rng, 1, 2048) for _ in range(N)]
    past = [rng.choice([0, _log_int(rng, 1, max(2, min(16384, keys // N)))]) for _ in range(N)]
    # no more products than the largest listed case, and a plain pass well below a second
    while sum(a * (a + b) for a, b in zip(new, past)) * H * d > (4e9 if dtype == "f32" else 3e10):
        new = [max(1, a // 2) for a in new]
    return _paged("", "attend", H, Hk, d, new, past, dtype)


def _ints(text):
    return [int(t) for t in text.split()]


# ---- inputs ------------------------------------------------------------------------

def _td(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _rand(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _log_gates(g, T, H):
    """log f [T, H] = -softplus(-a), a ~ N(mu_h, 0.5), rounded from float64."""
    mu = torch.tensor([_mean(h, H) for h in range(H)], device="cuda", dtype=torch.float64)
    a = _rand(g, T, H).double() * 0.5 + mu
    return (-torch.nn.functional.softplus(-a)).float()


def _mean(h, H):
    return 1.0 + 9.0 * (h + 0.5) / H


def _qk_normed(g, rows, heads, d, weights, td):
    """Rows of N(0, 1) features, RMS-normalised (a little shorter, so that rounding keeps
    |row| <= gamma sqrt(d)) and scaled by the head's weights."""
    x = _rand(g, rows, heads, d)
    x *= torch.rsqrt((x * x).mean(dim=-1, keepdim=True)) * (1.0 - 2.0 ** -7)
    return (x * weights).to(td)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    make = {"norm": _prepare_norm, "rotary": _prepare_rotary, "append": _prepare_paged,
            "attend": _prepare_paged}[case["kind"]]
    return make(case, g)


def _prepare_norm(c, g):
    B, H, L, n = c["B"], c["H"], c["L"], c["n"]
    x = (_rand(g, B, L, H, n) if c["strided"] else _rand(g, B, H, L, n)) * 2.0 + 0.5
    x = x.to(_td(c))
    if c["strided"]:
        x = x.transpose(1, 2)
    shape = (H, n) if c["groups"] else (n,)
    s = {"c": c, "x": x, "w": 1.0 + 0.2 * _rand(g, *shape),
         "b": 0.1 * _rand(g, *shape) if c["center"] else None, "eps": 1e-5}
    if c["train"]:
        s["dy"] = _rand(g, B, H, L, n).to(_td(c))
    return s


_SCALING = {"none": {}, "linear": {"factor": 4.0}, "base": {"factor": 8.0},
            "ramp": {"factor": 32.0, "train_len": 4096}}


def _prepare_rotary(c, g):
    B, L = c["B"], c["L"]
    s = {"c": c}
    for n, heads in (("q", c["H"]), ("k", c["Hk"])):
        s[n] = _rand(g, B, heads, L, c["d"]).to(_td(c))
        if c["train"]:
            s["d" + n] = _rand(g, B, heads, L, c["d"]).to(_td(c))
    # every sequence at its own place
    first = torch.randint(0, 64, (B, 1), generator=g, device="cuda")
    s["pos"] = (first + torch.arange(c["start"], c["start"] + L, device="cuda")).to(torch.int32)
    if own:
        from paper_2504_06949_amd import ops
        s["rope"] = ops.Rotary(c["rot"], layout=c["layout"], scaling=c["scaling"],
                               **_SCALING[c["scaling"]])
    else:
        s["freq"], s["amp"] = _freqs(c)
        s["freq"] = s["freq"].cuda()
    return s


def _freqs(c):
    """Frequencies (radians per position, float64) and amplitude."""
    rot, p = c["rot"], _SCALING[c["scaling"]]
    base, s = 10000.0, p.get("factor", 1.0)
    if c["scaling"] == "base":
        base *= s ** (rot / (rot - 2))
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if c["scaling"] == "linear":
        return f / s, 1.0
    if c["scaling"] == "ramp":
        turns = p["train_len"] * f / (2.0 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return f * keep + f / s * (1.0 - keep), 0.1 * math.log(s) + 1.0
    return f, 1.0


def _prepare_paged(c, g):
    H, Hk, d, td = c["H"], c["Hk"], c["d"], _td(c)
    new, past = _ints(c["new"]), _ints(c["past"])
    N, T = len(new), sum(new)
    need = [(a + b + PAGE - 1) // PAGE for a, b in zip(new, past)]
    P, W = sum(need) + 3, max(need)
    order = torch.randperm(P, generator=g, device="cuda")
    table = torch.full((N, W), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, m in enumerate(need):
        table[i, :m] = order[at:at + m].int()
        at += m
    wq = torch.rand((H, d), generator=g, device="cuda") + 0.5
    wk = torch.rand((Hk, d), generator=g, device="cuda") + 0.5
    cu = torch.tensor([0] + np.cumsum(new).tolist(), dtype=torch.int32, device="cuda")
    s = {"c": c, "table": table, "cu": cu, "past": torch.tensor(past, dtype=torch.int32, device="cuda"),
         "new_list": new, "past_list": past}
    kp = _qk_normed(g, P * PAGE, Hk, d, wk, td).view(P, PAGE, Hk, d).transpose(1, 2).contiguous()
    vp = _rand(g, P, Hk, PAGE, d).to(td)
    cp = torch.zeros((P, H, PAGE), dtype=torch.float64, device="cuda")
    # the gates of what the pages hold already (attend: of the new tokens too)
    for i in range(N):
        held = past[i] + (new[i] if c["kind"] == "attend" else 0)
        m = (held + PAGE - 1) // PAGE
        if m:
            lf = _log_gates(g, m * PAGE, H).double()
            cp[table[i, :m].long()] = torch.cumsum(lf, 0).view(m, PAGE, H).transpose(1, 2)
    if c["kind"] == "append":
        s["k"] = _qk_normed(g, T, Hk, d, wk, td)
        s["v"] = _rand(g, T, Hk, d).to(td)
        s["lf"] = _log_gates(g, T, H)
    else:
        s["q"] = _qk_normed(g, T, H, d, wq, td)
        s["gq"], s["gk"] = wq.amax(-1).contiguous(), wk.amax(-1).contiguous()
    if own:
        from paper_2504_06949_amd import ops
        s["cache"] = ops.PagedCache(P, H, d, Hk, td)
        for name, t in s["cache"].views().items():
            t.copy_({"k": kp, "v": vp, "c": cp}[name])
    else:
        s["kp"], s["vp"], s["cp"] = kp, vp, cp
    return s


# ---- one pass ------------------------------------------------------------------------

def run(state):
    kind = state["c"]["kind"]
    if own:
        return {"norm": _own_norm, "rotary": _own_rotary, "append": _own_append,
                "attend": _own_attend}[kind](state)
    return {"norm": _plain_norm, "rotary": _plain_rotary, "append": _plain_append,
            "attend": _plain_attend}[kind](state)


def _own_norm(s):
    from paper_2504_06949_amd import ops
    center = s["c"]["center"]
    if not s["c"]["train"]:
        y, _, _ = ops.norm_forward(s["x"], s["w"], s["b"], s["eps"], center=center, stats=False)
        return y
    y, mean, rstd = ops.norm_forward(s["x"], s["w"], s["b"], s["eps"], center=center)
    dx, dw, db = ops.norm_backward(s["dy"], s["x"], s["w"], mean, rstd, bias=s["b"] is not None)
    return [y, dx, dw] + ([db] if center else [])


def _plain_norm(s):
    c, x = s["c"], s["x"].float()
    w, b = s["w"], s["b"]
    if c["groups"]:
        w, b = w[:, None, :], None if b is None else b[:, None, :]
    xc = x - x.mean(-1, keepdim=True) if c["center"] else x
    rstd = torch.rsqrt((xc * xc).mean(-1, keepdim=True) + s["eps"])
    xh = xc * rstd
    y = (xh * w if b is None else xh * w + b).to(_td(c))
    if not c["train"]:
        return y
    dy = s["dy"].float()
    gw = dy * w
    dx = gw - xh * (gw * xh).mean(-1, keepdim=True)
    if c["center"]:
        dx = dx - gw.mean(-1, keepdim=True)
    over = (0, 2) if c["groups"] else (0, 1, 2)
    out = [y, (dx * rstd).to(_td(c)), (dy * xh).sum(over)]
    return out + ([dy.sum(over)] if c["center"] else [])


def _own_rotary(s):
    q, k = s["rope"].forward(s["q"], s["k"], positions=s["pos"])
    if not s["c"]["train"]:
        return [q, k]
    dq, dk = s["rope"].backward(s["dq"], s["dk"], positions=s["pos"])
    return [q, k, dq, dk]


def _rotate(x, cos, sin, c):
    rot = c["rot"]
    out = x.clone()
    xf = x[..., :rot].float()
    if c["layout"] == "half":
        a, b = xf[..., :rot // 2], xf[..., rot // 2:]
        out[..., :rot // 2] = (a * cos - b * sin).to(x.dtype)
        out[..., rot // 2:rot] = (a * sin + b * cos).to(x.dtype)
    else:
        a, b = xf[..., 0::2], xf[..., 1::2]
        out[..., 0:rot:2] = (a * cos - b * sin).to(x.dtype)
        out[..., 1:rot:2] = (a * sin + b * cos).to(x.dtype)
    return out


def _plain_rotary(s):
    c = s["c"]
    angle = s["pos"].double()[:, None, :, None] * s["freq"]
    cos, sin = (angle.cos() * s["amp"]).float(), (angle.sin() * s["amp"]).float()
    out = [_rotate(s["q"], cos, sin, c), _rotate(s["k"], cos, sin, c)]
    if c["train"]:
        out += [_rotate(s["dq"], cos, -sin, c), _rotate(s["dk"], cos, -sin, c)]
    return out


def _own_append(s):
    cache = s["cache"]
    cache.append(s["k"], s["v"], s["lf"], s["cu"], s["past"], s["table"])
    v = cache.views()
    return [v["k"], v["v"], v["c"]]


def _plain_append(s):
    at = 0
    for i, (n, past) in enumerate(zip(s["new_list"], s["past_list"])):
        p = torch.arange(past, past + n, device="cuda")
        page, slot = s["table"][i].long()[p // PAGE], p % PAGE
        s["kp"][page, :, slot] = s["k"][at:at + n]
        s["vp"][page, :, slot] = s["v"][at:at + n]
        c = torch.cumsum(s["lf"][at:at + n].double(), 0)
        if past:
            c = c + s["cp"][s["table"][i, (past - 1) // PAGE].long(), :, (past - 1) % PAGE]
        s["cp"][page, :, slot] = c
        at += n
    return [s["kp"], s["vp"], s["cp"]]


def _own_attend(s):
    o, lse = s["cache"].attend(s["q"], s["cu"], s["past"], s["table"], max_new=max(s["new_list"]),
                               gamma_q=s["gq"], gamma_k=s["gk"], eps=EPS, L_max=L_MAX)
    return [o, lse]


def _delta(s, H, Hk, d):
    u = s["gq"].double() * s["gk"].double().repeat_interleave(H // Hk) * math.sqrt(d)
    return -(2.0 * u + (math.log(L_MAX) - math.log(EPS)))


def _plain_attend(s):
    c = s["c"]
    H, Hk, d = c["H"], c["Hk"], c["d"]
    G = H // Hk
    T = s["q"].shape[0]
    o = torch.empty((T, H, d), dtype=_td(c), device="cuda")
    lse = torch.empty((T, H), dtype=torch.float32, device="cuda")
    delta = _delta(s, H, Hk, d)
    at = 0
    for i, (n, past) in enumerate(zip(s["new_list"], s["past_list"])):
        m = (past + n + PAGE - 1) // PAGE
        pages = s["table"][i, :m].long()
        pos = torch.arange(past, past + n, device="cuda")
        key = torch.arange(past + n, device="cuda")
        later = key[None, :] > pos[:, None]
        same_page = (key // PAGE)[None, :] == (pos // PAGE)[:, None]
        for hk in range(Hk):
            k = s["kp"][pages, hk].reshape(m * PAGE, d)[:past + n].float()
            v = s["vp"][pages, hk].reshape(m * PAGE, d)[:past + n].float()
            for h in range(hk * G, (hk + 1) * G):
                cc = s["cp"][pages, h].reshape(-1)
                x = (s["q"][at:at + n, h].float() @ k.t()) * (1.0 / math.sqrt(d))
                ci, end = cc[pos], cc[PAGE - 1::PAGE].repeat_interleave(PAGE)[:past + n]
                x += (ci[:, None] - cc[None, :past + n]).float()
                gone = ((ci[:, None] - end[None, :]) < delta[h]) & ~same_page
                x.masked_fill_(later | gone, -math.inf)
                top = x.amax(-1, keepdim=True)
                p = torch.exp(x - top)
                total = p.sum(-1, keepdim=True)
                o[at:at + n, h] = ((p @ v) / total).to(o.dtype)
                lse[at:at + n, h] = (top + total.log())[:, 0]
        at += n
    return [o, lse]


# ---- work ----------------------------------------------------------------------------

def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "norm":
        rows = c["B"] * c["H"] * c["L"]
        e = rows * c["n"]
        weights = 4 * c["n"] * (c["H"] if c["groups"] else 1) * (2 if c["center"] else 1)
        b, f = 2 * e * es + weights, 6 * e
        if c["train"]:
            b, f = b + 3 * e * es + 2 * weights, f + 12 * e
        return {"bytes": b, "flops": f}
    if c["kind"] == "rotary":
        e = c["B"] * (c["H"] + c["Hk"]) * c["L"] * c["d"]
        r = c["B"] * (c["H"] + c["Hk"]) * c["L"] * c["rot"]
        k = 2 if c["train"] else 1
        return {"bytes": k * (2 * e * es + 4 * c["B"] * c["L"]), "flops": k * 3 * r}
    new, past = _ints(c["new"]), _ints(c["past"])
    T, H, Hk, d = sum(new), c["H"], c["Hk"], c["d"]
    if c["kind"] == "append":
        return {"bytes": 4 * T * Hk * d * es + 12 * T * H, "flops": T * H}
    # the kept window of a head reaches back until the gates' mean decay spends -delta
    bytes_, flops = 2 * T * H * d * es + 4 * T * H, 0
    bound = 2.0 * 1.5 * 1.5 * math.sqrt(d) + math.log(L_MAX) - math.log(EPS)
    z = np.linspace(-4.0, 4.0, 801)
    wz = np.exp(-0.5 * z * z)
    window = []
    for h in range(H):
        a = _mean(h, H) + 0.5 * z
        window.append(bound / float((wz * np.log1p(np.exp(-a))).sum() / wz.sum()))
    G = H // Hk
    for n, p in zip(new, past):
        for hk in range(Hk):
            bytes_ += 2 * d * es * min(p + n, max(window[hk * G:(hk + 1) * G]) + n)
        for h in range(H):
            w = window[h]
            bytes_ += 8 * min(p + n, w + n)
            i = np.arange(p + 1, p + n + 1, dtype=np.float64)
            flops += 4 * d * float(np.minimum(i, w).sum())
    return {"bytes": int(bytes_), "flops": int(flops)}


# ---- the definitions in 64 bits --------------------------------------------------------

def exact(case, seed):
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    return {"norm": _exact_norm, "rotary": _exact_rotary, "append": _exact_append,
            "attend": _exact_attend}[case["kind"]](case, s)


def _exact_norm(c, s):
    n = c["n"]
    heads = c["H"] if c["groups"] else 1
    w = s["w"].double().view(heads, n)
    x = s["x"].double()
    y, dx = torch.empty_like(x), torch.empty_like(x)
    y, dx = y.contiguous(), dx.contiguous()
    dw = torch.zeros((heads, n), dtype=torch.float64, device="cuda")
    db = torch.zeros_like(dw)
    for h in range(c["H"]):
        i = h if c["groups"] else 0
        xr = x[:, h].reshape(-1, n)
        mu = xr.sum(1) / n if c["center"] else torch.zeros(xr.shape[0], dtype=torch.float64, device="cuda")
        dev = xr - mu[:, None]
        sigma = (dev.square().sum(1) / n + s["eps"]).sqrt()
        z = dev / sigma[:, None]
        yr = z * w[i]
        if s["b"] is not None:
            yr = yr + s["b"].double().view(heads, n)[i]
        y[:, h] = yr.view(x[:, h].shape)
        if c["train"]:
            up = s["dy"][:, h].double().reshape(-1, n)
            dw[i] += (up * z).sum(0)
            db[i] += up.sum(0)
            dz = up * w[i]
            grad = dz - z * ((dz * z).sum(1) / n)[:, None]
            if c["center"]:
                grad = grad - (dz.sum(1) / n)[:, None]
            dx[:, h] = (grad / sigma[:, None]).view(x[:, h].shape)
    if not c["train"]:
        return y
    shape = s["w"].shape
    return [y, dx, dw.view(shape)] + ([db.view(shape)] if c["center"] else [])


def _exact_rotary(c, s):
    f, amp = _freqs(c)
    rot = c["rot"]
    z = torch.polar(torch.full_like(s["pos"].double()[..., None] * f.cuda(), amp),
                    s["pos"].double()[..., None] * f.cuda())[:, None]

    def turn(x, by):
        x = x.double()
        r = x[..., :rot]
        r = r.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if c["layout"] == "half" \
            else r.unflatten(-1, (rot // 2, 2))
        t = torch.view_as_real(torch.view_as_complex(r.contiguous()) * by)
        t = t.transpose(-1, -2) if c["layout"] == "half" else t
        return torch.cat([t.flatten(-2), x[..., rot:]], -1)

    out = [turn(s["q"], z), turn(s["k"], z)]
    if c["train"]:
        out += [turn(s["dq"], z.conj()), turn(s["dk"], z.conj())]
    return out


def _exact_append(c, s):
    table, lf = s["table"].cpu().numpy(), s["lf"].cpu().numpy()
    pages = s["cp"].cpu().numpy().copy()
    at = 0
    for i, (n, past) in enumerate(zip(s["new_list"], s["past_list"])):
        run_sum = np.cumsum(lf[at:at + n].astype(np.longdouble), axis=0)
        if past:
            run_sum = run_sum + pages[table[i, (past - 1) // PAGE], :, (past - 1) % PAGE]
        p = np.arange(past, past + n)
        pages[table[i, p // PAGE], :, p % PAGE] = run_sum.astype(np.float64)
        at += n
    return [None, None, torch.from_numpy(pages).cuda()]


def _exact_attend(c, s):
    H, Hk, d = c["H"], c["Hk"], c["d"]
    if sum(a * (a + b) for a, b in zip(s["new_list"], s["past_list"])) * H * d > 1e12:
        return None
    T = s["q"].shape[0]
    o = torch.empty((T, H, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((T, H), dtype=torch.float64, device="cuda")
    table = s["table"].long()
    log_share = math.log(EPS / L_MAX)
    at = 0
    for i, (n, past) in enumerate(zip(s["new_list"], s["past_list"])):
        end = past + n
        j = torch.arange(end, device="cuda")
        page, slot = table[i, j // PAGE], j % PAGE
        for h in range(H):
            hk = h // (H // Hk)
            bound = float(s["gq"][h].double() * s["gk"][hk].double()) * math.sqrt(d)
            least = log_share - 2.0 * bound
            keys, vals = s["kp"][page, hk, slot].double(), s["vp"][page, hk, slot].double()
            decay = s["cp"][page, h, slot]
            # rows in pieces, so that a piece's weights stay near a gigabyte
            for r0 in range(0, n, max(1, 100000000 // end)):
                r1 = min(n, r0 + max(1, 100000000 // end))
                rows = torch.arange(past + r0, past + r1, device="cuda")
                # the last position of a key's page, or the row itself on its own page
                last = torch.minimum((j // PAGE) * PAGE + PAGE - 1, rows[:, None])
                seen = (j <= rows[:, None]) & ((last // PAGE == rows[:, None] // PAGE)
                                               | (decay[rows][:, None] - decay[last] >= least))
                logits = s["q"][at + r0:at + r1, h].double() @ keys.t() / math.sqrt(d)
                logits = logits + (decay[rows][:, None] - decay[None, :])
                logits = torch.where(seen, logits, -math.inf)
                lse[at + r0:at + r1, h] = torch.logsumexp(logits, 1)
                o[at + r0:at + r1, h] = torch.exp(logits - lse[at + r0:at + r1, h, None]) @ vals
        at += n
    return [o, lse]
