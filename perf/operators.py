"""Operators of an attention layer over packed documents, as cases that can be timed and compared: attention in which every
query sees a range of the keys, rotary positions, and layer norm.

A case is one pass as a program makes it: the forward pass alone where it answers, forward and backward where it trains.
Documents are given by their lengths, packed one behind the other; geometries are those of the repository's workloads and
tests, with fewer key heads where a case says so.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

ATTENTION = dict(op="attention", dtype="bf16", heads=16, kv_heads=16, width=128, q_lens="", k_lens="", causal=True, window=0, prefix="",
                 cap=0.0, bias=False, train=False)
ROTARY = dict(op="rotary", dtype="bf16", heads=16, width=128, dims=128, interleaved=False, lens="", start=0, scaling="none", factor=1.0,
              original=0, transposed=False, inside=0)
NORM = dict(op="norm", dtype="bf16", rows=0, cols=0, train=False)


def listed():
    return [
        # the next token of eight chats: one query each, keys of a few hundred tokens; latency
        dict(ATTENTION, name="attention_next_token", heads=16, kv_heads=4, q_lens="1,1,1,1,1,1,1,1", k_lens="212,37,1001,450,1,777,128,1500"),
        # the next token of a few long documents: reading the keys and values bounds it
        dict(ATTENTION, name="attention_next_token_long", heads=32, kv_heads=8, q_lens="1,1,1,1,1", k_lens="32768,9001,20480,513,30011"),
        # a prompt behind what its sequence holds already, prefix seen from everywhere, distance bias, heads 64 wide
        dict(ATTENTION, name="attention_prompts", heads=12, kv_heads=12, width=64, q_lens="611,300,1200", k_lens="2011,300,1703", prefix="128,17,0",
             bias=True),
        # the headline batch's tokens as packed documents of a chat data set, a training step
        dict(ATTENTION, name="attention_packed_step", q_lens="517,33,1,730,211,299,257", train=True),
        # half a block's heads share keys, capped scores, a window: a training step of odd length
        dict(ATTENTION, name="attention_capped_window_step", heads=16, kv_heads=8, width=64, q_lens="3001,1094", window=1024, cap=50.0, train=True),
        # one document of the longest sequence of the benchmark, four query heads to a key head
        dict(ATTENTION, name="attention_long_step", kv_heads=4, q_lens="8192", train=True),
        # float32, to check a run's gradients: two documents, distance bias
        dict(ATTENTION, name="attention_f32_step", dtype="f32", heads=4, kv_heads=2, width=64, q_lens="301,450", bias=True, train=True),
        # queries of a handful of new tokens, far along in their sequences; latency
        dict(ROTARY, name="rotary_next_tokens", heads=20, lens="1,1,1,1,1,1,1,1", start=30000, inside=24),
        # queries and keys of a packed batch in one call, in place in the rows of a fused projection, scaled to a longer context
        dict(ROTARY, name="rotary_packed", heads=40, lens="5000,2101,1090,1", scaling="wavelength", factor=8.0, original=8192, inside=48),
        # gradient at the rotation of half of each head, pairs side by side, float32
        dict(ROTARY, name="rotary_partial_grad_f32", dtype="f32", heads=32, dims=64, interleaved=True, lens="2048,2048", transposed=True),
        # a prompt of the model twice as wide as the headline's
        dict(NORM, name="norm_prompt", rows=611, cols=4096),
        # a training batch, gradients of gain and bias among the results
        dict(NORM, name="norm_step", rows=8192, cols=2048, train=True),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _lengths(rng, total, most):
    lens = []
    while total > 0 and len(lens) < most - 1:
        n = min(total, _spread(rng, 1, total))
        lens.append(n)
        total -= n
    if total > 0:
        lens.append(total)
    rng.shuffle(lens)
    return lens


def _text(lens):
    return ",".join(str(n) for n in lens)


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "rotary", "norm"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "rotary":
        width = rng.choice([32, 64, 80, 128])
        heads = rng.choice([4, 5, 12, 20, 40])
        return dict(ROTARY, dtype=dtype, heads=heads, width=width, dims=rng.choice([width, width // 2]), interleaved=rng.random() < 0.5,
                    lens=_text(_lengths(rng, _spread(rng, 1, 8192), 6)), start=_spread(rng, 1, 100000), scaling=rng.choice(["none", "linear", "base", "wavelength"]),
                    factor=rng.choice([2.0, 8.0]), original=4096, transposed=rng.random() < 0.5, inside=rng.choice([0, heads + 3]))
    if op == "norm":
        rows, cols = _spread(rng, 1, 8192), _spread(rng, 64, 4096)
        return dict(NORM, dtype=dtype, rows=rows, cols=cols - cols % 8 if rng.random() < 0.7 else cols, train=rng.random() < 0.6)
    group, kv_heads, width = rng.choice([1, 2, 4]), rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
    case = dict(ATTENTION, dtype=dtype, heads=group * kv_heads, kv_heads=kv_heads, width=width, cap=rng.choice([0.0, 0.0, 30.0]), bias=rng.random() < 0.3)
    kind = rng.choice(["next", "prompt", "train", "train"])
    if kind == "next":
        lens = [_spread(rng, 1, 16384) for _ in range(rng.randint(1, 9))]
        return dict(case, q_lens=_text([1] * len(lens)), k_lens=_text(lens))
    lens = _lengths(rng, _spread(rng, 16, 2048 if dtype == "f32" else 5000), 7)
    if kind == "prompt":
        before = [_spread(rng, 1, 600) - 1 for _ in lens]
        return dict(case, q_lens=_text(lens), k_lens=_text([a + b for a, b in zip(lens, before)]), prefix=_text([_spread(rng, 1, 300) - 1 for _ in lens]))
    return dict(case, q_lens=_text(lens), causal=rng.random() < 0.8, train=True)


def _lens(text):
    return [int(n) for n in text.split(",")] if text else []


def _ranges(case):
    """First and one past the last key row that each query row sees, and the key row at which it stands (numpy int64)."""
    q_lens = _lens(case["q_lens"])
    k_lens = _lens(case["k_lens"]) or q_lens
    prefix = _lens(case["prefix"]) or [0] * len(q_lens)
    lo, hi, at, k0 = [], [], [], 0
    for nq, nk, np_ in zip(q_lens, k_lens, prefix):
        a = k0 + nk - nq + np.arange(nq)
        first, end = np.full(nq, k0), np.full(nq, k0 + nk)
        if case["causal"]:
            end = np.maximum(a + 1, min(k0 + np_, k0 + nk))
            if case["window"]:
                first = np.maximum(first, a + 1 - case["window"])
        lo.append(first), hi.append(end), at.append(a)
        k0 += nk
    return np.concatenate(lo), np.concatenate(hi), np.concatenate(at), k0


def _slopes(heads):
    return 2.0 ** (-8.0 * (np.arange(heads) + 1) / heads)


def _frequencies(case):
    """Angle per position of each pair, in 64 bits."""
    dims, theta = case["dims"], 10000.0
    if case["scaling"] == "base":
        theta *= case["factor"] ** (dims / (dims - 2))
    f = theta ** (-2.0 * np.arange(dims // 2) / dims)
    if case["scaling"] == "linear":
        f = f / case["factor"]
    if case["scaling"] == "wavelength":
        share = np.clip((case["original"] * f / (2 * math.pi) - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        f = share * f + (1 - share) * f / case["factor"]
    return f


def _magnitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "wavelength" else 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    dt = TYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    ints = lambda a: torch.from_numpy(np.asarray(a)).to("cuda", torch.int32)
    st = dict(case)
    if case["op"] == "attention":
        lo, hi, at, keys = _ranges(case)
        n, H, Hkv, dh = len(lo), case["heads"], case["kv_heads"], case["width"]
        st["q"], st["k"], st["v"] = normal(n, H, dh).to(dt), normal(keys, Hkv, dh).to(dt), normal(keys, Hkv, dh).to(dt)
        q_lens = _lens(case["q_lens"])
        st["cu_q"] = ints(np.cumsum([0] + q_lens))
        st["cu_k"] = ints(np.cumsum([0] + (_lens(case["k_lens"]) or q_lens)))
        st["pre"] = ints(_lens(case["prefix"])) if case["prefix"] else None
        st["slopes"] = torch.from_numpy(_slopes(H)).to("cuda", torch.float32) if case["bias"] else None
        st["lo"], st["hi"], st["at"] = ints(lo), ints(hi), ints(at)
        st["used"] = ints([n, keys])
        st["o"], st["lse"] = torch.empty_like(st["q"]), torch.empty(H, n, dtype=torch.float32, device="cuda")
        if case["train"]:
            st["do"] = normal(n, H, dh).to(dt)
            st["dq"], st["dk"], st["dv"] = torch.empty_like(st["q"]), torch.empty_like(st["k"]), torch.empty_like(st["v"])
    elif case["op"] == "rotary":
        pos = np.concatenate([case["start"] + np.arange(n) for n in _lens(case["lens"])])
        wide = case["inside"] or case["heads"]
        st["rows"] = normal(len(pos), wide, case["width"]).to(dt)          # a projection's rows, of which the first heads are rotated
        st["x"] = st["rows"][:, : case["heads"]]
        st["y"] = torch.empty(len(pos), case["heads"], case["width"], dtype=dt, device="cuda")
        st["pos"] = ints(pos)
        st["freq"] = torch.from_numpy(_frequencies(case)).cuda()
    else:
        rows, cols = case["rows"], case["cols"]
        st["x"] = (normal(rows, cols) * 1.5 + 0.4 * normal(cols)).to(dt)
        st["gain"], st["bias"] = (1 + 0.1 * normal(cols)).to(dt), (0.1 * normal(cols)).to(dt)
        st["y"] = torch.empty_like(st["x"])
        st["mean"], st["rstd"] = torch.empty(rows, dtype=torch.float32, device="cuda"), torch.empty(rows, dtype=torch.float32, device="cuda")
        if case["train"]:
            st["dy"] = normal(rows, cols).to(dt)
            st["dx"], st["dgain"], st["dbias"] = torch.empty_like(st["x"]), torch.empty_like(st["gain"]), torch.empty_like(st["bias"])
    if own:
        _plan(st)
    return st


def _plan(st):
    """What the program keeps from call to call: descriptors and workspaces."""
    import paper_2512_20920_amd as R
    st["dt"] = 1 if st["dtype"] == "bf16" else 0
    if st["op"] == "attention":
        st["desc"] = R.AttnDesc(dtype=st["dt"], H=st["heads"], Hkv=st["kv_heads"], dh=st["width"], Tq=st["q"].shape[0], Tk=st["k"].shape[0],
                                softcap=st["cap"], slopes=st["slopes"])
        st["mask"] = R.AttnMask(lo=st["lo"], hi=st["hi"], at=st["at"], used=st["used"])
        size = R.revffn_op_attention_masked_workspace(st["desc"], st["train"])
        st["work"] = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
    elif st["op"] == "rotary":
        st["rotary"] = R.Rotary(dims=st["dims"], interleaved=st["interleaved"], theta=10000.0,
                                scaling=("none", "linear", "base", "wavelength").index(st["scaling"]), factor=st["factor"], original=st["original"],
                                few_turns=1.0, many_turns=32.0, magnitude=_magnitude(st))
    elif st["train"]:
        st["work"] = torch.empty(max(R.revffn_op_layernorm_workspace(st["rows"], st["cols"]), 16), dtype=torch.uint8, device="cuda")


def run(st):
    return {"attention": _attention, "rotary": _rotary, "norm": _norm}[st["op"]](st)


def _attention(st):
    if own:
        import paper_2512_20920_amd as R
        if st["train"]:          # a batch's ranges are made from its documents once; here with every pass
            R.revffn_op_attention_ranges(st["cu_q"], None, st["pre"], st["cu_q"].numel() - 1, st["causal"], st["window"], st["desc"].Tq, st["desc"].Tk,
                                         st["lo"], st["hi"], st["at"], st["used"])
        R.revffn_op_attention_masked_fwd(st["desc"], st["mask"], st["q"], st["k"], st["v"], st["o"], st["lse"], st["work"])
        if not st["train"]:
            return st["o"], st["lse"]
        R.revffn_op_attention_masked_bwd(st["desc"], st["mask"], st["q"], st["k"], st["v"], st["o"], st["do"], st["lse"], st["dq"], st["dk"], st["dv"],
                                         st["work"])
        return st["o"], st["lse"], st["dq"], st["dk"], st["dv"]
    H, Hkv, dh = st["heads"], st["kv_heads"], st["width"]
    G, n, scale = H // Hkv, st["q"].shape[0], 1.0 / math.sqrt(dh)
    by_head = lambda t, h: t.float().permute(1, 0, 2).reshape(Hkv, h, -1, dh).contiguous()      # [key head, query head of it, row, column]
    back = lambda t: t.reshape(-1, t.shape[2], dh).permute(1, 0, 2).contiguous()
    q, k, v = by_head(st["q"], G), by_head(st["k"], 1), by_head(st["v"], 1)
    j = torch.arange(k.shape[2], device="cuda")
    sees = (j >= st["lo"][:, None]) & (j < st["hi"][:, None])
    s = torch.matmul(q.reshape(Hkv, G * n, dh), k[:, 0].transpose(1, 2).contiguous()).reshape(Hkv, G, n, -1) * scale
    if st["cap"]:
        t = torch.tanh(s / st["cap"])
        s = t * st["cap"]
    if st["bias"]:
        s = s - st["slopes"].reshape(Hkv, G, 1, 1) * (st["at"][:, None] - j).abs().float()
    s = torch.where(sees, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    lse = (torch.log(total) + top).reshape(H, n)
    p = p / torch.where(total == 0, 1.0, total)
    pair = lambda a, b: torch.matmul(a.reshape(Hkv, G * n, -1), b[:, 0]).reshape(Hkv, G, n, -1)
    o = pair(p, v)
    if not st["train"]:
        return back(o).to(st["q"].dtype), lse
    do = by_head(st["do"], G)
    dp = pair(do, v.transpose(2, 3).contiguous())
    ds = p * (dp - (o * do).sum(-1, keepdim=True))
    if st["cap"]:
        ds = ds * (1 - t * t)
    over = lambda a, b: torch.matmul(a.reshape(Hkv, G * n, -1).transpose(1, 2).contiguous(), b.reshape(Hkv, G * n, dh))
    dq, dk, dv = pair(ds, k) * scale, over(ds, q)[:, None] * scale, over(p, do)[:, None]
    dt = st["q"].dtype
    return back(o).to(dt), lse, back(dq).to(dt), back(dk).to(dt), back(dv).to(dt)


def _rotary(st):
    T, H, dh, dims = st["x"].shape[0], st["heads"], st["width"], st["dims"]
    if own:
        import paper_2512_20920_amd as R
        R.revffn_op_rotary(st["dt"], st["rotary"], st["x"], st["y"], st["pos"], T, T, H, dh, st["x"].stride(0), H * dh, st["transposed"])
        return st["y"]
    x = st["x"].float()
    a = st["pos"].double()[:, None] * st["freq"]                          # far positions: the angle in 64 bits
    c = (torch.cos(a) * _magnitude(st)).float()[:, None, :]
    s = (torch.sin(a) * (_magnitude(st) * (-1 if st["transposed"] else 1))).float()[:, None, :]
    y = x.clone()
    if st["interleaved"]:
        u, w = x[..., 0:dims:2], x[..., 1:dims:2]
        y[..., 0:dims:2], y[..., 1:dims:2] = u * c - w * s, u * s + w * c
    else:
        u, w = x[..., : dims // 2], x[..., dims // 2 : dims]
        y[..., : dims // 2], y[..., dims // 2 : dims] = u * c - w * s, u * s + w * c
    return y.to(st["x"].dtype)


EPS = 1e-5


def _norm(st):
    rows, cols = st["rows"], st["cols"]
    if own:
        import paper_2512_20920_amd as R
        R.revffn_op_layernorm_fwd(st["dt"], st["x"], st["gain"], st["bias"], st["y"], st["mean"], st["rstd"], rows, cols, cols, cols, EPS)
        if not st["train"]:
            return st["y"], st["mean"], st["rstd"]
        R.revffn_op_layernorm_bwd(st["dt"], st["dy"], st["x"], st["gain"], st["mean"], st["rstd"], st["dx"], st["dgain"], st["dbias"], rows, cols,
                                  cols, cols, cols, False, st["work"])
        return st["y"], st["mean"], st["rstd"], st["dx"], st["dgain"], st["dbias"]
    x, dt = st["x"].float(), st["x"].dtype
    gain, bias = st["gain"].float(), st["bias"].float()
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)
    xh = (x - mean) * rstd
    y = (xh * gain + bias).to(dt)
    if not st["train"]:
        return y, mean[:, 0], rstd[:, 0]
    dy = st["dy"].float()
    d = dy * gain
    dx = rstd * (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True))
    return y, mean[:, 0], rstd[:, 0], dx.to(dt), (dy * xh).sum(0).to(dt), dy.sum(0).to(dt)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "attention":
        lo, hi, _, keys = _ranges(case)
        pairs, n, H, Hkv, dh = int((hi - lo).sum()), len(lo), case["heads"], case["kv_heads"], case["width"]
        forward = size * dh * (2 * n * H + 2 * keys * Hkv) + 4 * n * H
        if not case["train"]:
            return {"bytes": forward, "flops": 4 * pairs * dh * H}
        return {"bytes": forward + size * dh * (2 * n * H + 2 * keys * Hkv), "flops": 14 * pairs * dh * H}
    if case["op"] == "rotary":
        n = sum(_lens(case["lens"]))
        return {"bytes": 2 * size * n * case["heads"] * case["width"] + 4 * n, "flops": 3 * n * case["heads"] * case["dims"]}
    values = case["rows"] * case["cols"]
    params = size * case["cols"]
    if not case["train"]:
        return {"bytes": 2 * size * values + 2 * params + 8 * case["rows"], "flops": 7 * values}
    return {"bytes": 4 * size * values + 4 * params + 8 * case["rows"], "flops": 20 * values}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attention":
        return _exact_attention(case, st)
    if case["op"] == "rotary":
        x, dims = st["x"].double(), case["dims"]
        turn = torch.polar(torch.full_like(st["freq"], _magnitude(case)).expand(x.shape[0], -1).contiguous(),
                           st["pos"].double()[:, None] * st["freq"] * (-1 if case["transposed"] else 1))[:, None, :]
        part = x[..., :dims]
        if case["interleaved"]:
            z = torch.complex(part[..., 0::2].contiguous(), part[..., 1::2].contiguous()) * turn
            part = torch.stack([z.real, z.imag], -1).flatten(-2)
        else:
            z = torch.complex(part[..., : dims // 2].contiguous(), part[..., dims // 2 :].contiguous()) * turn
            part = torch.cat([z.real, z.imag], -1)
        return torch.cat([part, x[..., dims:]], -1)
    x = st["x"].double().requires_grad_(case["train"])
    gain, bias = st["gain"].double().requires_grad_(case["train"]), st["bias"].double().requires_grad_(case["train"])
    mean = x.sum(1) / case["cols"]
    var = ((x - mean[:, None]) ** 2).sum(1) / case["cols"]
    rstd = (var + EPS) ** -0.5
    y = (x - mean[:, None]) * rstd[:, None] * gain + bias
    if not case["train"]:
        return y, mean, rstd
    grads = torch.autograd.grad(y, (x, gain, bias), st["dy"].double())
    return (y.detach(), mean.detach(), rstd.detach()) + grads


def _exact_attention(case, st):
    lo, hi, at, keys = _ranges(case)
    H, Hkv, dh, train = case["heads"], case["kv_heads"], case["width"], case["train"]
    if keys * len(lo) * H * dh * (14 if train else 4) > 3e12:
        return None
    j = np.arange(keys)
    hidden = torch.from_numpy((j[None, :] < lo[:, None]) | (j[None, :] >= hi[:, None])).cuda()
    apart = torch.from_numpy(np.abs(at[:, None] - j[None, :])).cuda().double()
    o, lse = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda"), torch.empty(H, len(lo), dtype=torch.float64, device="cuda")
    dq = torch.empty_like(o)
    dk, dv = torch.zeros(st["k"].shape, dtype=torch.float64, device="cuda"), torch.zeros(st["v"].shape, dtype=torch.float64, device="cuda")
    slopes = _slopes(H).astype(np.float32).astype(np.float64)
    for h in range(H):
        q = st["q"][:, h].double().requires_grad_(train)
        k, v = st["k"][:, h * Hkv // H].double().requires_grad_(train), st["v"][:, h * Hkv // H].double().requires_grad_(train)
        s = q @ k.t() / math.sqrt(dh)
        if case["cap"]:
            s = torch.tanh(s / case["cap"]) * case["cap"]
        if case["bias"]:
            s = s - float(slopes[h]) * apart
        s = s.masked_fill(hidden, -math.inf)
        norm = torch.logsumexp(s, 1)
        out = torch.exp(s - norm[:, None]) @ v
        o[:, h], lse[h] = out.detach(), norm.detach()
        if train:
            a, b, c = torch.autograd.grad(out, (q, k, v), st["do"][:, h].double())
            dq[:, h] = a
            dk[:, h * Hkv // H] += b
            dv[:, h * Hkv // H] += c
    return (o, lse, dq, dk, dv) if train else (o, lse)
