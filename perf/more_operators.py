"""Operators of an attention layer that answers in 8 bits, as cases that can be timed and compared: new keys and values appended to a paged
cache (rotated on the way), attention over that cache, and projections as products of 8-bit integers.

A case is one call of a serving step's layer.  Sequences are given by the tokens that they hold after the step and by how many of
those are new; widths and heads are those of the repository's workloads and tests, with fewer key heads where a case says so.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CODES = torch.float8_e4m3fn

APPEND = dict(op="append", dtype="bf16", heads=16, kv_heads=16, width=128, page=64, held="", new="", dims=128, interleaved=False)
ATTENTION = dict(op="attention", dtype="bf16", heads=16, kv_heads=16, width=128, page=64, held="", new="", window=0, cap=0.0)
PRODUCT = dict(op="product", dtype="bf16", rows=0, inner=0, outer=0, bias=False)


def listed():
    return [
        # the next tokens of eight chats; latency
        dict(APPEND, name="append_next_tokens", kv_heads=4, held="212,37,1001,450,1,777,128,1500", new="1,1,1,1,1,1,1,1"),
        # a scheduler's mixed step, small pages: prompts behind what is held already and single tokens
        dict(APPEND, name="append_mixed", heads=32, kv_heads=8, width=64, dims=64, page=16, held="611,2011,301,1703,9,4096", new="611,300,1,1200,1,1"),
        # a long prompt into an empty cache
        dict(APPEND, name="append_long_prompt", heads=32, kv_heads=8, held="8192", new="8192"),
        # the next tokens of eight chats; latency
        dict(ATTENTION, name="attention_next_tokens", kv_heads=4, held="212,37,1001,450,1,777,128,1500", new="1,1,1,1,1,1,1,1"),
        # the next tokens of long documents: reading the cache bounds it
        dict(ATTENTION, name="attention_next_tokens_long", heads=32, kv_heads=8, page=32, new="1,1,1,1,1,1,1,1,1,1,1,1",
             held="32768,9001,20480,513,30011,16384,25000,7777,31999,12345,28672,4097"),
        # a scheduler's mixed step, heads 64 wide, capped scores, a window
        dict(ATTENTION, name="attention_mixed", heads=32, kv_heads=8, width=64, page=16, held="611,2011,301,1703,9,4096", new="611,300,1,1200,1,1",
             window=1024, cap=50.0),
        # a long prompt's last piece, behind what it holds already
        dict(ATTENTION, name="attention_prompt_piece", heads=32, kv_heads=8, held="8192", new="4096"),
        # float32, to check a run's answers
        dict(ATTENTION, name="attention_f32", dtype="f32", heads=8, kv_heads=2, width=64, page=32, held="301,450,1000", new="301,1,250"),
        # projections of the next tokens of eight chats: reading the weights bounds it
        dict(PRODUCT, name="product_next_tokens", rows=8, inner=2048, outer=6144, bias=True),
        # a prompt of odd length through the gate and up projections of the headline's shared expert
        dict(PRODUCT, name="product_prompt", rows=611, inner=2048, outer=11264),
        # a training-sized batch through the wide geometry's expert, the largest
        dict(PRODUCT, name="product_batch", rows=8192, inner=4096, outer=14336),
        # float32 activations, odd sizes
        dict(PRODUCT, name="product_odd_f32", dtype="f32", rows=333, inner=1001, outer=999, bias=True),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _text(lens):
    return ",".join(str(n) for n in lens)


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "attention", "product", "product"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "product":
        rows = _spread(rng, 1, 8192)
        inner, outer = _spread(rng, 64, 4096), _spread(rng, 64, 11264)
        if rng.random() < 0.7:
            inner, outer = inner - inner % 64 or 64, outer - outer % 8
        return dict(PRODUCT, dtype=dtype, rows=rows, inner=inner, outer=outer, bias=rng.random() < 0.5)
    group, kv_heads, width = rng.choice([1, 2, 4, 7]), rng.choice([1, 2, 4, 8]), rng.choice([64, 64, 80, 128, 128, 128])
    case = dict(dtype=dtype, heads=group * kv_heads, kv_heads=kv_heads, width=width, page=rng.choice([16, 32, 64, 128]))
    kind = rng.choice(["next", "prompt", "mixed"])
    if kind == "next":
        held = [_spread(rng, 1, 16384) for _ in range(_spread(rng, 1, 24))]
        new = [1] * len(held)
    elif kind == "prompt":
        new = [_spread(rng, 2, 2048)]
        held = [new[0] + _spread(rng, 1, 4096) - 1]
    else:
        new = [_spread(rng, 1, 700) for _ in range(rng.randint(2, 6))]
        held = [n + _spread(rng, 1, 2000) - 1 for n in new]
    case.update(held=_text(held), new=_text(new))
    if op == "append":
        return dict(APPEND, **case, dims=rng.choice([width, width // 16 // 2 * 16]), interleaved=rng.random() < 0.5)
    return dict(ATTENTION, **case, window=rng.choice([0, 0, 0, 512]), cap=rng.choice([0.0, 0.0, 30.0]))


def _lens(text):
    return [int(n) for n in text.split(",")]


THETA = 10000.0


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 29)
    dt = TYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    st = dict(case)
    if case["op"] == "product":
        M, N, K = case["rows"], case["outer"], case["inner"]
        st["x"] = (normal(M, K) * (1 + 7 * (normal(K) > 2.3))).to(dt)               # activations, a few columns of which are large
        w = normal(N, K) * 0.02
        st["wscale"] = w.abs().amax(1) / 127.0
        ld = (K + 15) // 16 * 16                                                   # weights are laid out once, rows at multiples of 16 bytes
        st["w"] = torch.zeros(N, ld, dtype=torch.int8, device="cuda")
        st["w"][:, :K] = torch.round(w / st["wscale"][:, None]).to(torch.int8)
        st["bias"] = (0.1 * normal(N)).to(dt) if case["bias"] else None
        st["codes"], st["scale"] = torch.empty(M, ld, dtype=torch.int8, device="cuda"), torch.empty(M, dtype=torch.float32, device="cuda")
        st["y"] = torch.empty(M, N, dtype=dt, device="cuda")
        return st
    held, new, P, H, Hkv, dh = _lens(case["held"]), _lens(case["new"]), case["page"], case["heads"], case["kv_heads"], case["width"]
    S, T = len(held), sum(new)
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", torch.int32)
    longs = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", torch.int64)
    # a pool of pages, of which the sequences hold some, in no order
    need = [-(-n // P) for n in held]
    pages = sum(need) + sum(need) // 8 + 2
    order = np.random.default_rng(seed + 5).permutation(pages)
    table = np.full((S, max(need)), -1)
    for s in range(S):
        table[s, : need[s]] = order[sum(need[:s]) : sum(need[: s + 1])]
    st["table"], st["held"], st["cu"] = ints(table), ints(held), ints(np.cumsum([0] + new))
    column = 1 + 5 * (normal(dh) > 1.8)                                           # keys have a few large columns
    k, v = normal(pages, Hkv, P, dh) * column, normal(pages, Hkv, P // 16, dh, 16)
    for name, x in (("k", k), ("v", v)):
        top = x.abs().flatten(2).amax(2)
        scale = torch.exp2(torch.ceil(torch.log2(top / 448.0)))
        st[name + "_scale"] = scale
        st[name + "_codes"] = (x / scale.reshape([pages, Hkv] + [1] * (x.dim() - 2))).to(CODES)
    # the projection's rows: queries, keys and values side by side
    size = torch.exp2(normal(T, 1, 1).round() * 0.5)                              # later tokens may be larger than those that are held
    rows = torch.cat([normal(T, H, dh), normal(T, Hkv, dh) * column * size, normal(T, Hkv, dh) * size], 1)
    st["rows"] = rows.to(dt)
    st["q"], st["key"], st["value"] = st["rows"][:, :H], st["rows"][:, H : H + Hkv], st["rows"][:, H + Hkv :]
    seq = np.repeat(np.arange(S), new)
    at = np.concatenate([h - n + np.arange(n) for h, n in zip(held, new)])         # where the new rows stand
    # the same as a program that pads would keep it: the rows of each sequence, and the pages that the step writes to
    pad = np.zeros((S, max(new)), int)
    place = np.concatenate([np.arange(n) for n in new])
    pad[seq, place] = np.arange(T)
    st["pad"], st["seq"], st["place"], st["at"] = longs(pad), longs(seq), longs(place), longs(at)
    if case["op"] == "append":
        visits = [(s, p) for s in range(S) for p in range((held[s] - new[s]) // P, need[s])]
        first = {v: i for i, v in enumerate(visits)}
        st["visited"] = longs([table[v] for v in visits])
        st["below"] = longs([max(held[s] - new[s] - p * P, 0) for s, p in visits])  # rows of the page that were there before
        st["visit"] = longs([first[s, a // P] for s, a in zip(seq, at)])
        st["turned"] = torch.empty(T, H, dh, dtype=dt, device="cuda")
        st["pos"] = ints(at)
    else:
        st["o"], st["lse"] = torch.empty(T, H, dh, dtype=dt, device="cuda"), torch.empty(H, T, dtype=torch.float32, device="cuda")
    if own:
        _plan(st)
    return st


def _plan(st):
    """What the program keeps from call to call: descriptors and workspaces."""
    import paper_2512_20920_amd as R
    S, most = st["table"].shape
    st["cache"] = R.Cache(st["k_codes"], st["v_codes"], st["k_scale"], st["v_scale"], st["table"], st["held"], st["cu"], pages=st["k_codes"].shape[0],
                          page=st["page"], max_pages=most, n_seqs=S, Hkv=st["kv_heads"], dh=st["width"])
    if st["op"] == "append":
        st["rotary"] = R.Rotary(dims=st["dims"], interleaved=st["interleaved"], theta=THETA)
    else:
        st["desc"] = R.AttnDesc(dtype=1 if st["dtype"] == "bf16" else 0, H=st["heads"], Hkv=st["kv_heads"], dh=st["width"], Tq=st["q"].shape[0],
                                ldq=st["rows"].stride(0), softcap=st["cap"])
        st["work"] = torch.empty(max(R.revffn_op_attention_cached_workspace(st["desc"], st["cache"]), 16), dtype=torch.uint8, device="cuda")


def run(st):
    return {"append": _append, "attention": _attention, "product": _product}[st["op"]](st)


def _need(top):
    """The least power of two that brings values up to `top` within what an 8-bit number holds (448)."""
    part, power = torch.frexp(top)
    return torch.ldexp(torch.ones_like(top), torch.where(top == 0, -96, torch.where(part <= 0.875, power - 9, power - 8)).clamp(-96, 119))


def _turn(x, at, dims, interleaved):
    """Rotary positions; the angle in 64 bits, as positions may be far."""
    f = THETA ** (-2.0 * torch.arange(dims // 2, device="cuda", dtype=torch.float64) / dims)
    a = at.double()[:, None] * f
    c, s = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]
    y = x.float().clone()
    one, two = (slice(0, dims, 2), slice(1, dims, 2)) if interleaved else (slice(0, dims // 2), slice(dims // 2, dims))
    u, w = x[..., one].float(), x[..., two].float()
    y[..., one], y[..., two] = u * c - w * s, u * s + w * c
    return y.to(x.dtype)


def _append(st):
    """The turned queries and the cache: its numbers of 8 bits, each in units of its page's and head's scale, and those scales."""
    H, Hkv, dh, P = st["heads"], st["kv_heads"], st["width"], st["page"]
    if own:
        import paper_2512_20920_amd as R
        wide = st["rows"].stride(0)
        R.revffn_op_cache_append(1 if st["dtype"] == "bf16" else 0, st["cache"], st["rotary"], st["pos"], st["q"], st["turned"], st["key"], st["value"],
                                 st["q"].shape[0], H, wide, H * dh, wide, wide)
        return st["turned"], st["k_codes"], st["v_codes"], st["k_scale"], st["v_scale"]
    q, k = _turn(st["q"], st["at"], st["dims"], st["interleaved"]), _turn(st["key"], st["at"], st["dims"], st["interleaved"])
    visit, row, n = st["visit"], st["at"] % P, st["visited"].numel()
    below = st["below"][:, None]
    for name, x in (("k", k.float()), ("v", st["value"].float())):
        codes, scale = st[name + "_codes"].view(torch.uint8), st[name + "_scale"]
        top = torch.zeros(n, Hkv, device="cuda").scatter_reduce(0, visit[:, None].expand(-1, Hkv), x.abs().amax(2), "amax")
        old = scale[st["visited"]]
        now = torch.where(below > 0, torch.maximum(old, _need(top)), _need(top))
        held = codes[st["visited"]]
        rows = held if name == "k" else held.permute(0, 1, 2, 4, 3).reshape(n, Hkv, P, dh)
        again = (rows.view(CODES).float() * (old / now)[:, :, None, None]).to(CODES).view(torch.uint8)
        rows = torch.where(torch.arange(P, device="cuda")[:, None] < below[:, :, None, None], again, rows)
        rows[visit, :, row] = (x / now[visit][:, :, None]).to(CODES).view(torch.uint8)
        codes[st["visited"]] = rows if name == "k" else rows.reshape(n, Hkv, P // 16, 16, dh).permute(0, 1, 2, 4, 3)
        scale[st["visited"]] = now
    return q, st["k_codes"], st["v_codes"], st["k_scale"], st["v_scale"]


def _attention(st):
    if own:
        import paper_2512_20920_amd as R
        R.revffn_op_attention_cached(st["desc"], st["cache"], True, st["window"], st["q"], st["o"], st["lse"], st["work"])
        return st["o"], st["lse"]
    H, Hkv, dh, P = st["heads"], st["kv_heads"], st["width"], st["page"]
    G, (S, most), n = H // Hkv, st["table"].shape, st["pad"].shape[1]
    table = st["table"].long().clamp(min=0)
    k = st["k_codes"].view(torch.uint8)[table].view(CODES).float() * st["k_scale"][table][..., None, None]
    v = st["v_codes"].view(torch.uint8)[table].view(CODES).float() * st["v_scale"][table][..., None, None, None]
    k = k.permute(0, 2, 4, 1, 3).reshape(S, Hkv, dh, most * P)                     # [sequence, key head, column, token]
    v = v.permute(0, 2, 1, 3, 5, 4).reshape(S, Hkv, most * P, dh)
    q = st["q"].float()[st["pad"]].reshape(S, n, Hkv, G, dh).permute(0, 2, 1, 3, 4).reshape(S, Hkv, n * G, dh)
    s = torch.matmul(q, k).mul_(1.0 / math.sqrt(dh)).reshape(S, Hkv, n, G, -1)
    if st["cap"]:
        s = torch.tanh(s / st["cap"]) * st["cap"]
    j, at = torch.arange(most * P, device="cuda"), st["at"][st["pad"]][..., None]
    sees = (j <= at) & (j < st["held"][:, None, None])
    if st["window"]:
        sees = sees & (j > at - st["window"])
    s = torch.where(sees[:, None, :, None], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(S, Hkv, n * G, -1), v).reshape(S, Hkv, n, G, dh) / torch.where(total == 0, 1.0, total)
    lse = (torch.log(total) + top)[..., 0]
    rows = lambda t: t.transpose(1, 2).flatten(2, 3)[st["seq"], st["place"]]       # [row, head, ...]
    return rows(o).to(st["q"].dtype), rows(lse).t().contiguous()


def _product(st):
    M, N, K = st["rows"], st["outer"], st["inner"]
    if own:
        import paper_2512_20920_amd as R
        dt, ld = 1 if st["dtype"] == "bf16" else 0, st["w"].stride(0)
        R.revffn_op_quantize_rows(dt, st["x"], st["codes"], st["scale"], M, K, K, ld)
        R.revffn_op_gemm_int(dt, 0, st["codes"], st["scale"], st["w"], st["wscale"], st["bias"], st["y"], M, N, K, ld, ld, N)
        return st["y"]
    x = st["x"].float()
    scale = (x.abs().amax(1, keepdim=True).double() / 127.0).float()
    codes = torch.round(x.double() / torch.where(scale == 0, 1.0, scale).double()).float()      # (64 bits: which side of a half a quotient is on)
    y = torch.matmul(codes, st["w"][:, :K].float().t()) * scale * st["wscale"]
    if st["bias"] is not None:
        y = y + st["bias"].float()
    return y.to(st["x"].dtype)


def _pairs(case):
    """How many keys the queries see, in all."""
    total = 0
    for h, n in zip(_lens(case["held"]), _lens(case["new"])):
        sees = np.arange(h - n, h) + 1
        total += int((np.minimum(sees, case["window"]) if case["window"] else sees).sum())
    return total


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "product":
        M, N, K = case["rows"], case["outer"], case["inner"]
        return {"bytes": size * M * K + N * K + 4 * N + size * M * N + (size * N if case["bias"] else 0), "flops": 2 * M * N * K}
    T, H, Hkv, dh = sum(_lens(case["new"])), case["heads"], case["kv_heads"], case["width"]
    if case["op"] == "append":
        return {"bytes": size * T * (2 * H + 2 * Hkv) * dh + 2 * T * Hkv * dh + 4 * T, "flops": 3 * T * (H + Hkv) * case["dims"] + 4 * T * Hkv * dh}
    seen = sum(min(h, n + case["window"] - 1) if case["window"] else h for h, n in zip(_lens(case["held"]), _lens(case["new"])))
    return {"bytes": 2 * size * T * H * dh + 4 * T * H + 2 * seen * Hkv * dh + 8 * (seen // case["page"]) * Hkv, "flops": 4 * _pairs(case) * dh * H}


def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "product": _exact_product}[case["op"]](case, st)


def _nearest8(x):
    """The 8-bit number (4 bits of exponent, 3 of mantissa) nearest to each value, ties to even, in 64 bits."""
    size = x.abs()
    step = torch.exp2(torch.floor(torch.log2(size.clamp(min=2.0 ** -6))) - 3)
    return torch.sign(x) * torch.round(size / step) * step


def _exact_append(case, st):
    P, dh, dims, dt = case["page"], case["width"], case["dims"], st["q"].dtype
    at = st["at"].double()
    f = torch.tensor([THETA ** (-2.0 * i / dims) for i in range(dims // 2)], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones(len(at), dims // 2, dtype=torch.float64, device="cuda"), at[:, None] * f)[:, None]

    def turned(x):
        x = x.double()
        a, b = (x[..., 0:dims:2], x[..., 1:dims:2]) if case["interleaved"] else (x[..., : dims // 2], x[..., dims // 2 : dims])
        z = torch.complex(a.contiguous(), b.contiguous()) * turn
        part = torch.stack([z.real, z.imag], -1).flatten(-2) if case["interleaved"] else torch.cat([z.real, z.imag], -1)
        return torch.cat([part, x[..., dims:]], -1)

    out = []
    new = {"k": turned(st["key"]).to(dt).double(), "v": st["value"].double()}       # (a key is rounded to its type, then to 8 bits)
    held, fresh, table = _lens(case["held"]), _lens(case["new"]), st["table"].cpu().numpy()
    for name in ("k", "v"):
        codes, scale = st[name + "_codes"].double(), st[name + "_scale"].double()
        if name == "v":
            codes = codes.transpose(3, 4).flatten(2, 3)
        codes = codes.clone()
        row = 0
        for s, (h, n) in enumerate(zip(held, fresh)):
            for p in range((h - n) // P, -(-h // P)):
                a, b, page = max(h - n - p * P, 0), min(h - p * P, P), int(table[s, p])
                x = new[name][row : row + b - a].transpose(0, 1)                   # [key head, row, column]
                row += b - a
                top = x.abs().amax((1, 2))
                power = torch.exp2(torch.ceil(torch.log2(top / 448.0)).clamp(-96, 119))
                if a > 0:
                    power = torch.maximum(power, scale[page])
                    codes[page, :, :a] = _nearest8(codes[page, :, :a] * (scale[page] / power)[:, None, None])
                codes[page, :, a:b] = _nearest8(x / power[:, None, None])
                scale[page] = power
        if name == "v":
            codes = codes.unflatten(2, (P // 16, 16)).transpose(3, 4)
        out.append((codes, scale))
    return turned(st["q"]), out[0][0], out[1][0], out[0][1], out[1][1]


def _exact_attention(case, st):
    if _pairs(case) * case["heads"] * case["width"] > 1.2e11:
        return None
    H, Hkv, dh, P = case["heads"], case["kv_heads"], case["width"], case["page"]
    G, T = H // Hkv, st["q"].shape[0]
    o, lse = torch.zeros(T, H, dh, dtype=torch.float64, device="cuda"), torch.zeros(H, T, dtype=torch.float64, device="cuda")
    row = 0
    for s, (h, n) in enumerate(zip(_lens(case["held"]), _lens(case["new"]))):
        pages = st["table"][s, : -(-h // P)].long().cpu()
        for c in range(Hkv):
            k = torch.cat([st["k_codes"][p, c].double() * st["k_scale"][p, c].double() for p in pages.tolist()])[:h]
            v = torch.cat([(st["v_codes"][p, c].double() * st["v_scale"][p, c].double()).transpose(1, 2).flatten(0, 1) for p in pages.tolist()])[:h]
            q = st["q"][row : row + n, c * G : (c + 1) * G].double()
            z = torch.tensordot(q, k, ([2], [1])) * dh ** -0.5
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            far = torch.arange(h - n, h, device="cuda")[:, None] - torch.arange(h, device="cuda")      # how far behind the query a key is
            hidden = far < 0
            if case["window"]:
                hidden |= far >= case["window"]
            z = z.masked_fill(hidden[:, None], -math.inf)
            norm = torch.logsumexp(z, 2)
            o[row : row + n, c * G : (c + 1) * G] = torch.tensordot(torch.exp(z - norm[..., None]), v, ([2], [0]))
            lse[c * G : (c + 1) * G, row : row + n] = norm.t()
        row += n
    return o, lse


def _exact_product(case, st):
    K = case["inner"]
    w, ws = st["w"][:, :K].double(), st["wscale"].double()
    out = []
    for x in st["x"].split(1024):
        x = x.double()
        unit = (x.abs().amax(1) / 127).float().double()                            # (the scale is a 32-bit number)
        codes = torch.round(x / torch.where(unit == 0, torch.ones_like(unit), unit)[:, None])
        y = (codes @ w.t()) * unit[:, None] * ws
        out.append(y + st["bias"].double() if st["bias"] is not None else y)
    return torch.cat(out)
