"""The paged cache of 8-bit numbers, its attention and the integer products through the C ABI, against 64 bits: what is stored bit for bit, what is
computed within bounds from the arithmetic."""
import numpy as np
import pytest
import torch

import cache_reference as ref
from operators_reference import outside

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2512_20920_amd as R

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN = float("nan")


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", torch.int32)


def _normal(rng, dtype, *shape, scale=1.0):
    return torch.from_numpy((scale * rng.standard_normal(shape)).astype(np.float32)).to(TORCH[dtype]).cuda()


class Paged:
    """A cache on the GPU beside the reference's.  Its memory starts out as NaNs throughout."""

    def __init__(self, dtype, Hkv, dh, page, tables, pages=None, seed=0):
        self.dtype, self.Hkv, self.dh, self.page = dtype, Hkv, dh, page
        self.table = np.asarray(tables)
        self.pages = int(self.table.max()) + 2 if pages is None else pages
        one = lambda *s: torch.full(s, 255, dtype=torch.uint8, device="cuda")
        self.k, self.v = one(self.pages, Hkv, page, dh), one(self.pages, Hkv, page // 16, dh, 16)
        self.ks, self.vs = (torch.full((self.pages, Hkv), NAN, dtype=torch.float32, device="cuda") for _ in range(2))
        self.model = ref.Cache(self.pages, page, Hkv, dh)
        self.rng = np.random.default_rng(seed)

    def cache(self, held, cu):
        self.lists = (_ints(self.table), _ints(held), None if cu is None else _ints(cu))
        return R.Cache(self.k, self.v, self.ks, self.vs, *self.lists, pages=self.pages, page=self.page, max_pages=self.table.shape[1],
                       n_seqs=self.table.shape[0], Hkv=self.Hkv, dh=self.dh)

    def values(self):
        """{name: [pages, Hkv, page, dh]} of what the memory stands for, in units of its scales."""
        v = ref.decode(self.v.cpu().numpy()).transpose(0, 1, 2, 4, 3).reshape(self.model.numbers["v"].shape)
        return {"k": ref.decode(self.k.cpu().numpy()), "v": v}

    def check(self):
        got = self.values()
        for name, scale in (("k", self.ks), ("v", self.vs)):
            assert np.array_equal(_np(scale), self.model.scale[name], equal_nan=True), name
            assert np.array_equal(got[name], self.model.numbers[name], equal_nan=True), name

    def append(self, held, new, H=2, rotary=None, pos=None, pad=0, k=None, v=None, in_place=False, no_q=False, stream=None, single=False, extra=3):
        """Rows of a projection [T + extra, H + 2 Hkv heads + pad]; checks the cache and the queries against the rotation alone."""
        T, dh, Hkv, dtype = sum(new), self.dh, self.Hkv, self.dtype
        rows = T + extra
        wide = torch.full((rows, (H + 2 * Hkv) * dh + pad), NAN, dtype=TORCH[dtype], device="cuda")
        wide[:T, :(H + 2 * Hkv) * dh] = _normal(self.rng, dtype, T, (H + 2 * Hkv) * dh)
        q, kk, vv = wide[:, :H * dh], wide[:, H * dh:(H + Hkv) * dh], wide[:, (H + Hkv) * dh:(H + 2 * Hkv) * dh]
        if k is not None:
            kk[:T], vv[:T] = k.reshape(T, -1), v.reshape(T, -1)
        if pos is None:
            at = np.concatenate([np.arange(h - n, h) for h, n in zip(held, new)] + [np.zeros(extra, int)])
        else:
            at = np.concatenate([pos, np.zeros(extra, int)])
        before, ld, dt = wide.clone(), wide.stride(0), 1 if dtype == "bf16" else 0
        out = q if in_place else torch.full((rows, H * dh), NAN, dtype=TORCH[dtype], device="cuda")
        heads = lambda t, n: _np(t[:T]).reshape(T, n, dh)
        want_q, want_k = heads(before[:, :H * dh], H), heads(before[:, H * dh:(H + Hkv) * dh], Hkv)
        if rotary is not None:
            want_q, want_k = (ref.turned(x, at[:T], R.revffn_op_rotary_frequencies(rotary), rotary.interleaved, rotary.magnitude or 1.0) for x in (want_q, want_k))
            want_k = _np(torch.from_numpy(want_k).float().to(TORCH[dtype]))
        c = self.cache(held, None if single else np.cumsum([0] + list(new)))
        R.revffn_op_cache_append(dt, c, rotary, None if pos is None else _ints(at), None if no_q else q, None if no_q else out, kk, vv, T if single else rows, H, ld,
                                 out.stride(0), ld, ld, stream=stream)
        torch.cuda.synchronize()
        owned = np.concatenate([(np.arange(h - n, h) >= 0) & (np.arange(h - n, h) < self.page * self.table.shape[1]) for h, n in zip(held, new)])
        if not no_q:
            mine = torch.from_numpy(owned).cuda()
            # one rounding to float32 and one to the type
            got = _np(out[:T]).reshape(T, H, dh)[owned]
            assert (np.abs(got - want_q[owned]) <= (np.abs(want_q[owned]) + 2.0 ** -126) * (2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0)) * (1 + 2.0 ** -8)).all()
            rest = before[:, :H * dh] if in_place else torch.full_like(before[:, :H * dh], NAN)
            assert torch.equal(out[:T][~mine].nan_to_num(7.0), rest[:T][~mine].nan_to_num(7.0)) and torch.isnan(out[T:]).all()
        if not in_place:
            assert torch.equal(wide.nan_to_num(7.0), before.nan_to_num(7.0))       # the inputs are as they were
        self.model.append(self.table, held, new, want_k, heads(before[:, (H + Hkv) * dh:(H + 2 * Hkv) * dh], Hkv))
        self.check()


def _tables(rng, lens, page, spare=1):
    need = [-(-n // page) for n in lens]
    order = rng.permutation(sum(need) + 2)
    t = np.full((len(lens), max(max(need), 1) + spare), -1)
    for s in range(len(lens)):
        t[s, :need[s]] = order[sum(need[:s]):sum(need[:s + 1])]
    return t


def _rotary(dims, interleaved=False, **kw):
    return R.Rotary(dims=dims, interleaved=interleaved, theta=1e4, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv,dh,page,H,dims,interleaved", [
    (2, 64, 16, 4, 64, False), (1, 128, 64, 2, 128, False), (2, 128, 128, 2, 64, True), (3, 16, 16, 3, 16, False), (1, 256, 64, 1, 256, False),
    (2, 80, 32, 6, 32, True), (2, 96, 128, 2, 96, False), (5, 48, 64, 5, 16, False), (1, 144, 32, 2, 144, True), (8, 64, 128, 16, 64, False)])
def test_append(Hkv, dh, page, H, dims, interleaved, dtype):
    """A prompt each, pieces that end inside pages, single tokens, a sequence that gets nothing."""
    rng = np.random.default_rng(page + dh)
    c = Paged(dtype, Hkv, dh, page, _tables(rng, [150, 3 * page + 2, 40, 9], page))
    r = _rotary(dims, interleaved)
    held = np.zeros(4, int)
    for new in ([37, 3 * page, 0, 1], [1, 1, 0, 0], [page, 0, 17, 3], [1, 1, 1, 1], [30, 0, 1, 0]):
        held = held + new
        c.append(list(held), new, H, r)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(pad=8), dict(pad=3), dict(pad=1, in_place=True), dict(in_place=True), dict(no_q=True), dict(no_q=True, pad=5)])
def test_append_strides_and_places(kw, dtype):
    c = Paged(dtype, 2, 64, 32, [[1, 0, 3], [4, 2, -1]])
    c.append([70, 33], [70, 33], 3, _rotary(64), **kw)
    c.append([71, 40], [1, 7], 3, None, **kw)
    c.append([75, 41], [4, 1], 3, _rotary(32, True, scaling=1, factor=4.0, magnitude=1.2), pos=np.array([90000, 5, 0, 7, 2 ** 30]), **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 200])
def test_append_single_tokens(n, dtype):
    """One row each, with and without a list of first rows, around the number of sequences that a wave looks at at once."""
    rng = np.random.default_rng(n)
    lens = rng.integers(1, 40, n)
    for single in (False, True):
        c = Paged(dtype, 1, 16, 16, _tables(rng, lens + 1, 16), seed=n)
        c.append(list(lens), list(lens), 1, _rotary(16))
        c.append(list(lens + 1), [1] * n, 1, _rotary(16), single=single, extra=0 if single else 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_of_many_sequences(dtype):
    """Prompts, pieces, single tokens and nothing, in a list longer than a wave looks at at once."""
    rng = np.random.default_rng(8)
    n = 150
    new = rng.integers(0, 3, n) * rng.integers(0, 30, n)
    more = rng.integers(0, 2, n)
    more[[2, 70, 149]] = 100, 33, 64
    c = Paged(dtype, 2, 32, 16, _tables(rng, new + more, 16), seed=9)
    c.append([int(x) for x in new], [int(x) for x in new], 2, _rotary(32))
    c.append([int(x) for x in new + more], [int(x) for x in more], 2, _rotary(32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_values(dtype):
    """Zeros, values that are not finite, far apart in size, around powers of two, and pages whose unit grows with each token."""
    dh, t = 32, TORCH[dtype]
    c = Paged(dtype, 2, dh, 16, [[0, 1, 2, 3, 4]])
    rng = np.random.default_rng(3)
    k = rng.standard_normal((16, 2, dh)) * 2.0 ** rng.integers(-30, 30, (16, 2, 1))
    k[0] = 0
    k[1, 0, ::3], k[1, 1, 1], k[2, :, 5] = np.inf, np.nan, -np.inf
    v = rng.standard_normal((16, 2, dh))
    v[:, 1] = 0
    v[3, 0] = np.nan
    up = lambda x: torch.from_numpy(x.astype(np.float32)).to(t).cuda()
    c.append([16], [16], 1, None, k=up(k), v=up(v))
    c.append([18], [2], 1, None, k=up(np.full((2, 2, dh), np.nan)), v=up(np.zeros((2, 2, dh))))      # a page begun with nothing finite
    for j in range(14):
        size = 2.0 ** (3 * j - 20)
        c.append([19 + j], [1], 1, None, k=up(rng.standard_normal((1, 2, dh)) * size), v=up(rng.standard_normal((1, 2, dh)) / size))
    edge = np.array([448.0, 449, 447, 464, 480, 1e30, 3e38, 2.0 ** -100, 1e-38, 2.0 ** -9, 2.0 ** -10, 1.0, 240.0, 232, 248, 17.0] * 2).reshape(1, 1, dh) * np.ones((3, 2, 1))
    edge[1] *= 2.0 ** -20
    edge[2, 1] = 2.0 ** -130
    c.append([35], [3], 1, None, k=up(edge), v=up(-edge))
    if dtype == "f32":
        low = np.full((1, 2, dh), 1e-42)
        c.append([36], [1], 1, None, k=up(low), v=up(low))


def test_append_pages_that_are_none():
    """Entries of the table out of range, tokens behind its end, rows that would stand before token 0, more rows than the sequences own,
    numbers out of range: what has no place is left out, everything else is as it should be."""
    c = Paged("bf16", 2, 64, 16, [[0, -1, 2, 99], [3, 4, 5, -2 ** 31], [1, 2 ** 31 - 1, 6, 7]], pages=8)
    c.append([64, 40, 17], [64, 20, 17], 2, _rotary(64))
    c.append([70, 100, 18], [6, 60, 1], 2, _rotary(64))          # behind the table's end
    c.append([70, 3, 18], [0, 9, 0], 2, _rotary(64))             # six rows before token 0
    # first rows and lengths out of range
    T = 4
    x = torch.zeros(T, 4 * 64, dtype=torch.bfloat16, device="cuda")
    before = [t.clone() for t in (c.k, c.v, c.ks, c.vs)]
    out = torch.full((T, 128), NAN, dtype=torch.bfloat16, device="cuda")
    for held, cu in (([-5, -2 ** 31, 0], [0, 1, 2, 3]), ([5, 6, 7], [9, 4, 100, 4]), ([5, 6, 7], [-7, -3, 0, 0])):
        cache = c.cache(held, cu)
        R.revffn_op_cache_append(1, cache, _rotary(64), None, x[:, :128], out, x[:, 128:], x[:, 128:].clone(), T, 2, 256, 128, 256, 128)
        torch.cuda.synchronize()
        assert all(torch.equal(a.nan_to_num(9.0) if a.is_floating_point() else a, b.nan_to_num(9.0) if b.is_floating_point() else b) for a, b in zip((c.k, c.v, c.ks, c.vs), before))


# name: heads, key heads, width, page, tokens held, new ones, options
SHAPES = {
    "one_token": (2, 2, 64, 16, [1], [1], {}),
    "next_tokens": (8, 2, 128, 64, [212, 37, 1001, 1, 128, 300], [1] * 6, {}),
    "next_tokens_small_pages": (4, 4, 64, 16, [15, 16, 17, 32, 33, 100], [1] * 6, {}),
    "next_tokens_large_pages": (16, 1, 128, 128, [127, 128, 129, 500], [1] * 4, {}),
    "forty_heads_to_one": (40, 1, 64, 32, [70, 200], [1, 1], {}),
    "hundred_heads_to_one": (100, 1, 16, 16, [50], [1], {}),
    "three_heads_to_one": (6, 2, 128, 32, [30, 90, 5], [12, 3, 5], {}),
    "prompt": (4, 2, 128, 64, [150], [150], {}),
    "prompt_behind_a_cache": (4, 1, 64, 16, [333], [70], {}),
    "mixed": (4, 2, 64, 32, [200, 77, 260, 1, 5], [130, 1, 40, 1, 0], {}),
    "window": (4, 2, 64, 16, [300, 77, 40], [100, 1, 40], dict(window=33)),
    "window_of_one": (2, 2, 64, 16, [100, 33], [40, 1], dict(window=1)),
    "not_causal": (2, 1, 64, 32, [100, 33], [40, 33], dict(causal=False)),
    "capped": (4, 4, 64, 16, [140, 61], [100, 1], dict(cap=5.0)),
    "biased": (4, 2, 128, 32, [140, 61], [100, 1], dict(bias=True)),
    "capped_biased": (4, 2, 64, 32, [140, 61], [100, 1], dict(cap=5.0, bias=True)),
    "capped_wide": (2, 2, 128, 16, [140, 61], [20, 1], dict(cap=3.0)),
    "width_16": (2, 1, 16, 16, [70, 65], [70, 1], {}),
    "width_32": (2, 1, 32, 64, [70, 65], [33, 1], {}),
    "width_80": (3, 1, 80, 32, [70, 65], [40, 1], dict(cap=20.0)),
    "width_96": (2, 2, 96, 128, [150], [60], {}),
    "width_112": (2, 2, 112, 16, [150], [60], dict(bias=True)),
    "width_144": (2, 1, 144, 16, [50, 40], [20, 1], {}),
    "width_256": (2, 1, 256, 64, [100, 40], [35, 1], {}),
    "width_256_capped": (2, 2, 256, 16, [60, 40], [5, 1], dict(cap=4.0)),
    "width_208_prompt": (2, 1, 208, 32, [170], [100], {}),
    "width_256_prompt": (2, 2, 256, 16, [170, 5], [150, 5], dict(cap=4.0, bias=True)),
    "more_rows_than_tokens": (2, 2, 64, 16, [5, 0, 20], [9, 3, 1], {}),
    "nothing_held": (2, 2, 64, 16, [0, 0], [2, 1], dict(causal=False)),
}
MODES = pytest.mark.parametrize("dtype,mode", [("bf16", 2), ("bf16", 1), ("f32", 2), ("f32", 1)])


def _slopes(H):
    return 2.0 ** (-8.0 * (np.arange(H) + 1) / H)


def _fill(c, held, k=None, v=None):
    """All tokens of all sequences into the cache at once (written by the reference: the append has tests of its own)."""
    n = int(np.sum(held))
    k = c.rng.standard_normal((n, c.Hkv, c.dh)) if k is None else k
    v = c.rng.standard_normal((n, c.Hkv, c.dh)) if v is None else v
    c.model.append(c.table, list(held), list(held), k, v)
    for name, codes, scale in (("k", c.k, c.ks), ("v", c.v, c.vs)):
        x = torch.from_numpy(c.model.numbers[name]).float().to(torch.float8_e4m3fn).view(torch.uint8)
        if name == "v":
            x = x.reshape(c.pages, c.Hkv, c.page // 16, 16, c.dh).transpose(3, 4)
        codes.copy_(x.contiguous())
        scale.copy_(torch.from_numpy(c.model.scale[name]).float())


class Attend:
    def __init__(self, c, held, new, H, mode=0, pad=0, extra=2, scale=0.0, cap=0.0, slopes=None, cu=True, qscale=1.0):
        self.c, self.held, self.new, self.H = c, held, new, H
        T, dh = sum(new), c.dh
        self.T = T
        self.q = torch.full((T + extra, H * dh + pad), NAN, dtype=TORCH[c.dtype], device="cuda")
        self.q[:T, :H * dh] = _normal(c.rng, c.dtype, T, H * dh, scale=qscale)
        self.o = torch.full_like(self.q, NAN)
        self.lse = torch.full((H, T + extra), NAN, dtype=torch.float32, device="cuda")
        self.scale, self.cap, self.slopes = scale, cap, slopes
        self.cache = c.cache(held, np.cumsum([0] + list(new)) if cu else None)
        self.slope_t = None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device="cuda")
        self.desc = R.AttnDesc(dtype=1 if c.dtype == "bf16" else 0, kernel_mode=mode, H=H, Hkv=c.Hkv, dh=dh, Tq=T + extra, ldq=self.q.stride(0), ldo=self.o.stride(0),
                               scale=scale, softcap=cap, slopes=self.slope_t)
        n = R.revffn_op_attention_cached_workspace(self.desc, self.cache)
        self.work = torch.full((n,), 255, dtype=torch.uint8, device="cuda")         # NaN patterns throughout

    def run(self, causal=True, window=0, stream=None):
        self.how = dict(causal=causal, window=window)
        R.revffn_op_attention_cached(self.desc, self.cache, causal, window, self.q, self.o, self.lse, self.work, stream=stream)

    def queries(self):
        return _np(self.q[:self.T, :self.H * self.c.dh]).reshape(self.T, self.H, self.c.dh)

    def results(self):
        torch.cuda.synchronize()
        return _np(self.o[:self.T, :self.H * self.c.dh]).reshape(self.T, self.H, self.c.dh), _np(self.lse[:, :self.T])

    def check(self):
        o, lse = self.results()
        sl = None if self.slopes is None else np.asarray(self.slopes, np.float32).astype(np.float64)
        want = ref.attention(self.c.model, self.c.table, self.held, self.new, self.queries(), scale=self.scale or None, cap=self.cap, slopes=sl, dtype=self.c.dtype, **self.how)
        worst = outside(o, *want["o"]), outside(lse, *want["lse"])
        assert max(worst) <= 1.0, worst
        assert torch.isnan(self.o[self.T:]).all() and torch.isnan(self.o[:, self.H * self.c.dh:]).all() and torch.isnan(self.lse[:, self.T:]).all()


def _attend(name, dtype, mode, **kw):
    H, Hkv, dh, page, held, new, opt = SHAPES[name]
    if dtype == "f32" and dh > 128 and mode == 2:
        mode = 0                                             # (refused on the matrix cores: see the host's tests)
    opt = dict(opt)
    c = Paged(dtype, Hkv, dh, page, _tables(np.random.default_rng(len(name)), held, page), seed=len(name))
    _fill(c, held)
    a = Attend(c, held, new, H, mode, cap=opt.pop("cap", 0.0), slopes=_slopes(H) if opt.pop("bias", False) else None, **kw)
    a.run(**opt)
    return a


@MODES
@pytest.mark.parametrize("name", list(SHAPES))
def test_attention(name, dtype, mode):
    _attend(name, dtype, mode).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,mode", [(8, 2), (64, 0), (3, 0), (1, 1)])
def test_attention_strides(pad, mode, dtype):
    _attend("mixed", dtype, mode, pad=pad).check()


@MODES
def test_attention_without_a_list_of_first_rows(dtype, mode):
    _attend("next_tokens", dtype, mode, cu=False, extra=0).check()


@MODES
@pytest.mark.parametrize("scale,cap", [(0.3, 0.0), (-0.2, 0.0), (-0.2, 3.0), (1e-3, 0.5), (4.0, 0.0), (0.1, 1e6)])
def test_attention_scales(scale, cap, dtype, mode):
    """Scores of hundreds among them: one key takes nearly all of a query's weight, and maxima rise late."""
    c = Paged(dtype, 1, 64, 32, [[2, 0, 1, 4, 3, 5], [7, 6, 8, 9, 10, 11]])
    _fill(c, [150, 70])
    a = Attend(c, [150, 70], [110, 1], 2, mode, scale=scale, cap=cap)
    a.run()
    a.check()


@MODES
def test_attention_holes_and_ends(dtype, mode):
    """Pages that are none in the middle and at the end, lengths behind the table's end, a sequence all of whose pages are none."""
    table = np.array([[0, -1, 2, 99, 4], [-1, -1, -1, -1, -1], [5, 6, 7, 8, -3], [9, 2 ** 31 - 1, 10, 11, 12]])
    for page in (16, 32):
        c = Paged(dtype, 2, 64, page, table, pages=13)
        held = [5 * page, 40, 4 * page - 3, 5 * page + 9]
        _fill(c, held)
        a = Attend(c, held, [3, 2, 50, 30], 4, mode)
        a.run()
        a.check()
        o, lse = a.results()
        assert (o[3:5] == 0).all() and np.isneginf(lse[:, 3:5]).all()


@MODES
def test_attention_lists_out_of_range(dtype, mode):
    """Lengths and first rows out of range end the call in order, and nobody's rows but the owned ones are written."""
    c = Paged(dtype, 2, 64, 16, [[0, 1, 2], [3, 4, 5], [6, 7, 8]])
    _fill(c, [48, 48, 48])
    a = Attend(c, [48, 48, 48], [1, 2, 3], 4, mode)
    for held, cu in (([-4, -2 ** 31, 2 ** 31 - 1], [0, 1, 3, 6]), ([48, 48, 48], [100, -7, 2 ** 31 - 1, -1]), ([48, 48, 48], [5, 4, 3, 2]), ([0, 0, 0], [0, 0, 0, 0])):
        a.cache = c.cache(held, cu)
        a.run()
        a.results()
        assert torch.isnan(a.o[a.T:]).all()


@MODES
@pytest.mark.parametrize("held,new", [([70, 300, 45, 200], [60, 1, 5, 200]), ([1000, 40], [1, 1])])
def test_attention_values_that_are_not_finite(held, new, dtype, mode):
    """A NaN among one sequence's values (keys, queries): who sees it gets it, everybody else's results are what they are without, rows of the same
    tile that may not see it yet among them."""
    for where in ("k", "v", "q"):
        c, clean = (Paged(dtype, 1, 64, 16, _tables(np.random.default_rng(7), held, 16), seed=5) for _ in range(2))
        n = int(np.sum(held))
        k, v = np.random.default_rng(6).standard_normal((2, n, 1, 64))
        _fill(clean, held, k, v)
        token = held[0] - 2                                  # of the first sequence: its last query but one sees it first, if it has so many
        if where != "q":
            (k if where == "k" else v)[token, 0, 3] = np.nan
        _fill(c, held, k, v)
        a, b = Attend(c, held, new, 2, mode), Attend(clean, held, new, 2, mode)
        a.q.copy_(b.q)
        if where == "q":
            a.q[0, 5] = NAN
        a.run()
        b.run()
        b.check()
        o, lse = a.results()
        o2, lse2 = b.results()
        want = ref.attention(clean.model, clean.table, held, new, b.queries(), dtype=dtype)
        at = held[0] - new[0] + np.arange(new[0])
        sees = np.zeros((a.T, 2), bool)
        if where == "q":
            sees[0, 0] = True
        else:
            sees[:new[0]][at >= token] = True
        assert np.isnan(o[sees]).any(axis=-1).all() and sees.any()
        # (rows worked out again add in another order: both are within the bounds, so at most two of them apart)
        assert outside(o[~sees], o2[~sees], 2 * want["o"][1][~sees]) <= 1.0, where
        assert outside(lse[~sees.T], lse2[~sees.T], 2 * want["lse"][1][~sees.T]) <= 1.0


@pytest.mark.parametrize("H,dh,rows,dtype", [(64, 256, 140, "bf16"), (128, 256, 390, "bf16"), (64, 128, 260, "bf16"), (256, 128, 390, "bf16"),
                                             (128, 64, 260, "bf16"), (512, 64, 390, "bf16"), (128, 64, 260, "f32"), (256, 128, 390, "f32")])
def test_attention_of_many_rows(H, dh, rows, dtype):
    """So many that a workgroup takes 64 of them, or 128, not 32 as with the shapes above; tokens, a few rows and nobody beside them."""
    held, new = [rows + 37, 90, 33, 0, 20], [rows, 1, 3, 0, 20]
    page = 16 if dh == 64 else 64
    c = Paged(dtype, H // 4, dh, page, _tables(np.random.default_rng(rows), held, page), seed=rows)
    _fill(c, held)
    a = Attend(c, held, new, H, 0)
    a.run(window=(200 if rows == 390 else 0))
    a.check()


@MODES
@pytest.mark.parametrize("n,prompts", [(64, 0), (65, 0), (65, 3), (150, 0), (150, 5), (300, 2)])
def test_attention_of_many_sequences(n, prompts, dtype, mode):
    """Lists longer than a wave looks at at once, long sequences and prompts among them, so that some keys are split and most are not."""
    rng = np.random.default_rng(n + prompts)
    held, new = rng.integers(0, 90, n), rng.integers(0, 2, n)
    held[[3, n // 2, n - 1]] = 2600, 700, 1500
    for s in rng.permutation(n)[:prompts]:
        new[s] = min(held[s], 75)
    held, new = [int(x) for x in held], [int(x) for x in new]
    c = Paged(dtype, 2, 64, 16, _tables(rng, held, 16), seed=n)
    _fill(c, held)
    a = Attend(c, held, new, 8, mode)
    a.run()
    a.check()


@MODES
@pytest.mark.parametrize("held,new", [([70, 300, 45, 17], [60, 1, 5, 17]), ([1000, 33], [1, 1]), ([150, 3000], [150, 1])])
def test_attention_beside_pages_not_begun(held, new, dtype, mode):
    """Entries behind a sequence's last token may name pages that nothing was appended to, whose units are NaN: the bits are those without them."""
    table = _tables(np.random.default_rng(2), held, 16, spare=4)
    out = []
    for behind in (-1, table.max() + 1):
        c = Paged(dtype, 1, 64, 16, np.where(table < 0, behind, table), pages=int(table.max()) + 2, seed=4)
        _fill(c, held)
        for s, n in enumerate(held):                         # nor is there anything in a last page's other places
            if n % 16:
                c.k[table[s, n // 16], :, n % 16:] = 255
                c.v[table[s, n // 16], :, 0, :, n % 16:] = 255
        a = Attend(c, held, new, 2, mode)
        a.run()
        a.check()
        out.append((a.o, a.lse))
    assert all(torch.equal(x.nan_to_num(5.0), y.nan_to_num(5.0)) for x, y in zip(*out))


@MODES
def test_attention_over_shared_pages(dtype, mode):
    """Two sequences that begin alike name the same pages for it."""
    table = np.array([[4, 1, 5, 0, -1], [4, 1, 5, 2, 3]])
    held, new = [120, 155], [60, 2]
    k, v = np.random.default_rng(3).standard_normal((2, sum(held), 2, 64))
    k[120:216], v[120:216] = k[:96], v[:96]
    c = Paged(dtype, 2, 64, 32, table)
    _fill(c, held, k, v)
    a = Attend(c, held, new, 4, mode)
    a.run()
    a.check()


@pytest.mark.parametrize("dtype,rows,keys", [("bf16", 1, 9000), ("bf16", 33, 5000), ("f32", 1, 9000), ("bf16", 1, 40000)])
def test_attention_of_long_sequences(dtype, rows, keys):
    """Keys split over many workgroups, their pages far apart in a large memory; spot rows against the reference."""
    page = 64
    n = -(-keys // page)
    rng = np.random.default_rng(keys)
    c = Paged(dtype, 1, 128, page, rng.permutation(n + 3)[None, :n + 1], pages=n + 3)
    _fill(c, [keys])
    a = Attend(c, [keys], [rows], 4, 0)
    a.run()
    a.check()


def test_attention_far_into_memory():
    """A memory of more than 2^32 bytes of keys: the last pages are where they should be, for both operators."""
    page, Hkv, dh = 128, 8, 128
    pages = (1 << 32) // (page * Hkv * dh) + 40
    k, v = (torch.empty(pages, Hkv, page * dh, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.empty(pages, Hkv, dtype=torch.float32, device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = torch.randn(200, 10, dh, generator=g, device="cuda").to(torch.bfloat16)
    out = []
    for first in (0, pages - 2):
        table, held, cu = _ints([[first + 1, first]]), _ints([200]), _ints([0, 200])
        cache = R.Cache(k, v, ks, vs, table, held, cu, pages=pages, page=page, max_pages=2, n_seqs=1, Hkv=Hkv, dh=dh)
        kk, vv = (torch.randn(200, Hkv, dh, generator=torch.Generator(device="cuda").manual_seed(s), device="cuda").to(torch.bfloat16) for s in (1, 2))
        R.revffn_op_cache_append(1, cache, None, None, None, None, kk, vv, 200, 0, 0, 0, Hkv * dh, Hkv * dh)
        q = rows[:, :8].contiguous()
        o, lse = torch.empty_like(q), torch.empty(8, 200, dtype=torch.float32, device="cuda")
        desc = R.AttnDesc(dtype=1, H=8, Hkv=Hkv, dh=dh, Tq=200)
        work = torch.empty(R.revffn_op_attention_cached_workspace(desc, cache), dtype=torch.uint8, device="cuda")
        R.revffn_op_attention_cached(desc, cache, True, 0, q, o, lse, work)
        torch.cuda.synchronize()
        out.append((o, lse, k[first:first + 2].clone(), v[first:first + 2].clone(), ks[first:first + 2].clone(), vs[first:first + 2].clone()))
    assert all(torch.equal(x, y) for x, y in zip(*out)) and torch.isfinite(out[0][0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graph_replays_follow_the_lists(dtype):
    """A step of append and attention captured once and replayed as the sequences grow: every replay equals the same calls made eagerly on a cache of
    its own, with eager work between the replays."""
    page, Hkv, H, dh, S = 16, 2, 4, 64, 3
    table = [[0, 1, 2, 3], [4, 5, 6, 7], [8, 9, 10, 11]]
    held0 = np.array([5, 15, 31])
    rng = np.random.default_rng(8)
    a, b = Paged(dtype, Hkv, dh, page, table), Paged(dtype, Hkv, dh, page, table)
    k, v = rng.standard_normal((2, held0.sum(), Hkv, dh))
    _fill(a, held0, k, v)
    _fill(b, held0, k, v)
    dt, r = 1 if dtype == "bf16" else 0, _rotary(dh)
    x = torch.zeros(S, (H + 2 * Hkv) * dh, dtype=TORCH[dtype], device="cuda")
    desc = R.AttnDesc(dtype=dt, H=H, Hkv=Hkv, dh=dh, Tq=S)

    def state(c):
        cache = c.cache(held0, None)
        return cache, c.lists[1], torch.empty(S, H * dh, dtype=TORCH[dtype], device="cuda"), torch.empty(S, H * dh, dtype=TORCH[dtype], device="cuda"), \
            torch.empty(H, S, dtype=torch.float32, device="cuda"), torch.empty(R.revffn_op_attention_cached_workspace(desc, cache), dtype=torch.uint8, device="cuda")

    def step(st):
        cache, _, q, o, lse, work = st
        w = x.stride(0)
        R.revffn_op_cache_append(dt, cache, r, None, x, q, x[:, H * dh:], x[:, (H + Hkv) * dh:], S, H, w, H * dh, w, w)
        R.revffn_op_attention_cached(desc, cache, True, 0, q, o, lse, work)
    sa, sb = state(a), state(b)
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            step(sa)
    torch.cuda.synchronize()
    for n in range(6):
        x.copy_(_normal(rng, dtype, *x.shape))
        for st in (sa, sb):
            st[1].add_(1)
        graph.replay()
        step(sb)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in ((a.k, b.k), (a.v, b.v), (sa[2], sb[2]), (sa[3], sb[3]), (sa[4], sb[4])))
        assert torch.isfinite(sa[3]).all() and torch.equal(a.ks.nan_to_num(0), b.ks.nan_to_num(0))
        torch.randn(1000, device="cuda").sum().item()


def test_another_stream():
    a = _attend("mixed", "bf16", 2)
    torch.cuda.synchronize()
    want = a.o.clone()
    a.o.fill_(NAN)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    a.run(stream=s)
    s.synchronize()
    assert torch.equal(a.o.nan_to_num(3.0), want.nan_to_num(3.0))


def test_two_calls_at_once():
    """Two layers' attention on two streams, a workspace each, over and over: the bits of each alone."""
    calls = [_attend("next_tokens", "bf16", 2), _attend("mixed", "bf16", 2)]
    torch.cuda.synchronize()
    want = [a.o.clone() for a in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(20):
        for a, s in zip(calls, streams):
            a.run(stream=s)
    torch.cuda.synchronize()
    for a, w in zip(calls, want):
        assert torch.equal(a.o.nan_to_num(3.0), w.nan_to_num(3.0))


# ---- integer products ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (5, 64, 0), (7, 63, 1), (300, 1000, 8), (3, 1024, 0), (2, 1025, 7), (9, 4096, 16), (4, 5000, 3), (2, 40000, 0)])
def test_quantize_rows(rows, cols, pad, dtype):
    rng = np.random.default_rng(rows + cols)
    x = torch.full((rows, cols + pad), 1e30, dtype=TORCH[dtype], device="cuda")
    x[:, :cols] = _normal(rng, dtype, rows, cols) * (2.0 ** torch.from_numpy(rng.integers(-20, 20, (rows, 1))).float().cuda()).to(TORCH[dtype])
    if rows > 2:
        x[1, :cols] = 0
        x[2, :cols] = torch.arange(cols, device="cuda").remainder(255) / 2 - 63.5        # with a value of 63.5: every half a tie
        x[2, 0] = 63.5
    if rows > 6:
        x[3, cols // 2], x[4, 0], x[5, :cols] = NAN, float("-inf"), 1e-39 if dtype == "f32" else 1e-38
    codes = torch.full((rows, cols + pad), 99, dtype=torch.int8, device="cuda")
    scale = torch.full((rows + 1,), 5.0, dtype=torch.float32, device="cuda")
    R.revffn_op_quantize_rows(1 if dtype == "bf16" else 0, x, codes, scale, rows, cols, cols + pad, cols + pad)
    torch.cuda.synchronize()
    want, unit = ref.quantized(_np(x[:, :cols]))
    assert np.array_equal(_np(scale[:rows]), unit, equal_nan=True) and scale[rows] == 5.0
    assert np.array_equal(codes[:, :cols].cpu().numpy(), want) and (codes[:, cols:] == 99).all()


def _product(dtype, M, N, K, mode, pad=0, bias=True, seed=0, off=0):
    """Codes of all sizes; what lies in a row behind K is not zero."""
    rng = np.random.default_rng(seed + M + 3 * N + 7 * K)
    ld = (K + 15) // 16 * 16 + pad if off == 0 else K + pad
    ints = lambda n: torch.from_numpy(rng.integers(-128, 128, (n, ld)).astype(np.int8)).cuda()
    a, b = ints(M), ints(N)
    sa, sb = (torch.from_numpy(rng.uniform(0.001, 0.1, n).astype(np.float32)).cuda() for n in (M, N))
    z = _normal(rng, dtype, N) if bias else None
    c = torch.full((M + 1, N + 3), NAN, dtype=TORCH[dtype], device="cuda")
    R.revffn_op_gemm_int(1 if dtype == "bf16" else 0, mode, a, sa, b, sb, z, c, M, N, K, ld, ld, N + 3)
    torch.cuda.synchronize()
    exact = a[:, :K].cpu().numpy().astype(np.int64) @ b[:, :K].cpu().numpy().astype(np.int64).T
    want = exact * _np(sa)[:, None] * _np(sb) + (_np(z) if bias else 0.0)
    # the sum to float32, times one scale, times the other and the bias added: half a step each, then half a step of the type
    size = np.abs(exact * _np(sa)[:, None] * _np(sb))
    bound = 3 * 2.0 ** -24 * size + 2.0 ** -24 * np.abs(want) + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want)
    assert outside(_np(c[:M, :N]), want, bound * 1.001) <= 1.0
    assert torch.isnan(c[M]).all() and torch.isnan(c[:, N:]).all()
    return c


FORMS = [0, 1] + [256 * t for t in range(1, 6)]


@pytest.mark.parametrize("mode", FORMS)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 64, 16), (3, 5, 100), (8, 200, 333), (33, 129, 128), (64, 64, 129), (70, 300, 640), (130, 257, 1000), (300, 520, 2049), (257, 1024, 4096)])
def test_product(M, N, K, mode):
    for dtype in ("bf16", "f32"):
        _product(dtype, M, N, K, mode)


@pytest.mark.parametrize("mode", [0, 1])
def test_product_rows_that_are_not_aligned(mode):
    _product("bf16", 40, 70, 333, mode, off=1)
    _product("bf16", 40, 70, 200, mode, off=1, pad=5, bias=False)


def test_product_forms_agree():
    """One answer, bit for bit, whatever kernel gives it."""
    got = [_product("f32", 200, 300, 777, mode) for mode in FORMS]
    for c in got[1:]:
        assert torch.equal(c.nan_to_num(1.0), got[0].nan_to_num(1.0))


def test_product_of_the_largest_sums():
    """128 * 128 * 131071: the last k's that a 32-bit sum holds."""
    K = 131071
    a = torch.full((2, 131072), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(2, dtype=torch.float32, device="cuda")
    for mode in FORMS:
        c = torch.empty(2, 2, dtype=torch.float32, device="cuda")
        R.revffn_op_gemm_int(0, mode, a, one, a.clone(), one, None, c, 2, 2, K, 131072, 131072, 2)
        torch.cuda.synchronize()
        assert (c == float(128 * 128 * K)).all()


def test_product_of_a_poisoned_row():
    x = torch.randn(5, 256, device="cuda")
    x[2, 17] = float("inf")
    codes, scale = torch.empty(5, 256, dtype=torch.int8, device="cuda"), torch.empty(5, dtype=torch.float32, device="cuda")
    R.revffn_op_quantize_rows(0, x, codes, scale, 5, 256, 256, 256)
    w, ws = torch.ones(40, 256, dtype=torch.int8, device="cuda"), torch.ones(40, dtype=torch.float32, device="cuda")
    c = torch.empty(5, 40, dtype=torch.float32, device="cuda")
    R.revffn_op_gemm_int(0, 0, codes, scale, w, ws, None, c, 5, 40, 256, 256, 256, 40)
    torch.cuda.synchronize()
    assert torch.isnan(c[2]).all() and torch.isfinite(c[[0, 1, 3, 4]]).all()


# ---- together --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_served_layer(dtype):
    """Projections as integer products, rotation and append, attention over the cache, the output projection: a prompt and then tokens, against
    the same layer in 64 bits.  Each step's own rounding is tested above; here the parts have to fit together, so what is compared is the
    layer's result with the reference fed by the stored numbers."""
    d, H, Hkv, dh, page = 256, 4, 2, 64, 32
    dt, t = 1 if dtype == "bf16" else 0, TORCH[dtype]
    rng = np.random.default_rng(4)
    width = (H + 2 * Hkv) * dh

    def weights(n, k):
        w = _normal(rng, "f32", n, k, scale=k ** -0.5)
        codes, scale = torch.empty(n, k, dtype=torch.int8, device="cuda"), torch.empty(n, dtype=torch.float32, device="cuda")
        R.revffn_op_quantize_rows(0, w, codes, scale, n, k, k, k)
        return codes, scale
    wqkv, sqkv = weights(width, d)
    wo, so = weights(d, H * dh)
    c = Paged(dtype, Hkv, dh, page, _tables(rng, [120, 75, 40], page))
    held = np.array([0, 0, 0])
    for new in ([90, 33, 1], [1, 1, 1], [20, 1, 30], [1, 1, 1]):
        held, T = held + new, sum(new)
        x = _normal(rng, dtype, T, d)

        def product(x, w, ws, n, k):
            codes, scale = torch.empty(T, k, dtype=torch.int8, device="cuda"), torch.empty(T, dtype=torch.float32, device="cuda")
            y = torch.empty(T, n, dtype=t, device="cuda")
            R.revffn_op_quantize_rows(dt, x, codes, scale, T, k, x.stride(0), k)
            R.revffn_op_gemm_int(dt, 0, codes, scale, w, ws, None, y, T, n, k, k, k, n)
            exact = (codes.double() @ w.double().t()) * scale.double()[:, None] * ws.double()
            assert (y.double() - exact).abs().max() <= exact.abs().max() * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -21)
            return y
        qkv = product(x, wqkv, sqkv, width, d)
        cache = c.cache(held, np.cumsum([0] + new))
        at = np.concatenate([np.arange(h - n, h) for h, n in zip(held, new)])
        key = ref.turned(_np(qkv[:, H * dh:(H + Hkv) * dh]).reshape(T, Hkv, dh), at, R.revffn_op_rotary_frequencies(_rotary(dh)))
        query = ref.turned(_np(qkv[:, :H * dh]).reshape(T, H, dh), at, R.revffn_op_rotary_frequencies(_rotary(dh)))
        value = qkv[:, (H + Hkv) * dh:]
        R.revffn_op_cache_append(dt, cache, _rotary(dh), None, qkv, qkv, qkv[:, H * dh:], value, T, H, width, width, width, width)
        c.model.append(c.table, list(held), new, _np(torch.from_numpy(key).float().to(t)), _np(value).reshape(T, Hkv, dh))
        o, lse = torch.empty(T, H * dh, dtype=t, device="cuda"), torch.empty(H, T, dtype=torch.float32, device="cuda")
        desc = R.AttnDesc(dtype=dt, H=H, Hkv=Hkv, dh=dh, Tq=T, ldq=width)
        work = torch.empty(R.revffn_op_attention_cached_workspace(desc, cache), dtype=torch.uint8, device="cuda")
        R.revffn_op_attention_cached(desc, cache, True, 0, qkv, o, lse, work)
        torch.cuda.synchronize()
        c.check()
        assert np.abs(_np(qkv[:, :H * dh]).reshape(T, H, dh) - query).max() <= np.abs(query).max() * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23)
        want = ref.attention(c.model, c.table, list(held), new, _np(qkv[:, :H * dh]).reshape(T, H, dh), dtype=dtype)
        assert outside(_np(o).reshape(T, H, dh), *want["o"]) <= 1.0 and outside(_np(lse), *want["lse"]) <= 1.0
        y = product(o, wo, so, d, H * dh)
        assert torch.isfinite(y).all()


# ---- calls at the ends of what is allowed ----------------------------------------------------------------------------
@MODES
@pytest.mark.parametrize("cap,bias", [(5000.0, False), (1e5, True), (1e6, False)])
def test_attention_caps_above_some_rows_scores(cap, bias, dtype, mode):
    """Rows whose scores are of order one beside rows whose scores reach a cap of thousands and more, in the same tiles: a score's error goes by its own
    size, not by the cap (the bounds' 8 half steps of each score)."""
    c = Paged(dtype, 1, 64, 32, [[2, 0, 1, 4, 3, 5], [7, 6, 8, 9, 10, 11]])
    _fill(c, [150, 70])
    a = Attend(c, [150, 70], [110, 2], 2, mode, scale=cap / 8, cap=cap, slopes=_slopes(2) if bias else None)
    a.q[1:112:2] *= 2.0 ** -round(np.log2(cap))
    a.run()
    a.check()


@MODES
@pytest.mark.parametrize("cap", [1e31, 3.4e38])
def test_attention_caps_without_end(cap, dtype, mode):
    """A cap near the type's largest value changes no score: the results are those without, single keys with negative scores among them."""
    held, new = [1, 1, 1, 1, 1, 40, 90], [1, 1, 1, 1, 1, 1, 60]
    c = Paged(dtype, 2, 64, 32, _tables(np.random.default_rng(1), held, 32))
    _fill(c, held)
    a = Attend(c, held, new, 4, mode, scale=0.3, cap=cap)
    a.run()
    a.check()


def test_quantize_rows_of_the_smallest_scales():
    """Scales just above 2^-126, where half of one may lie between two numbers: values a 2^-149 to both sides of each half."""
    rng = np.random.default_rng(11)
    unit, rows = 2.0 ** -149, 3000
    steps = 2 ** 23 + 2 * rng.integers(0, 2 ** 20, rows) + 1         # the scale: an odd number of 2^-149
    x = np.zeros((rows, 16))
    x[:, 0] = np.float32(127 * steps * unit)
    for i in range(7):
        for side in range(2):                                # (the two numbers around a half of the scale, or one and a half: exact, below 2^24 units)
            x[:, 1 + 2 * i + side] = ((steps * (1 + 2 * (i % 2)) // 2) + side) * unit * (-1) ** i
    x = torch.from_numpy(x.astype(np.float32)).cuda()
    codes, scale = torch.empty(rows, 16, dtype=torch.int8, device="cuda"), torch.empty(rows, dtype=torch.float32, device="cuda")
    R.revffn_op_quantize_rows(0, x, codes, scale, rows, 16, 16, 16)
    torch.cuda.synchronize()
    want, unit = ref.quantized(_np(x))
    assert np.array_equal(_np(scale), unit) and np.array_equal(codes.cpu().numpy(), want)


@pytest.mark.parametrize("mode", [2, 1])
def test_attention_of_more_than_two_to_the_24_rows(mode):
    """131075 rows of 128 heads: one sequence with nearly all, two with a few; every row against float32, spot rows against 64 bits."""
    H, Hkv, dh, page, held, new = 128, 2, 16, 16, [20, 40, 33], [1, 131072, 2]
    T, G = sum(new), H // Hkv
    c = Paged("bf16", Hkv, dh, page, _tables(np.random.default_rng(2), held, page), seed=12)
    _fill(c, held)
    q = torch.randn(T, H, dh, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    o, lse = torch.full_like(q, NAN), torch.full((H, T), NAN, dtype=torch.float32, device="cuda")
    cache = c.cache(held, np.cumsum([0] + new))
    desc = R.AttnDesc(dtype=1, kernel_mode=mode, H=H, Hkv=Hkv, dh=dh, Tq=T)
    work = torch.empty(R.revffn_op_attention_cached_workspace(desc, cache), dtype=torch.uint8, device="cuda")
    R.revffn_op_attention_cached(desc, cache, False, 0, q, o, lse, work)
    torch.cuda.synchronize()
    row = 0
    for s, n in enumerate(new):
        k, v = (torch.from_numpy(c.model.rows(x, c.table, s, held[s])).float().cuda() for x in "kv")
        for at in range(row, row + n, 16384):
            end = min(at + 16384, row + n)
            for h in range(Hkv):
                qq = q[at:end, h * G:(h + 1) * G].float().reshape(-1, dh)
                x = qq @ k[:, h].T.contiguous() / 4
                p = torch.softmax(x, -1)
                want, size = p @ v[:, h], p @ v[:, h].abs()
                # half a step of bfloat16 for the probabilities, one for the result; then float32's on both sides, scores (24 half steps of sums up to 6) and sums (56)
                bound = 2.0 ** -8 * (size + want.abs()) + 2.0 ** -14 * size
                got = o[at:end, h * G:(h + 1) * G].float().reshape(-1, dh)
                assert ((got - want).abs() <= bound).all(), (s, at, h)
                l = lse[h * G:(h + 1) * G, at:end].T.reshape(-1)
                assert ((l - torch.logsumexp(x, -1)).abs() <= 2.0 ** -14).all()
        row += n
    for i, s in ((0, 0), (1, 1), (77777, 1), (131072, 1), (131073, 2), (131074, 2)):
        want = ref.attention(c.model, c.table[s:s + 1], held[s:s + 1], [1], _np(q[i:i + 1]), causal=False)
        assert outside(_np(o[i:i + 1]), *want["o"]) <= 1.0 and outside(_np(lse[:, i:i + 1]), *want["lse"]) <= 1.0


def _among_many(at, n, held, new, table):
    """Lists of n sequences that hold nothing and get nothing, but for those at `at`."""
    many = np.full((n, table.shape[1]), -1)
    many[at] = table
    h, r = np.zeros(n, int), np.zeros(n, int)
    h[at], r[at] = held, new
    return _ints(many), _ints(h), _ints(np.concatenate([[0], np.cumsum(r)]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_among_a_million_sequences(dtype):
    """As many sequences as there may be, four of them with rows."""
    held, new, n = [20, 100, 5, 64], [1, 2, 1, 30], 2 ** 20
    c = Paged(dtype, 4, 64, 16, _tables(np.random.default_rng(3), held, 16))
    _fill(c, held)
    a = Attend(c, held, new, 8, 2)
    lists = _among_many([0, 77, 2 ** 19, n - 1], n, held, new, c.table)
    cache = R.Cache(c.k, c.v, c.ks, c.vs, *lists, pages=c.pages, page=16, max_pages=c.table.shape[1], n_seqs=n, Hkv=4, dh=64)
    work = torch.empty(R.revffn_op_attention_cached_workspace(a.desc, cache), dtype=torch.uint8, device="cuda")
    R.revffn_op_attention_cached(a.desc, cache, True, 0, a.q, a.o, a.lse, work)
    b = ref.attention(c.model, c.table, held, new, a.queries(), dtype=dtype)
    o, lse = a.results()
    assert torch.isnan(a.o[a.T:]).all() and torch.isnan(a.lse[:, a.T:]).all()
    assert outside(o, *b["o"]) <= 1.0 and outside(lse, *b["lse"]) <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_among_a_million_sequences(dtype):
    """As many sequences as there may be, four of them with rows: the cache and the queries of a call of those alone."""
    held, new, n, Hkv, H, dh = [20, 100, 5, 64], [1, 2, 1, 30], 2 ** 20, 4, 8, 64
    table, T = _tables(np.random.default_rng(4), held, 16), 34
    x = _normal(np.random.default_rng(5), dtype, T, (H + 2 * Hkv) * dh)
    w, out = x.stride(0), []
    for many in (False, True):
        c = Paged(dtype, Hkv, dh, 16, table, seed=6)
        _fill(c, [19, 98, 4, 34])                            # what is there already
        for t in (c.ks, c.vs):
            t.nan_to_num_(0)
        cache = c.cache(held, np.cumsum([0] + new))
        if many:
            lists = _among_many([0, 77, 2 ** 19, n - 1], n, held, new, table)
            cache = R.Cache(c.k, c.v, c.ks, c.vs, *lists, pages=c.pages, page=16, max_pages=table.shape[1], n_seqs=n, Hkv=Hkv, dh=dh)
        q = torch.full((T + 1, H * dh), NAN, dtype=TORCH[dtype], device="cuda")
        R.revffn_op_cache_append(1 if dtype == "bf16" else 0, cache, _rotary(dh), None, x, q, x[:, H * dh:], x[:, (H + Hkv) * dh:], T, H, w, H * dh, w, w)
        torch.cuda.synchronize()
        assert torch.isfinite(q[:T]).all() and torch.isnan(q[T:]).all()
        out.append((c.k, c.v, c.ks, c.vs, q[:T]))
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("M,N,K,mode", [(32768, 151936, 16, 0), (32768, 151936, 16, 256 * 4), (5000, 2 ** 20 + 7, 3, 1), (1, 2 ** 27 + 3, 16, 0), (3, 2 ** 27 + 1, 16, 2), (2 ** 27 + 33, 1, 16, 0)])
def test_product_of_more_than_two_to_the_32_results(M, N, K, mode):
    """Many rows by many columns, or one of them beyond what 32 by 32 tiles of a launch reach; every result: sums and scales are such that only the last rounding is one."""
    g = torch.Generator(device="cuda").manual_seed(M + K)
    ints = lambda n: torch.randint(-128, 128, (n, 16), generator=g, device="cuda", dtype=torch.int8)
    units = lambda n: torch.exp2(-torch.randint(0, 9, (n,), generator=g, device="cuda").float())
    a, b, sa, sb = ints(M), ints(N), units(M), units(N)
    c = torch.full((M, N), NAN, dtype=torch.bfloat16, device="cuda")
    R.revffn_op_gemm_int(1, mode, a, sa, b, sb, None, c, M, N, K, 16, 16, N)
    torch.cuda.synchronize()
    m = min(M, 1024)
    n = (1 << 27) // m
    for i in range(0, M, m):
        for j in range(0, N, n):
            x, y = a[i:i + m, :K].float() * sa[i:i + m, None], b[j:j + n, :K].float() * sb[j:j + n, None]
            assert torch.equal(c[i:i + m, j:j + n], (x @ y.T.contiguous()).to(torch.bfloat16)), (i, j)


# ---- whose rows are written, and the four calls in a graph -------------------------------------------------------------
# lengths, first rows of eight rows in a call, and (sequence, first row, rows) of those that are owned after numbers have been clamped
LISTS = [([-4, -2 ** 31, 2 ** 31 - 1], [0, 1, 3, 6], [(0, 0, 1), (1, 1, 2), (2, 3, 3)]), ([48, 48, 48], [100, -7, 2 ** 31 - 1, -1], [(1, 0, 8)]),
         ([48, 48, 48], [5, 4, 3, 2], []), ([0, 0, 0], [0, 0, 0, 0], []), ([30, 48, 20], [2, 2, 5, 2 ** 31 - 1], [(1, 2, 3), (2, 5, 3)])]


@MODES
@pytest.mark.parametrize("held,cu,owned", LISTS)
def test_attention_writes_the_rows_of_its_sequences(held, cu, owned, dtype, mode):
    """Exactly those, whatever the lists hold, and what they should be: lengths past the table see all of it, none sees nothing."""
    c = Paged(dtype, 2, 64, 16, [[0, 1, 2], [3, 4, 5], [6, 7, 8]])
    _fill(c, [48, 48, 48])
    a = Attend(c, [48, 48, 48], [2, 3, 3], 4, mode, extra=0)
    a.cache = c.cache(held, cu)
    a.run()
    o, lse = a.results()
    mine = np.zeros(8, bool)
    for s, first, n in owned:
        length = min(max(held[s], 0), 2 ** 30)
        want = ref.attention(c.model, c.table[s:s + 1], [length], [n], a.queries()[first:first + n], dtype=dtype)
        assert outside(o[first:first + n], *want["o"]) <= 1.0 and outside(lse[:, first:first + n], *want["lse"]) <= 1.0
        mine[first:first + n] = True
    assert np.isnan(o[~mine]).all() and np.isnan(lse[:, ~mine]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("held,cu,owned", LISTS)
def test_append_writes_the_rows_of_its_sequences(held, cu, owned, dtype):
    """Their queries, keys and values where they have a place, and nothing else."""
    Hkv, H, dh = 2, 4, 64
    c = Paged(dtype, Hkv, dh, 16, [[0, 1, 2], [3, 4, 5], [6, 7, 8]])
    _fill(c, [48, 48, 48])
    x = _normal(np.random.default_rng(9), dtype, 8, (H + 2 * Hkv) * dh)
    out = torch.full((8, H * dh), NAN, dtype=TORCH[dtype], device="cuda")
    w = x.stride(0)
    R.revffn_op_cache_append(1 if dtype == "bf16" else 0, c.cache(held, cu), None, None, x, out, x[:, H * dh:], x[:, (H + Hkv) * dh:], 8, H, w, H * dh, w, w)
    torch.cuda.synchronize()
    mine = np.zeros(8, bool)
    k, v = (_np(x[:, n * dh:(n + Hkv) * dh]).reshape(8, Hkv, dh) for n in (H, H + Hkv))
    for s, first, n in owned:
        length = min(max(held[s], 0), 2 ** 30)
        at = length - n + np.arange(n)
        mine[first:first + n] = (at >= 0) & (at < 48)
        c.model.append(c.table[s:s + 1], [length], [n], k[first:first + n], v[first:first + n])
    c.check()
    mine = torch.from_numpy(mine).cuda()
    assert torch.equal(out[mine], x[mine][:, :H * dh]) and torch.isnan(out[~mine]).all()


@pytest.mark.parametrize("mode", [0] + FORMS[2:])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graph_replays_of_a_layer(dtype, mode):
    """All four calls captured once and replayed as the sequences grow: every replay equals the same calls made eagerly on a cache of its own, with eager
    work between the replays."""
    d, page, Hkv, H, dh, S = 256, 16, 2, 4, 64, 3
    table, held0 = [[0, 1, 2, 3], [4, 5, 6, 7], [8, 9, 10, 11]], np.array([5, 15, 31])
    rng, t, dt, width = np.random.default_rng(10), TORCH[dtype], 1 if dtype == "bf16" else 0, (H + 2 * Hkv) * dh
    new = lambda *s, ty=t: torch.full(s, 1, dtype=ty, device="cuda")
    ints = lambda n, k: (torch.from_numpy(rng.integers(-127, 128, (n, k)).astype(np.int8)).cuda(), torch.from_numpy(rng.uniform(1e-4, 1e-3, n).astype(np.float32)).cuda())
    (wqkv, sqkv), (wo, so) = ints(width, d), ints(d, H * dh)
    x, r, desc = new(S, d), _rotary(dh), R.AttnDesc(dtype=dt, H=H, Hkv=Hkv, dh=dh, Tq=S, ldq=width)
    k, v = rng.standard_normal((2, held0.sum(), Hkv, dh))

    class Layer:
        def __init__(self):
            self.c = Paged(dtype, Hkv, dh, page, table)
            _fill(self.c, held0, k, v)
            self.cache, self.held = self.c.cache(held0, None), self.c.lists[1]
            self.work = torch.empty(R.revffn_op_attention_cached_workspace(desc, self.cache), dtype=torch.uint8, device="cuda")
            self.codes, self.scale, self.qkv, self.o, self.y = new(S, d, ty=torch.int8), new(S, ty=torch.float32), new(S, width), new(S, H * dh), new(S, d)
            self.lse = new(H, S, ty=torch.float32)

        def step(self):
            qkv = self.qkv
            R.revffn_op_quantize_rows(dt, x, self.codes, self.scale, S, d, d, d)
            R.revffn_op_gemm_int(dt, mode, self.codes, self.scale, wqkv, sqkv, None, qkv, S, width, d, d, d, width)
            R.revffn_op_cache_append(dt, self.cache, r, None, qkv, qkv, qkv[:, H * dh:], qkv[:, (H + Hkv) * dh:], S, H, width, width, width, width)
            R.revffn_op_attention_cached(desc, self.cache, True, 0, qkv, self.o, self.lse, self.work)
            R.revffn_op_quantize_rows(dt, self.o, self.codes, self.scale, S, H * dh, H * dh, d)
            R.revffn_op_gemm_int(dt, mode, self.codes, self.scale, wo, so, None, self.y, S, d, H * dh, d, H * dh, d)
    a, b = Layer(), Layer()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            a.step()
    torch.cuda.synchronize()
    for _ in range(5):
        x.copy_(_normal(rng, dtype, S, d))
        for layer in (a, b):
            layer.held.add_(1)
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        for n in ("codes", "scale", "qkv", "o", "lse", "y"):
            p, q = getattr(a, n), getattr(b, n)
            assert torch.equal(p, q) and torch.isfinite(p.float()).all(), n
        assert torch.equal(a.c.k, b.c.k) and torch.equal(a.c.v, b.c.v) and torch.equal(a.c.ks.nan_to_num(0), b.c.ks.nan_to_num(0))
        torch.randn(1000, device="cuda").sum().item()
