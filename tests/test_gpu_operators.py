"""The operators for attention layers through the C ABI, each against float64 with bounds from the arithmetic."""
import numpy as np
import pytest
import torch

import operators_reference as ref

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2512_20920_amd as R

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN = float("nan")


def _rand(rng, shape, dtype, scale=1.0):
    return torch.from_numpy((scale * rng.standard_normal(shape)).astype(np.float32)).to(TORCH[dtype])


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _ints(a):
    return torch.from_numpy(np.asarray(a)).to("cuda", torch.int32)


class Attention:
    """One call's tensors; q, k, v may be parts of wider rows, and rows past `used` hold NaN."""

    def __init__(self, dtype, H, Hkv, dh, Tq, Tk, seed=0, pad=0, extra_rows=0, scale=1.0):
        rng = np.random.default_rng(seed + 31 * Tq + 7 * Tk + dh + H)
        self.dtype, self.H, self.Hkv, self.dh, self.Tq, self.Tk = dtype, H, Hkv, dh, Tq, Tk
        self.rows_q, self.rows_k = Tq + extra_rows, Tk + extra_rows

        def rows(n, used, heads, sc=1.0, fill=NAN):
            wide = torch.full((n, heads * dh + pad), fill, dtype=TORCH[dtype], device="cuda")
            wide[:used, : heads * dh] = _rand(rng, (used, heads * dh), dtype, sc).cuda()
            return wide
        self.q, self.k, self.v = rows(self.rows_q, Tq, H, scale), rows(self.rows_k, Tk, Hkv, scale), rows(self.rows_k, Tk, Hkv)
        self.do = rows(self.rows_q, Tq, H)
        self.o, self.dq = torch.full_like(self.q, NAN), torch.full_like(self.q, NAN)
        self.dk, self.dv = torch.full_like(self.k, NAN), torch.full_like(self.v, NAN)
        self.lse = torch.full((H, self.rows_q), NAN, dtype=torch.float32, device="cuda")

    def part(self, name):
        """[rows in use, heads, dh] of a tensor in float64."""
        n, heads = (self.Tk, self.Hkv) if name in ("k", "v", "dk", "dv") else (self.Tq, self.H)
        return _np(getattr(self, name)[:n, : heads * self.dh].reshape(n, heads, self.dh))

    def run(self, lo, hi, at=None, mode=0, backward=True, cap=0.0, slopes=None, scale=0.0, used=False, stream=None):
        self.slopes = None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device="cuda")
        wide = lambda t: t.stride(0)
        self.desc = R.AttnDesc(dtype=1 if self.dtype == "bf16" else 0, kernel_mode=mode, H=self.H, Hkv=self.Hkv, dh=self.dh, Tq=self.rows_q,
                               Tk=self.rows_k, ldq=wide(self.q), ldk=wide(self.k), ldv=wide(self.v), ldo=wide(self.o), scale=scale, softcap=cap,
                               slopes=self.slopes)
        full = lambda a, n: _ints(np.concatenate([a, np.zeros(n - len(a), int)]))
        self.mask = R.AttnMask(full(lo, self.rows_q), full(hi, self.rows_q), None if at is None else full(at, self.rows_q),
                               _ints([self.Tq, self.Tk]) if used else None)
        n = R.revffn_op_attention_masked_workspace(self.desc, backward)
        self.work = torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")        # NaN patterns throughout
        R.revffn_op_attention_masked_fwd(self.desc, self.mask, self.q, self.k, self.v, self.o, self.lse, self.work, stream=stream)
        if backward:
            R.revffn_op_attention_masked_bwd(self.desc, self.mask, self.q, self.k, self.v, self.o, self.do, self.lse, self.dq, self.dk, self.dv,
                                             self.work, stream=stream)
        torch.cuda.synchronize()

    def check(self, lo, hi, at=None, backward=True, cap=0.0, slopes=None, scale=None):
        sl = None if slopes is None else np.asarray(slopes, np.float32).astype(np.float64)
        want = ref.attention(self.part("q"), self.part("k"), self.part("v"), lo, hi, at, scale, cap, sl,
                             self.part("do") if backward else None, self.dtype)
        got = {"o": self.part("o"), "lse": _np(self.lse[:, : self.Tq])}
        if backward:
            got |= {"dq": self.part("dq"), "dk": self.part("dk"), "dv": self.part("dv")}
        worst = {name: ref.outside(got[name], *want[name]) for name in got}
        assert max(worst.values()) <= 1.0, worst


def _slopes(H):
    return 2.0 ** (-8.0 * (np.arange(H) + 1) / H)


# name: heads, key heads, width, query documents, key documents (None: the same), options
SHAPES = {
    "one_token": (2, 2, 64, [1], None, {}),
    "one_key_each": (4, 2, 128, [1, 1, 1], None, {}),
    "packed": (4, 2, 128, [37, 1, 130, 64, 5, 0, 66], None, {}),
    "packed_both_ways": (3, 3, 64, [70, 3, 150], None, dict(causal=False)),
    "long": (2, 1, 128, [517], None, {}),
    "window": (4, 1, 64, [300, 77], None, dict(window=33)),
    "window_of_one": (2, 2, 64, [100], None, dict(window=1)),
    "prefix": (2, 2, 128, [200, 90], None, dict(prefix=[77, 200])),
    "capped": (4, 4, 64, [140, 61], None, dict(cap=5.0)),
    "biased": (4, 2, 128, [140, 61], None, dict(bias=True)),
    "capped_biased_prefix": (6, 2, 64, [129, 200], None, dict(cap=30.0, bias=True, prefix=[100, 0])),
    "capped_wide": (2, 2, 128, [140, 61], None, dict(cap=5.0)),
    "capped_biased_wide": (4, 1, 128, [200, 30], None, dict(cap=8.0, bias=True)),
    "biased_narrow": (4, 2, 64, [140, 61], None, dict(bias=True)),
    "behind_a_cache": (4, 2, 64, [40, 7, 129], [300, 7, 500], dict(bias=True)),
    "more_queries_than_keys": (2, 1, 64, [50, 20], [20, 20], {}),
    "no_keys": (2, 1, 64, [20, 30], [0, 30], dict(causal=False)),
    "width_32": (2, 1, 32, [70, 65], None, {}),
    "width_80": (3, 1, 80, [70, 65], None, dict(cap=20.0)),
    "width_96": (2, 2, 96, [150], None, {}),
    "width_120": (2, 1, 120, [33, 100], None, {}),
    "width_odd": (2, 1, 33, [40, 35], None, dict(bias=True)),
    "width_256": (2, 1, 256, [40, 35], None, {}),
    "width_500": (1, 1, 500, [70], None, {}),
    "many_heads_to_one": (16, 1, 64, [65, 64], None, {}),
    "forty_heads_to_one": (40, 1, 64, [3, 30], [3, 300], {}),
    "three_heads_to_one": (6, 2, 128, [30, 11], [70, 11], {}),
    "next_tokens": (8, 2, 128, [1] * 9, [212, 37, 1001, 450, 1, 777, 128, 0, 1500], {}),
    "next_tokens_capped": (4, 4, 64, [1] * 40, [(37 * i) % 111 for i in range(40)], dict(cap=10.0, bias=True)),
    "next_token_of_one": (2, 1, 80, [1], [2500], dict(bias=True)),
    "few_new_tokens": (4, 2, 128, [3, 4, 1], [900, 4, 33], {}),
}


def _case(name):
    H, Hkv, dh, q_lens, k_lens, opt = SHAPES[name]
    opt = dict(opt)
    cap, slopes = opt.pop("cap", 0.0), _slopes(H) if opt.pop("bias", False) else None
    lo, hi, at = ref.ranges(q_lens, k_lens, **opt)
    return H, Hkv, dh, sum(q_lens), sum(k_lens or q_lens), lo, hi, at, dict(cap=cap, slopes=slopes)


@pytest.mark.parametrize("dtype,mode", [("bf16", 1), ("bf16", 256), ("bf16", 512), ("f32", 0), ("f32", 1)])
@pytest.mark.parametrize("name", list(SHAPES))
def test_attention(name, mode, dtype):
    H, Hkv, dh, Tq, Tk, lo, hi, at, opt = _case(name)
    a = Attention(dtype, H, Hkv, dh, Tq, Tk)
    a.run(lo, hi, at, mode, **opt)
    a.check(lo, hi, at, **opt)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,mode", [(8, 0), (64, 0), (3, 0), (3, 1)])
def test_attention_strides_and_rows_behind_the_last_document(pad, mode, dtype):
    """q, k, v inside wider rows; the rows behind the last document hold NaN and their results stay as they were."""
    H, Hkv, dh, Tq, Tk, lo, hi, at, opt = _case("packed")
    a = Attention(dtype, H, Hkv, dh, Tq, Tk, pad=pad, extra_rows=70)
    a.run(lo, hi, at, mode, used=True, **opt)
    a.check(lo, hi, at, **opt)
    for t, n, heads in ((a.o, Tq, H), (a.dq, Tq, H), (a.dk, Tk, Hkv), (a.dv, Tk, Hkv)):
        assert torch.isnan(t[n:]).all() and torch.isnan(t[:, heads * dh:]).all()
    assert torch.isnan(a.lse[:, Tq:]).all()


@pytest.mark.parametrize("dtype,mode", [("bf16", 1), ("bf16", 256), ("bf16", 512), ("f32", 0), ("f32", 1)])
def test_attention_any_ranges(mode, dtype):
    """Ranges that no documents make, out of bounds ones among them, and queries that see nothing."""
    rng = np.random.default_rng(5)
    n, m = 203, 331
    lo, hi = rng.integers(-50, m, n), rng.integers(0, m + 50, n)
    lo[7], hi[7], lo[8], hi[8] = 5, 5, 2 ** 31 - 1, -2 ** 31
    hi[64:96] = lo[64:96]                                   # a whole tile of queries without keys
    cl, ch = np.maximum(lo, 0), np.minimum(hi, m)
    a = Attention(dtype, 4, 2, 64, n, m)
    a.run(lo, hi, np.arange(n), mode)
    a.check(cl, ch)
    none = cl >= ch
    assert none.sum() > 32 and (a.part("o")[none] == 0).all() and (a.part("dq")[none] == 0).all()
    assert torch.isneginf(a.lse[:, torch.from_numpy(none).cuda()]).all()


@pytest.mark.parametrize("dtype,mode", [("bf16", 1), ("bf16", 256), ("bf16", 512), ("f32", 0), ("f32", 1)])
@pytest.mark.parametrize("value", [NAN, float("inf"), float("-inf")])
def test_attention_values_that_are_not_finite_stay_where_they_are(value, mode, dtype):
    """One document's rows hold NaN or infinities, in each tensor by turns: the other documents' results are what they are
    without, in every tile that two documents share."""
    lens = [45, 30, 70, 100]
    lo, hi, at = ref.ranges(lens)
    inside = np.zeros(sum(lens), bool)
    inside[45:75] = True
    for where in ("q", "k", "v", "do"):
        a = Attention(dtype, 2, 1, 64, sum(lens), sum(lens))
        clean = Attention(dtype, 2, 1, 64, sum(lens), sum(lens))
        getattr(a, where)[50] = value
        a.run(lo, hi, at, mode)
        clean.run(lo, hi, at, mode)
        clean.check(lo, hi, at)
        for name in ("o", "dq", "dk", "dv"):
            got, want = a.part(name)[~inside], clean.part(name)[~inside]
            # (a tile worked out again adds in another order: both are within the bounds, so at most two of them apart)
            bound = ref.attention(clean.part("q"), clean.part("k"), clean.part("v"), lo, hi, at, do=clean.part("do"), dtype=dtype)[name][1][~inside]
            assert ref.outside(got, want, 2 * bound) <= 1.0, (where, name)
        row = a.part("o")[50]
        if where in ("k", "v"):
            assert not np.isfinite(row).all()               # and who sees it, gets it


@pytest.mark.parametrize("dtype,mode", [("bf16", 1), ("bf16", 256), ("bf16", 512), ("f32", 0)])
@pytest.mark.parametrize("scale,cap", [(0.3, 0.0), (-0.2, 0.0), (-0.2, 3.0), (1e-3, 0.5)])
def test_attention_scales(scale, cap, mode, dtype):
    lo, hi, at = ref.ranges([70, 40])
    a = Attention(dtype, 2, 1, 64, 110, 110)
    a.run(lo, hi, at, mode, cap=cap, scale=scale)
    a.check(lo, hi, at, cap=cap, scale=scale)


@pytest.mark.parametrize("dtype,mode", [("bf16", 256), ("bf16", 512), ("f32", 0)])
def test_attention_far_apart(mode, dtype):
    """Queries next to each other whose keys lie far apart: what nobody sees between is left out."""
    n, m = 70, 40000
    lo = np.where(np.arange(n) % 2 == 0, 3, m - 130)
    lo[40:] = 20000 + np.arange(30)
    hi = lo + 1 + np.arange(n) % 97
    a = Attention(dtype, 2, 1, 64, n, m)
    a.run(lo, hi, None, mode)
    a.check(lo, hi)


def test_attention_ranges():
    for q_lens, k_lens, kw in [([3, 0, 5, 1], None, {}), ([3, 0, 5, 1], None, dict(causal=False)), ([1, 1], [700, 3], {}),
                               ([4, 9], [2, 20], dict(prefix=[1, 30])), ([300, 9], None, dict(window=7))]:
        n, m = sum(q_lens), sum(k_lens or q_lens)
        lo, hi, at = ref.ranges(q_lens, k_lens, Tq=n + 5, **kw)
        new = lambda k: torch.full((k,), -7, dtype=torch.int32, device="cuda")
        dl, dh, da, du = new(n + 5), new(n + 5), new(n + 5), new(2)
        cum = lambda l: _ints(np.cumsum([0] + l))
        R.revffn_op_attention_ranges(cum(q_lens), None if k_lens is None else cum(k_lens), _ints(kw["prefix"]) if "prefix" in kw else None, len(q_lens),
                                     kw.get("causal", True), kw.get("window", 0), n + 5, m + 9, dl, dh, da, du)
        torch.cuda.synchronize()
        assert dl.tolist() == list(lo) and dh.tolist() == list(hi) and du.tolist() == [n, m]
        assert da[:n].tolist() == list(at[:n])
    # equal documents without a table, with and without one for the keys
    lo, hi, at = ref.ranges([4, 4, 4], [7, 7, 7])
    dl, dh = torch.empty(12, dtype=torch.int32, device="cuda"), torch.empty(12, dtype=torch.int32, device="cuda")
    for cu_k in (None, _ints([0, 7, 14, 21])):
        R.revffn_op_attention_ranges(None, cu_k, None, 3, True, 0, 12, 21, dl, dh)
        torch.cuda.synchronize()
        assert dl.tolist() == list(lo) and dh.tolist() == list(hi)
    # rows out of bounds in the table: everything clamped
    R.revffn_op_attention_ranges(_ints([-3, 6, 40]), _ints([-9, 5, 2 ** 31 - 1]), None, 2, False, 0, 12, 21, dl, dh)
    torch.cuda.synchronize()
    assert dl.min() >= 0 and dh.max() <= 21


@pytest.mark.parametrize("docs", [1022, 1023, 1024, 1025, 5000])
def test_attention_ranges_of_many_documents(docs):
    rng = np.random.default_rng(docs)
    q_lens, more = rng.integers(0, 5, docs), rng.integers(0, 3, docs)
    cum = lambda l: _ints(np.cumsum(np.concatenate([[0], l])))
    for k_lens, kw in ((q_lens, {}), (q_lens + more, {}), (q_lens, dict(window=2)), (q_lens + more, dict(prefix=rng.integers(0, 4, docs).tolist()))):
        n, m = int(q_lens.sum()), int(k_lens.sum())
        lo, hi, at = ref.ranges(q_lens.tolist(), k_lens.tolist(), **kw)
        dl, dh, da, du = (torch.full((k,), -7, dtype=torch.int32, device="cuda") for k in (n, n, n, 2))
        R.revffn_op_attention_ranges(cum(q_lens), None if k_lens is q_lens else cum(k_lens), _ints(kw["prefix"]) if "prefix" in kw else None, docs, True,
                                     kw.get("window", 0), n, m, dl, dh, da, du)
        torch.cuda.synchronize()
        assert dl.tolist() == list(lo) and dh.tolist() == list(hi) and da.tolist() == list(at) and du.tolist() == [n, m]


def test_attention_ranges_of_no_queries():
    used = torch.full((2,), -7, dtype=torch.int32, device="cuda")
    nothing = torch.empty(0, dtype=torch.int32, device="cuda")
    for cu_q, cu_k, Tk, want in [(_ints([0, 0, 0]), _ints([0, 3, 5]), 9, [0, 5]), (None, None, 8, [0, 8]), (_ints([0, 0, 0]), None, 9, [0, 0])]:
        used.fill_(-7)
        R.revffn_op_attention_ranges(cu_q, cu_k, None, 2, True, 0, 0, Tk, nothing, nothing, nothing, used)
        torch.cuda.synchronize()
        assert used.tolist() == want


FORMS = pytest.mark.parametrize("dtype,mode", [("bf16", 1), ("bf16", 256), ("bf16", 512), ("f32", 0)])


@FORMS
@pytest.mark.parametrize("scale", [4.0, 40.0])
def test_attention_peaked(scale, mode, dtype):
    """Scores of hundreds: one key takes nearly all of a query's weight, and maxima rise late."""
    lo, hi, at = ref.ranges([150, 70])
    a = Attention(dtype, 2, 1, 64, 220, 220)
    a.run(lo, hi, at, mode, scale=scale)
    a.check(lo, hi, at, scale=scale)


@FORMS
@pytest.mark.parametrize("cap", [1.0, 3000.0, 1e6])
def test_attention_caps(cap, mode, dtype):
    lo, hi, at = ref.ranges([60, 45])
    a = Attention(dtype, 2, 1, 64, 105, 105)
    a.run(lo, hi, at, mode, cap=cap)
    a.check(lo, hi, at, cap=cap)


@FORMS
@pytest.mark.parametrize("dh", [64, 128])
def test_attention_bias_that_grows_with_the_distance(dh, mode, dtype):
    """Negative slopes: scores rise to hundreds away from the query, also where no query is (the rows behind the last one)."""
    lens = [3, 430, 8]
    lo, hi, at = ref.ranges(lens)
    a = Attention(dtype, 2, 1, dh, sum(lens), sum(lens), extra_rows=20)
    a.run(lo, hi, at, mode, slopes=[-1.0, -0.5], used=True)
    a.check(lo, hi, at, slopes=[-1.0, -0.5])


@FORMS
@pytest.mark.parametrize("where,value", [("k", NAN), ("q", float("inf")), ("v", float("-inf"))])
def test_attention_not_finite_beside_long_documents(where, value, mode, dtype):
    """A short document's value that is not finite between two whose keys (or queries) are split over workgroups, rows behind the last."""
    lens = [333, 40, 500]
    lo, hi, at = ref.ranges(lens)
    inside = np.zeros(sum(lens), bool)
    inside[333:373] = True
    a, clean = (Attention(dtype, 4, 2, 64, sum(lens), sum(lens), extra_rows=40) for _ in range(2))
    getattr(a, where)[350] = value
    a.run(lo, hi, at, mode, used=True)
    clean.run(lo, hi, at, mode, used=True)
    clean.check(lo, hi, at)
    bounds = ref.attention(clean.part("q"), clean.part("k"), clean.part("v"), lo, hi, at, do=clean.part("do"), dtype=dtype)
    for name in ("o", "dq", "dk", "dv"):
        assert ref.outside(a.part(name)[~inside], clean.part(name)[~inside], 2 * bounds[name][1][~inside]) <= 1.0, name
    assert torch.isnan(a.dq[sum(lens):]).all() and torch.isnan(a.dk[sum(lens):]).all()


@FORMS
def test_attention_not_finite_where_it_is_seen(mode, dtype):
    """A NaN that queries see is in their results and in no others (and the call ends)."""
    lo, hi, at = ref.ranges([100, 200])
    a = Attention(dtype, 2, 2, 128, 300, 300)
    a.v[150, :128] = NAN                                    # of the first head
    a.run(lo, hi, at, mode)
    o = a.part("o")
    assert np.isnan(o[150:, 0]).all() and np.isfinite(o[:150]).all() and np.isfinite(o[:, 1]).all()
    dk = a.part("dk")
    assert np.isfinite(dk[:100]).all() and np.isfinite(dk[:, 1]).all()


@pytest.mark.parametrize("mode", [256, 512])
@pytest.mark.parametrize("dh", [64, 128])
# root mean square errors as multiples of those of the float64 result rounded once to its type; the lines lie between what three seeds of these
# inputs give with a correction and without it:
#   biased: 16 bits of dS and the sum of dS in D: dq 1.08..1.14, 1.48..1.52 without
#   short: D summed from the tile that holds all keys of a query: dq, dk 1.39..1.50, 1.63..1.76 without
#   capped: the forward pass's tanh from a polynomial (float32 lse): 1.67..1.90, 3.99..4.56 without
@pytest.mark.parametrize("kind,names,most", [("biased", ("dq",), 1.3), ("short", ("dq", "dk"), 1.57), ("capped", ("lse",), 2.75)])
def test_attention_errors_stay_near_a_single_rounding(kind, names, most, dh, mode):
    H, Hkv, lens, opt = {"biased": (4, 2, [140, 61, 300], dict(slopes=_slopes(4))), "capped": (2, 2, [140, 61], dict(cap=30.0)),
                         "short": (4, 2, [30, 17, 1, 25, 9, 3, 31, 12, 28, 5, 22, 16, 2, 30, 19], {})}[kind]
    lo, hi, at = ref.ranges(lens)
    a = Attention("bf16", H, Hkv, dh, sum(lens), sum(lens))
    a.run(lo, hi, at, mode, **opt)
    want = ref.attention(a.part("q"), a.part("k"), a.part("v"), lo, hi, at, cap=opt.get("cap", 0.0), slopes=opt.get("slopes"), do=a.part("do"))
    for name in names:
        x = want[name][0]
        once = x.astype(np.float32) if name == "lse" else _np(torch.from_numpy(x).to(torch.bfloat16))
        got = _np(a.lse) if name == "lse" else a.part(name)
        assert np.sqrt(((got - x) ** 2).mean()) <= most * np.sqrt(((once - x) ** 2).mean()), name


def _check_in_parts(a, lo, hi, at=None, cap=0.0, slopes=None, rows=64):
    """Attention.check for many rows: `rows` queries at a time against the keys that they see.  (Errors of dk's and dv's parts add up.)"""
    lo, hi, at = np.asarray(lo), np.asarray(hi), np.arange(len(lo)) if at is None else np.asarray(at)
    q, k, v, do = (a.part(x) for x in ("q", "k", "v", "do"))
    want = {n: [np.zeros(shape), np.zeros(shape)] for n, shape in (("o", q.shape), ("dq", q.shape), ("dk", k.shape), ("dv", k.shape))}
    want["lse"] = [np.full((a.H, a.Tq), -np.inf), np.zeros((a.H, a.Tq))]
    for i in range(0, a.Tq, rows):
        r = slice(i, min(i + rows, a.Tq))
        some = lo[r] < hi[r]
        if not some.any():
            continue
        c = slice(lo[r][some].min(), hi[r][some].max())
        part = ref.attention(q[r], k[c], v[c], np.maximum(lo[r] - c.start, 0), hi[r] - c.start, at[r] - c.start, cap=cap, slopes=slopes, do=do[r], dtype=a.dtype)
        for j in range(2):
            for name in ("o", "dq"):
                want[name][j][r] = part[name][j]
            want["lse"][j][:, r] = part["lse"][j]
            for name in ("dk", "dv"):
                want[name][j][c] += part[name][j]
    got = {n: a.part(n) for n in ("o", "dq", "dk", "dv")} | {"lse": _np(a.lse[:, : a.Tq])}
    worst = {name: ref.outside(got[name], *want[name]) for name in got}
    assert max(worst.values()) <= 1.0, worst


BY_SIZE = pytest.mark.parametrize("dtype,mode", [("bf16", 0), ("bf16", 256), ("bf16", 512), ("f32", 0)])


@BY_SIZE
@pytest.mark.parametrize("H,Hkv,dh,cap", [(2, 2, 64, 0.0), (3, 1, 64, 0.0), (4, 1, 128, 0.0), (6, 2, 128, 20.0)])
def test_attention_keys_seen_from_far_apart_blocks(H, Hkv, dh, cap, mode, dtype):
    """More than 64 blocks of 64 queries.  Each query sees some hundred keys, its own neighbours or, a few whole blocks of queries, the first ones: a block
    that is left out or taken twice is a large part of a key's gradients."""
    n = 4700
    i = np.arange(n)
    lo, hi = np.maximum(i - 100, 0), i + 1
    first = np.isin(i // 64, [30, 63, 64, 66, 70, 73])
    lo[first], hi[first] = 0, 50 + i[first] % 13
    a = Attention(dtype, H, Hkv, dh, n, n)
    a.run(lo, hi, None, mode, cap=cap)
    _check_in_parts(a, lo, hi, cap=cap)


# rows, heads, key heads, width: which form each kernel takes goes by these, on both sides of each line and with the forms of dq and of dk, dv apart;
# 1500 x 32: between 256 and 512 workgroups in the form for many rows, whose second 256 take their tiles in the other order
@BY_SIZE
@pytest.mark.parametrize("T,H,Hkv,dh", [(1500, 32, 32, 64), (1500, 32, 32, 128), (2048, 16, 16, 128), (2049, 16, 16, 128), (3000, 16, 8, 128), (2000, 16, 4, 64),
                                        (4500, 16, 16, 64), (3000, 24, 8, 64), (1500, 24, 8, 64), (2600, 16, 16, 128), (1900, 9, 3, 64)])
def test_attention_sizes_around_the_lines(T, H, Hkv, dh, mode, dtype):
    rng = np.random.default_rng(T + H)
    lens = []
    while sum(lens) < T:
        lens.append(min(int(rng.integers(1, 200)), T - sum(lens)))
    lo, hi, at = ref.ranges(lens)
    a = Attention(dtype, H, Hkv, dh, T, T)
    a.run(lo, hi, at, mode)
    _check_in_parts(a, lo, hi, at)


@FORMS
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("where", ["q", "k"])
def test_attention_queries_whose_scores_are_all_minus_infinity(where, dh, mode, dtype):
    """Such a query counts as one that sees nothing, whole tiles of keys (queries) among them: the results are those of empty ranges."""
    lens = [128, 320, 64]                                   # (so that blocks of queries see the tiles of keys whole)
    lo, hi, at = ref.ranges(lens, causal=False)
    T = sum(lens)
    a = Attention(dtype, 4, 4, dh, T, T)
    for h in range(4):                                      # column 0 of every head is positive: an infinity there makes no 0 * infinity
        a.q[:, h * dh] = a.q[:, h * dh].abs() + 0.5
        a.k[:, h * dh] = a.k[:, h * dh].abs() + 0.5
    none = np.zeros(T, bool)
    if where == "q":
        none[[0, 127, 170, 300, 447, 500]] = True
        a.q[torch.from_numpy(none).cuda(), ::dh] = float("-inf")
    else:
        none[128:448] = True
        a.k[128:448, ::dh] = float("-inf")
    a.run(lo, hi, at, mode)
    a.check(np.where(none, 0, lo), np.where(none, 0, hi))
    assert torch.isneginf(a.lse[:, torch.from_numpy(none).cuda()]).all()


@FORMS
def test_attention_same_bits_again(mode, dtype):
    lo, hi, at = ref.ranges([300, 211])
    runs = []
    for _ in range(2):
        a = Attention(dtype, 4, 2, 64, 511, 511)
        a.run(lo, hi, at, mode, slopes=_slopes(4))
        runs.append([t.clone() for t in (a.o, a.lse, a.dq, a.dk, a.dv)])
    assert all(torch.equal(x, y) for x, y in zip(*runs))


@FORMS
def test_attention_without_queries_or_keys(mode, dtype):
    a = Attention(dtype, 2, 1, 64, 0, 40)
    a.run(np.zeros(0, int), np.zeros(0, int), None, mode)
    assert (a.part("dk") == 0).all() and (a.part("dv") == 0).all()
    a = Attention(dtype, 2, 1, 64, 40, 0)
    a.run(np.zeros(40, int), np.full(40, 9), None, mode)
    assert (a.part("o") == 0).all() and (a.part("dq") == 0).all() and torch.isneginf(a.lse).all()
    a = Attention(dtype, 2, 1, 64, 70, 70, extra_rows=5)           # rows there, none in use
    a.Tq = a.Tk = 0
    a.run(np.zeros(75, int), np.full(75, 9), None, mode, used=True)
    assert all(torch.isnan(t).all() for t in (a.o, a.dq, a.dk, a.dv, a.lse))


@FORMS
def test_attention_tensors_that_start_anywhere(mode, dtype):
    """Rows that start one element after an aligned address go to kernels that take them."""
    lo, hi, at = ref.ranges([60, 45])
    a = Attention(dtype, 2, 1, 64, 105, 105, pad=8)
    for name in ("q", "k", "v", "do", "o", "dq", "dk", "dv"):
        t = getattr(a, name)
        room = torch.full((t.numel() + 1,), NAN, dtype=t.dtype, device="cuda")
        room[1:] = t.reshape(-1)
        setattr(a, name, room[1:].reshape(t.shape))
    a.run(lo, hi, at, mode)
    a.check(lo, hi, at)


@pytest.mark.parametrize("dtype,mode", [("bf16", 1), ("bf16", 256), ("bf16", 512), ("f32", 0)])
def test_attention_offsets_past_32_bits(mode, dtype):
    """Rows so far apart that keys, values and queries lie more than 2^32 bytes (and elements) behind the first."""
    n, H, dh, apart = 530, 2, 64, (1 << 23) + 8
    rng = np.random.default_rng(1)
    big = {name: torch.empty(n * apart, dtype=TORCH[dtype], device="cuda") for name in ("q", "k", "v", "do", "o", "dq", "dk", "dv")}
    a = Attention(dtype, H, H, dh, n, n)
    for name, t in big.items():
        rows = t.as_strided((n, H * dh), (apart, 1))
        if name in ("q", "k", "v", "do"):
            rows.copy_(getattr(a, name))
        setattr(a, name, rows)
    lo, hi, at = ref.ranges([100, 430])
    a.run(lo, hi, at, mode)
    a.check(lo, hi, at)


def test_attention_single_token_far_along_a_cache_past_4_gib():
    """One query each of two sequences in a cache of 2^22 key rows, 4 GiB a tensor: the last keys count as the first do."""
    rows, Hkv, H, dh = 1 << 22, 4, 16, 128
    k = torch.randn(rows, Hkv * dh, dtype=torch.bfloat16, device="cuda")
    v = torch.randn(rows, Hkv * dh, dtype=torch.bfloat16, device="cuda")
    q = torch.randn(2, H * dh, dtype=torch.bfloat16, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(H, 2, device="cuda")
    d = R.AttnDesc(dtype=1, H=H, Hkv=Hkv, dh=dh, Tq=2, Tk=rows)
    lo, hi = [rows - 700, 5], [rows, 805]
    work = torch.empty(R.revffn_op_attention_masked_workspace(d, False), dtype=torch.uint8, device="cuda")
    R.revffn_op_attention_masked_fwd(d, R.AttnMask(_ints(lo), _ints(hi)), q, k, v, o, lse, work)
    torch.cuda.synchronize()
    for i in range(2):
        part = lambda t: _np(t[lo[i]:hi[i]]).reshape(-1, Hkv, dh)
        want = ref.attention(_np(q[i:i + 1]).reshape(1, H, dh), part(k), part(v), [0], [hi[i] - lo[i]], dtype="bf16")
        assert ref.outside(_np(o[i:i + 1]).reshape(1, H, dh), *want["o"]) <= 1.0
        assert ref.outside(_np(lse[:, i:i + 1]), *want["lse"]) <= 1.0


def _graph_of(call):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    return g


class Layer:
    """An attention layer over packed documents, forward and backward: layer norm, a fused projection, rotary positions on the
    queries and keys where they lie, attention, the output projection."""

    def __init__(self, lens, d=256, H=4, Hkv=2, dh=64, seed=0, cap=0.0):
        rng = np.random.default_rng(seed)
        self.lens, self.d, self.H, self.Hkv, self.dh, self.T = lens, d, H, Hkv, dh, sum(lens)
        T, self.wide = self.T, (H + 2 * Hkv) * dh
        bf = lambda *s, sc=1.0: _rand(rng, s, "bf16", sc).cuda()
        self.x, self.gain, self.bias, self.dout = bf(T, d), bf(d, sc=0.1) + 1, bf(d, sc=0.1), bf(T, d)
        self.w, self.wo = bf(self.wide, d, sc=d ** -0.5), bf(d, H * dh, sc=(H * dh) ** -0.5)
        new = lambda *s, t=torch.bfloat16: torch.empty(s, dtype=t, device="cuda")
        self.n, self.qkv, self.o, self.out = new(T, d), new(T, self.wide), new(T, H * dh), new(T, d)
        self.dn, self.dqkv, self.do, self.dx = new(T, d), new(T, self.wide), new(T, H * dh), new(T, d)
        self.dw, self.dwo, self.dgain, self.dbias = new(self.wide, d), new(d, H * dh), new(d), new(d)
        self.mean, self.rstd, self.lse = new(T, t=torch.float32), new(T, t=torch.float32), new(H, T, t=torch.float32)
        i32 = torch.int32
        self.lo, self.hi, self.at, self.used = new(T, t=i32), new(T, t=i32), new(T, t=i32), new(2, t=i32)
        self.cu = _ints(np.cumsum([0] + lens))
        self.pos = _ints(np.concatenate([np.arange(n) for n in lens]))
        self.rotary = R.Rotary(dims=dh, theta=10000.0)
        self.desc = R.AttnDesc(dtype=1, H=H, Hkv=Hkv, dh=dh, Tq=T, Tk=T, ldq=self.wide, ldk=self.wide, ldv=self.wide, ldo=H * dh, softcap=cap)
        self.mask = R.AttnMask(self.lo, self.hi, self.at, self.used)
        n = max(R.revffn_op_attention_masked_workspace(self.desc, True), R.revffn_op_layernorm_workspace(T, d))
        self.work = new(n, t=torch.uint8)

    def parts(self, t):
        a, b = self.H * self.dh, (self.H + self.Hkv) * self.dh
        return t[:, :a], t[:, a:b], t[:, b:]

    def run(self):
        T, d, w, H, Hkv, dh = self.T, self.d, self.wide, self.H, self.Hkv, self.dh
        R.revffn_op_attention_ranges(self.cu, None, None, len(self.lens), True, 0, T, T, self.lo, self.hi, self.at, self.used)
        R.revffn_op_layernorm_fwd(1, self.x, self.gain, self.bias, self.n, self.mean, self.rstd, T, d, d, d, 1e-5)
        R.revffn_op_gemm(1, 0, self.n, self.w, self.qkv, T, w, d, d, d, w, 0, 0)
        R.revffn_op_rotary(1, self.rotary, self.qkv, self.qkv, self.pos, T, T, H + Hkv, dh, w, w)
        R.revffn_op_attention_masked_fwd(self.desc, self.mask, *self.parts(self.qkv), self.o, self.lse, self.work)
        R.revffn_op_gemm(1, 0, self.o, self.wo, self.out, T, d, H * dh, H * dh, H * dh, d, 0, 0)
        R.revffn_op_gemm(1, 0, self.dout, self.o, self.dwo, d, H * dh, T, d, H * dh, H * dh, 1, 1)
        R.revffn_op_gemm(1, 0, self.dout, self.wo, self.do, T, H * dh, d, d, H * dh, H * dh, 0, 1)
        R.revffn_op_attention_masked_bwd(self.desc, self.mask, *self.parts(self.qkv), self.o, self.do, self.lse, *self.parts(self.dqkv), self.work)
        R.revffn_op_rotary(1, self.rotary, self.dqkv, self.dqkv, self.pos, T, T, H + Hkv, dh, w, w, True)
        R.revffn_op_gemm(1, 0, self.dqkv, self.n, self.dw, w, d, T, w, d, d, 1, 1)
        R.revffn_op_gemm(1, 0, self.dqkv, self.w, self.dn, T, d, w, w, d, d, 0, 1)
        R.revffn_op_layernorm_bwd(1, self.dn, self.x, self.gain, self.mean, self.rstd, self.dx, self.dgain, self.dbias, T, d, d, d, d, False, self.work)

    def results(self):
        return {n: getattr(self, n).clone() for n in ("out", "dx", "dw", "dwo", "dgain", "dbias")}

    def reference(self):
        x, g, b, w, wo, dout = (_np(t) for t in (self.x, self.gain, self.bias, self.w, self.wo, self.dout))
        T, H, Hkv, dh = self.T, self.H, self.Hkv, self.dh
        n = ref.layernorm(x, g, b, 1e-5)[0]
        qkv = (n @ w.T).reshape(T, H + 2 * Hkv, dh)
        pos, f = self.pos.cpu().numpy(), R.revffn_op_rotary_frequencies(self.rotary)
        qk = ref.rotary(qkv[:, : H + Hkv], pos, f, False)
        lo, hi, at = ref.ranges(self.lens)
        fwd = ref.attention(qk[:, :H], qk[:, H:], qkv[:, H + Hkv:], lo, hi, at)
        o = fwd["o"][0].reshape(T, H * dh)
        do = (dout @ wo).reshape(T, H, dh)
        bwd = ref.attention(qk[:, :H], qk[:, H:], qkv[:, H + Hkv:], lo, hi, at, do=do)
        dqk = ref.rotary(np.concatenate([bwd["dq"][0], bwd["dk"][0]], 1), pos, f, False, transposed=True)
        dqkv = np.concatenate([dqk, bwd["dv"][0]], 1).reshape(T, -1)
        _, _, _, dx, dg, db = ref.layernorm(x, g, b, 1e-5, dqkv @ w)
        return dict(out=o @ wo.T, dx=dx, dw=dqkv.T @ n, dwo=dout.T @ o, dgain=dg, dbias=db)


@pytest.mark.parametrize("lens", [[70, 1, 200, 33], [5], [1, 1, 1]])
def test_layer_run_together(lens):
    layer = Layer(lens)
    layer.run()
    torch.cuda.synchronize()
    got, want = layer.results(), layer.reference()
    # a result passes through at most eight tensors rounded to bf16 (half a step: 2^-8 of each value) and two roundings of matrix
    # operands; errors of a row's many terms don't line up, so the norm of a result's error stays under that many half steps of its own
    for name, w in want.items():
        err = np.linalg.norm(_np(got[name]) - w) / np.linalg.norm(w)
        assert err < 10 * 2.0 ** -8, (name, err)


def test_layer_captured_and_replayed():
    """One captured graph, replayed with new inputs and eager work between; then a second graph on the same workspace."""
    layer = Layer([130, 60, 1, 200], seed=1)
    layer.run()
    torch.cuda.synchronize()
    g = _graph_of(layer.run)
    other = Layer([300, 91], seed=2)
    other.work = layer.work if layer.work.numel() >= other.work.numel() else other.work
    g2 = _graph_of(other.run)
    for seed in range(3):
        fresh = Layer([130, 60, 1, 200], seed=10 + seed)
        layer.x.copy_(fresh.x)
        layer.dout.copy_(fresh.dout)
        layer.run()
        torch.cuda.synchronize()
        want = layer.results()
        for name in want:
            getattr(layer, name).fill_(NAN)
        layer.work.fill_(255)
        g.replay()
        g2.replay()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, getattr(layer, n)) for n, a in want.items())


def test_calls_on_two_streams_at_once():
    """Two layers on streams of their own, each with its own workspace, give what each gives alone."""
    layers = [Layer([300, 200], seed=3, H=8, Hkv=2), Layer([257, 3, 100], seed=4)]
    want = []
    for layer in layers:
        layer.run()
        torch.cuda.synchronize()
        want.append(layer.results())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for layer, s in zip(layers, streams):
            with torch.cuda.stream(s):
                layer.run()
    torch.cuda.synchronize()
    for layer, w in zip(layers, want):
        assert all(torch.equal(a, getattr(layer, n)) for n, a in w.items())


def test_tensors_of_another_type_are_refused():
    b, f = torch.zeros(64, dtype=torch.bfloat16, device="cuda"), torch.zeros(64, device="cuda")
    with pytest.raises(R.RevffnError, match="bfloat16"):
        R.revffn_op_layernorm_fwd(1, f, None, None, b, None, None, 1, 64, 64, 64, 1e-5)
    with pytest.raises(R.RevffnError, match="float32"):
        R.revffn_op_layernorm_fwd(1, b, None, None, b, b, None, 1, 64, 64, 64, 1e-5)
    with pytest.raises(R.RevffnError, match="int32"):
        R.revffn_op_rotary(1, R.Rotary(dims=64, theta=1e4), b, b, torch.zeros(1, dtype=torch.int64, device="cuda"), 1, 1, 1, 64, 64, 64)
    with pytest.raises(R.RevffnError, match="device"):
        R.revffn_op_rotary(1, R.Rotary(dims=64, theta=1e4), b, b.cpu(), None, 1, 1, 1, 64, 64, 64)


def test_arrays_with_strides_or_too_few_elements_are_refused():
    """Ranges as columns of one table, for instance, would be read as something else; every array that has no stride argument."""
    T, H, dh = 6, 2, 64
    bf, f32 = (lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")), (lambda *s: torch.zeros(s, device="cuda"))
    ints = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    q, lse, work = bf(T, H * dh), f32(H, T), torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    r = R.Rotary(dims=64, theta=1e4)

    def ranges(cu=ints(3), pre=ints(2), lo=ints(T), hi=ints(T), at=ints(T), used=ints(2)):
        R.revffn_op_attention_ranges(cu, cu, pre, 2, True, 0, T, T, lo, hi, at, used)

    def attention(lo=ints(T), hi=ints(T), at=ints(T), used=ints(2), slopes=f32(H), lse=lse, work=work):
        d, m = R.AttnDesc(dtype=1, H=H, Hkv=H, dh=dh, Tq=T, Tk=T, slopes=slopes), R.AttnMask(lo, hi, at, used)
        R.revffn_op_attention_masked_fwd(d, m, q, q, q, bf(T, H * dh), lse, work)
        R.revffn_op_attention_masked_bwd(d, m, q, q, q, q, q, lse, bf(T, H * dh), bf(T, H * dh), bf(T, H * dh), work)

    def rotary(pos=ints(T)):
        R.revffn_op_rotary(1, r, q, bf(T, H * dh), pos, T, T, H, dh, H * dh, H * dh)

    def norm(gain=bf(H * dh), bias=bf(H * dh), mean=f32(T), rstd=f32(T), dgain=bf(H * dh), dbias=bf(H * dh), work=work):
        R.revffn_op_layernorm_fwd(1, q, gain, bias, bf(T, H * dh), mean, rstd, T, H * dh, H * dh, H * dh, 1e-5)
        R.revffn_op_layernorm_bwd(1, q, q, gain, mean, rstd, bf(T, H * dh), dgain, dbias, T, H * dh, H * dh, H * dh, H * dh, False, work)
    for call in (ranges, attention, rotary, norm):
        call()
        torch.cuda.synchronize()
        for name, t in zip(call.__code__.co_varnames, call.__defaults__):
            wide = torch.zeros(*t.shape, 2, dtype=t.dtype, device="cuda")[..., 0]
            with pytest.raises(R.RevffnError, match="strides"):
                call(**{name: wide})
            with pytest.raises(R.RevffnError):
                call(**{name: t.flatten()[:1]})
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
# T, H, dh, dims, extra columns in a row, scaling
@pytest.mark.parametrize("T,H,dh,dims,extra,scaling", [(1, 1, 2, 2, 0, 0), (5, 3, 64, 64, 0, 1), (70, 20, 128, 64, 32, 2), (33, 4, 128, 128, 64, 3),
                                                        (9, 3, 80, 20, 1, 3), (4, 2, 33, 30, 0, 0), (3, 2, 1000, 6, 3, 0), (2000, 2, 256, 256, 0, 2),
                                                        (17, 5, 24, 24, 0, 0), (3000, 7, 20, 12, 0, 1)])
def test_rotary(T, H, dh, dims, extra, scaling, interleaved, dtype):
    if scaling == 2 and dims == 2:
        scaling = 0
    rng = np.random.default_rng(T + dh + dims)
    r = R.Rotary(dims=dims, interleaved=interleaved, scaling=scaling, original=512, theta=10000.0, factor=4.0, few_turns=1.0, many_turns=32.0,
                 magnitude=1.25 if scaling == 3 else 0.0)
    freq = R.revffn_op_rotary_frequencies(r)
    i = np.arange(dims // 2)
    want = 10000.0 ** (-2.0 * i / dims)
    if scaling == 1:
        want = want / 4
    if scaling == 2:
        want = (10000.0 * 4.0 ** (dims / (dims - 2))) ** (-2.0 * i / dims)
    if scaling == 3:
        g = np.clip((512 * want / (2 * np.pi) - 1) / 31, 0, 1)
        want = g * want + (1 - g) * want / 4
    assert np.allclose(freq, want, rtol=1e-12, atol=0)
    mag = 1.25 if scaling == 3 else 1.0
    rows = _rand(rng, (T, H * dh + extra), dtype).cuda()
    x = _np(rows[:, : H * dh]).reshape(T, H, dh)
    pos = rng.integers(0, 1_000_000, T)
    pos[0] = -5
    u, w = HALF_STEP[dtype], 2.0 ** -24
    for transposed in (False, True):
        for p, dev in ((pos, _ints(pos)), (np.arange(T) % 7, None)):
            y = torch.full((T, H * dh + 2 * extra), NAN, dtype=TORCH[dtype], device="cuda")
            R.revffn_op_rotary(1 if dtype == "bf16" else 0, r, rows, y, dev, T, 7, H, dh, H * dh + extra, H * dh + 2 * extra, transposed)
            again = rows.clone()
            R.revffn_op_rotary(1 if dtype == "bf16" else 0, r, again, again, dev, T, 7, H, dh, H * dh + extra, H * dh + extra, transposed)
            torch.cuda.synchronize()
            ref_y = ref.rotary(x, p, freq, interleaved, mag, transposed)
            # a sine or cosine is off by 2 ulp of 1, products and their sum by half a step each; both columns are at most the pair's length
            pair = mag * np.abs(x).max(initial=0.0) * 1.5
            got = _np(y[:, : H * dh]).reshape(T, H, dh)
            assert ref.outside(got, ref_y, 8 * w * pair + u * np.abs(ref_y)) <= 1.0
            assert (got[..., dims:] == x[..., dims:]).all() and torch.isnan(y[:, H * dh:]).all()
            assert torch.equal(again[:, : H * dh], y[:, : H * dh]) and torch.equal(again[:, H * dh:], rows[:, H * dh:])


HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 7, 0), (5, 64, 0), (130, 500, 0), (9, 513, 0), (70, 1024, 8), (40, 1025, 3), (33, 2048, 0), (2100, 256, 0),
                                           (21, 2056, 0), (6, 4100, 4), (7, 8192, 0), (5, 8200, 1), (3, 32768, 0), (9, 32776, 0), (3, 40001, 0)])
@pytest.mark.parametrize("params", ["both", "none", "gain_f32"])
def test_layernorm(rows, cols, pad, params, dtype):
    rng = np.random.default_rng(rows + cols)
    wide = lambda sc, shift=0.0: (_rand(rng, (rows, cols + pad), dtype, sc).cuda() + shift).to(TORCH[dtype])
    x, dy = wide(1.5, 0.7), wide(1.0)
    gain = None if params == "none" else (1 + 0.2 * _rand(rng, cols, "f32")).to(TORCH[dtype]).cuda()
    bias = _rand(rng, cols, dtype).cuda() if params == "both" else None
    new = lambda: torch.full((rows, cols + pad), NAN, dtype=TORCH[dtype], device="cuda")
    y, dx, mean, rstd = new(), new(), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    gt = torch.float32 if params == "gain_f32" else TORCH[dtype]
    dgain = torch.full((cols,), NAN, dtype=gt, device="cuda") if params != "none" else None
    dbias = torch.full((cols,), NAN, dtype=gt, device="cuda") if params == "both" else None
    work = torch.full((R.revffn_op_layernorm_workspace(rows, cols),), 255, dtype=torch.uint8, device="cuda")
    dt, ld = (1 if dtype == "bf16" else 0), cols + pad
    R.revffn_op_layernorm_fwd(dt, x, gain, bias, y, mean, rstd, rows, cols, ld, ld, 1e-5)
    R.revffn_op_layernorm_bwd(dt, dy, x, gain, mean, rstd, dx, dgain, dbias, rows, cols, ld, ld, ld, params == "gain_f32", work)
    torch.cuda.synchronize()
    xn, dyn = _np(x[:, :cols]), _np(dy[:, :cols])
    g, b = (None if t is None else _np(t) for t in (gain, bias))
    ry, rm, rr, rdx, rdg, rdb = ref.layernorm(xn, g, b, 1e-5, dyn)
    u, e = HALF_STEP[dtype], 2.0 ** -24
    gm = 1.0 if g is None else np.abs(g)
    # a float32 sum of n terms in any order is off by n e of the sum of their sizes; it is taken over at most 64 terms per thread and a tree behind
    n = min(cols, 64) + 16
    e_mean = n * e * np.abs(xn).mean(1)
    e_r = (n + 8) * e + e_mean * rr                                       # relative, of rstd (at mean +- e_mean the variance is e_mean^2 larger)
    xh = np.abs((xn - rm[:, None]) * rr[:, None])
    e_xh = (e_mean * rr)[:, None] + (e_r[:, None] + 2 * e) * xh
    assert ref.outside(_np(mean), rm, e_mean + e * np.abs(rm)) <= 1.0
    assert ref.outside(_np(rstd), rr, e_r * rr) <= 1.0
    assert ref.outside(_np(y[:, :cols]), ry, e_xh * gm + 2 * e * (xh * gm + (0 if b is None else np.abs(b))) + u * np.abs(ry)) <= 1.0
    d = np.abs(dyn) * gm
    m1, m2 = d.mean(1, keepdims=True), (d * xh).mean(1, keepdims=True)
    e_dx = rr[:, None] * (4 * e * d + n * e * m1 + xh * ((n + 4) * e * m2 + (d * e_xh).mean(1, keepdims=True)) + e_xh * m2) + (e_r[:, None] + 4 * e) * (
        rr[:, None] * (d + m1 + xh * m2))
    assert ref.outside(_np(dx[:, :cols]), rdx, e_dx + u * np.abs(rdx)) <= 1.0
    ug = 2.0 ** -24 if params == "gain_f32" else u
    if dgain is not None:
        assert ref.outside(_np(dgain), rdg, ((rows + 16) * e * np.abs(dyn) * xh + np.abs(dyn) * e_xh).sum(0) + ug * np.abs(rdg)) <= 1.0
    if dbias is not None:
        assert ref.outside(_np(dbias), rdb, (rows + 16) * e * np.abs(dyn).sum(0) + ug * np.abs(rdb)) <= 1.0
    if pad:
        assert torch.isnan(y[:, cols:]).all() and torch.isnan(dx[:, cols:]).all()
    # in place, with the sums: the same bits
    dy3, g3, b3 = dy.clone(), None if dgain is None else torch.empty_like(dgain), None if dbias is None else torch.empty_like(dbias)
    work.fill_(255)
    R.revffn_op_layernorm_bwd(dt, dy3, x, gain, mean, rstd, dy3, g3, b3, rows, cols, ld, ld, ld, params == "gain_f32", work)
    torch.cuda.synchronize()
    assert torch.equal(dy3[:, :cols], dx[:, :cols]) and (g3 is None or torch.equal(g3, dgain)) and (b3 is None or torch.equal(b3, dbias))
    # without them
    x2, dy2 = x.clone(), dy.clone()
    R.revffn_op_layernorm_bwd(dt, dy2, x2, gain, mean, rstd, dy2, None, None, rows, cols, ld, ld, ld)
    R.revffn_op_layernorm_fwd(dt, x2, gain, bias, x2, None, None, rows, cols, ld, ld, 1e-5)
    torch.cuda.synchronize()
    assert torch.equal(x2[:, :cols], y[:, :cols]) and torch.equal(dy2[:, :cols], dx[:, :cols])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
# rows, columns, extra columns in a row: three rows and more for a workgroup (wave), not as many for each; a line of columns per form of the kernel
@pytest.mark.parametrize("rows,cols,pad", [(9001, 256, 0), (12301, 509, 0), (4500, 1000, 0), (6601, 777, 1), (2600, 2048, 0), (3333, 1500, 4), (2600, 2047, 0),
                                           (1100, 4096, 0), (1600, 2300, 0), (1100, 4001, 0), (1100, 4104, 0), (1030, 8190, 2), (530, 8200, 0), (800, 16001, 0),
                                           (70, 16392, 0), (131, 20001, 3)])
def test_layernorm_backward_of_many_rows(rows, cols, pad, dtype):
    """x and dy whole numbers, mean 0 and rstd 1: the sums over the rows are whole numbers below 2^24, which float32 adds without error in any order, so a
    row that is left out, taken twice or mixed up with the next one shows.  In place as well."""
    rng = np.random.default_rng(rows + cols)
    whole = lambda top: torch.from_numpy(rng.integers(-top, top + 1, (rows, cols + pad)).astype(np.float32)).to(TORCH[dtype]).cuda()
    x, dy = whole(8), whole(6)
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    xn, d = _np(x[:, :cols]), _np(dy[:, :cols])
    s, q = d.mean(1, keepdims=True), (d * xn).mean(1, keepdims=True)
    want = d - s - xn * q
    # s and q are exact sums divided once: half a step of each, of x q and of the two differences
    e = 2.0 ** -24
    bound = 4 * e * (np.abs(d) + np.abs(s) + np.abs(xn * q)) + HALF_STEP[dtype] * np.abs(want)
    dt, ld = (1 if dtype == "bf16" else 0), cols + pad
    results = []
    for in_place in (False, True):
        dx = dy.clone() if in_place else torch.full_like(dy, NAN)
        dgain, dbias = (torch.full((cols,), NAN, device="cuda") for _ in range(2))
        work = torch.full((R.revffn_op_layernorm_workspace(rows, cols),), 255, dtype=torch.uint8, device="cuda")
        R.revffn_op_layernorm_bwd(dt, dx if in_place else dy, x, None, mean, rstd, dx, dgain, dbias, rows, cols, ld, ld, ld, True, work)
        torch.cuda.synchronize()
        assert (_np(dgain) == (d * xn).sum(0)).all() and (_np(dbias) == d.sum(0)).all()
        assert ref.outside(_np(dx[:, :cols]), want, bound) <= 1.0
        results.append(dx[:, :cols].clone())
    dx = torch.full_like(dy, NAN)
    R.revffn_op_layernorm_bwd(dt, dy, x, None, mean, rstd, dx, None, None, rows, cols, ld, ld, ld)
    torch.cuda.synchronize()
    assert all(torch.equal(dx[:, :cols], r) for r in results) and (pad == 0 or torch.isnan(dx[:, cols:]).all())


def test_layernorm_without_rows():
    t, f = torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
    g, b = torch.full((8,), NAN, device="cuda"), torch.full((8,), NAN, device="cuda")
    work = torch.empty(R.revffn_op_layernorm_workspace(0, 8), dtype=torch.uint8, device="cuda")
    R.revffn_op_layernorm_fwd(0, t, None, None, f, None, None, 0, 8, 8, 8, 1e-5)
    R.revffn_op_layernorm_bwd(0, t, t, None, f, f, f, g, b, 0, 8, 8, 8, 8, False, work)
    torch.cuda.synchronize()
    assert (g == 0).all() and (b == 0).all()
