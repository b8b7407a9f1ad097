"""Host-only checks of the operators for attention layers: what they refuse, before anything reaches a GPU; the layouts of
their structs; and the float64 references against differences."""
import ctypes
import os
import re

import numpy as np
import pytest

import operators_reference as ref
import paper_2512_20920_amd as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ESHAPE, ENULL, EUNSUPPORTED = -1, -2, -3, -6
P = 4096                    # an address that is never read: every call here is refused


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(R.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return R.load_library()


def desc(**kw):
    return R.AttnDesc(**(dict(dtype=1, H=4, Hkv=2, dh=64, Tq=10, Tk=20) | kw))


def test_struct_layouts_match_header():
    header = open(os.path.join(ROOT, "include", "revffn.h")).read()
    for name, cls, size in (("revffn_attn_desc", R.AttnDesc, 80), ("revffn_attn_mask", R.AttnMask, 32), ("revffn_rotary", R.Rotary, 36)):
        body = re.sub(r"/\*.*?\*/", "", header[header.index(f"typedef struct {name} {{"):header.index(f"}} {name};")], flags=re.S)
        fields = []
        for line in re.findall(r"(?:const\s+)?(?:int32_t|int64_t|float)\s+([^;]+);", body):
            fields += [f.strip(" *") for f in line.split(",")]
        assert fields == [n for n, _ in cls._fields_], name
        assert ctypes.sizeof(cls) == size


BAD_DESCS = [(dict(dtype=2), EINVAL), (dict(dtype=-1), EINVAL), (dict(kernel_mode=3), EINVAL), (dict(kernel_mode=-1), EINVAL), (dict(kernel_mode=768), EINVAL),
             (dict(H=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(H=3), EINVAL), (dict(H=2, Hkv=4), EINVAL), (dict(H=65538), EINVAL), (dict(dh=0), EINVAL),
             (dict(dh=513), EINVAL), (dict(Tq=-1), EINVAL), (dict(Tk=-1), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL),
             (dict(softcap=-1.0), EINVAL), (dict(softcap=float("nan")), EINVAL), (dict(softcap=float("inf")), EINVAL),
             (dict(ldq=255), ESHAPE), (dict(ldk=127), ESHAPE), (dict(ldv=1), ESHAPE), (dict(ldo=-256), ESHAPE), (dict(Tq=2 ** 31 - 1), ESHAPE),
             (dict(Tk=2 ** 26), ESHAPE)]


@pytest.mark.parametrize("kw,code", BAD_DESCS)
def test_attention_refuses_bad_descs(lib, kw, code):
    d, m = desc(**kw), R.AttnMask(P, P)
    assert lib.revffn_op_attention_masked_workspace(ctypes.byref(d), 0) == 0
    assert lib.revffn_op_attention_masked_fwd(ctypes.byref(d), ctypes.byref(m), P, P, P, P, P, P, 1 << 40, None) == code
    assert lib.revffn_op_attention_masked_bwd(ctypes.byref(d), ctypes.byref(m), P, P, P, P, P, P, P, P, P, P, 1 << 40, None) == code
    with pytest.raises(R.RevffnError, match=str(code)):
        R.revffn_op_attention_masked_fwd(d, m, P, P, P, P, P, None, stream=0)


def test_attention_refuses_missing_and_small(lib):
    d, m = desc(), R.AttnMask(P, P)
    need = lib.revffn_op_attention_masked_workspace(ctypes.byref(d), 1)
    assert need >= 4 * 10 * 4 and lib.revffn_op_attention_masked_workspace(ctypes.byref(d), 0) <= need
    fwd = lambda d_, m_, *a: lib.revffn_op_attention_masked_fwd(d_, m_, *a, None)
    bd, bm = ctypes.byref(d), ctypes.byref(m)
    assert fwd(None, bm, P, P, P, P, P, P, need) == ENULL and fwd(bd, None, P, P, P, P, P, P, need) == ENULL
    assert fwd(bd, ctypes.byref(R.AttnMask(None, P)), P, P, P, P, P, P, need) == ENULL
    assert fwd(bd, ctypes.byref(R.AttnMask(P, None)), P, P, P, P, P, P, need) == ENULL
    for missing in (0, 1, 2, 3):
        a = [P] * 5
        a[missing] = None
        assert fwd(bd, bm, *a, P, need) == ENULL
    good = [P] * 10
    for missing in range(9):
        a = list(good)
        a[missing] = None
        assert lib.revffn_op_attention_masked_bwd(bd, bm, *a[:9], P, need, None) == ENULL, missing
    assert lib.revffn_op_attention_masked_bwd(bd, bm, *good[:9], None, 0, None) == ENULL
    assert lib.revffn_op_attention_masked_bwd(bd, bm, *good[:9], P, need - 1, None) == EINVAL
    assert lib.revffn_op_attention_masked_bwd(bd, bm, *good[:9], P + 8, need, None) == EINVAL
    # a long run of keys is split, which takes scratch memory
    d = desc(Tq=1, Tk=5000)
    need = lib.revffn_op_attention_masked_workspace(ctypes.byref(d), 0)
    assert need > 0
    assert fwd(ctypes.byref(d), bm, P, P, P, P, P, None, 0) == ENULL and fwd(ctypes.byref(d), bm, P, P, P, P, P, P, need - 1) == EINVAL
    # matrix-core kernels only, and a shape that they don't take
    for kw in (dict(dh=33), dict(dh=136), dict(dtype=0, dh=34), dict(dtype=0, dh=132), dict(ldq=257), dict(ldk=1 << 24)):
        d = desc(kernel_mode=2, **kw)
        n = lib.revffn_op_attention_masked_workspace(ctypes.byref(d), 1)
        assert fwd(ctypes.byref(d), bm, P, P, P, P, P, P, n) == EUNSUPPORTED, kw
        assert lib.revffn_op_attention_masked_bwd(ctypes.byref(d), bm, *good[:9], P, n, None) == EUNSUPPORTED, kw
    assert fwd(ctypes.byref(desc(kernel_mode=2)), bm, P + 2, P, P, P, P, P, 1 << 30) == EUNSUPPORTED


def test_attention_refuses_results_in_the_place_of_inputs(lib):
    """A gradient written over d_o, for instance, which the second half of the backward pass reads again."""
    bd, bm, n = ctypes.byref(desc()), ctypes.byref(R.AttnMask(P, P)), 1 << 30
    apart = [P * (i + 1) for i in range(9)]                 # q, k, v, o, (d_o, lse, dq, dk, dv or lse)
    for into in (3, 4):
        for other in range(into):
            a = apart[:5]
            a[into] = a[other]
            assert lib.revffn_op_attention_masked_fwd(bd, bm, *a, P, n, None) == EINVAL, (into, other)
    for into in (6, 7, 8):
        for other in range(into):
            a = apart[:9]
            a[into] = a[other]
            assert lib.revffn_op_attention_masked_bwd(bd, bm, *a, P, n, None) == EINVAL, (into, other)


def test_attention_scratch_memory_is_each_descs_own(lib):
    """A call of fewer rows may need more of it, and a workspace that is too small for it is refused, whatever larger call it was made for."""
    size = lambda backward, **kw: lib.revffn_op_attention_masked_workspace(ctypes.byref(desc(**kw)), backward)
    shape = dict(H=16, Hkv=4, dh=128, Tk=32768)
    big, small = size(0, Tq=4096, **shape), size(0, Tq=64, **shape)
    assert big < small
    f32 = dict(dtype=0, H=4, Hkv=2, dh=64)
    big_b, small_b = size(1, Tq=8192, Tk=8192, **f32), size(1, Tq=2048, Tk=2048, **f32)
    assert big_b < small_b
    bm = ctypes.byref(R.AttnMask(P, P))
    assert lib.revffn_op_attention_masked_fwd(ctypes.byref(desc(Tq=64, **shape)), bm, P, P, P, P, P, P, big, None) == EINVAL
    assert lib.revffn_op_attention_masked_bwd(ctypes.byref(desc(Tq=2048, Tk=2048, **f32)), bm, *[P] * 10, big_b, None) == EINVAL
    assert lib.revffn_op_layernorm_workspace(300, 20000) < lib.revffn_op_layernorm_workspace(300, 16384)


def test_attention_ranges_refuses(lib):
    f = lambda *a: lib.revffn_op_attention_ranges(*a, None)
    assert f(P, P, None, 2, 1, 0, 10, 10, None, P, None, None) == ENULL and f(P, P, None, 2, 1, 0, 10, 10, P, None, None, None) == ENULL
    for a in ((P, P, None, 0, 1, 0, 10, 10), (P, P, None, -1, 1, 0, 10, 10), (P, P, None, 2 ** 31 - 1, 1, 0, 10, 10), (P, P, None, 2, 2, 0, 10, 10),
              (P, P, None, 2, 1, -1, 10, 10), (P, P, None, 2, 1, 0, -1, 10), (P, P, None, 2, 1, 0, 10, -1), (P, P, P, 2, 1, 5, 10, 10),
              (P, P, P, 2, 0, 0, 10, 10), (P, P, None, 2, 0, 5, 10, 10)):
        assert f(*a, P, P, None, None) == EINVAL, a
    assert f(None, P, None, 3, 1, 0, 10, 10, P, P, None, None) == ESHAPE and f(None, None, None, 5, 1, 0, 10, 11, P, P, None, None) == ESHAPE


BAD_ROTARY = [dict(dims=0), dict(dims=7), dict(dims=258), dict(dims=66), dict(interleaved=2), dict(scaling=4), dict(scaling=-1), dict(theta=0.0), dict(theta=float("nan")),
              dict(theta=float("inf")), dict(magnitude=float("nan")), dict(scaling=1, factor=0.0), dict(scaling=1, factor=float("inf")), dict(scaling=2, dims=2),
              dict(scaling=3, original=0), dict(scaling=3, few_turns=-1.0), dict(scaling=3, many_turns=1.0), dict(scaling=3, many_turns=float("inf"))]


@pytest.mark.parametrize("kw", BAD_ROTARY)
def test_rotary_refuses_bad_descs(lib, kw):
    r = R.Rotary(**(dict(dims=64, theta=1e4, factor=2.0, original=512, few_turns=1.0, many_turns=32.0) | kw))
    assert lib.revffn_op_rotary(1, ctypes.byref(r), P, P, P, 5, 5, 4, 64, 256, 256, 0, None) == EINVAL
    if kw != dict(dims=66):            # (only wider than the head)
        with pytest.raises(R.RevffnError):
            R.revffn_op_rotary_frequencies(r)


def test_rotary_refuses(lib):
    r = R.Rotary(dims=64, theta=1e4)
    call = lambda dtype=1, x=P, y=P, pos=P, T=5, S=5, H=4, dh=64, ldx=256, ldy=256, back=0: lib.revffn_op_rotary(
        dtype, ctypes.byref(r), x, y, pos, T, S, H, dh, ldx, ldy, back, None)
    assert call(x=None) == ENULL and call(y=None) == ENULL and lib.revffn_op_rotary(1, None, P, P, P, 5, 5, 4, 64, 256, 256, 0, None) == ENULL
    assert lib.revffn_op_rotary_frequencies(None, P) == ENULL and lib.revffn_op_rotary_frequencies(ctypes.byref(r), None) == ENULL
    for kw in (dict(dtype=2), dict(T=-1), dict(pos=None, S=0), dict(H=0), dict(dh=1), dict(dh=1025, ldx=9999, ldy=9999), dict(back=2), dict(dh=32)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(ldx=255), dict(ldy=255), dict(T=2 ** 24), dict(ldx=512), dict(H=65536, dh=128, ldx=2 ** 23, ldy=2 ** 23)):
        assert call(**kw) == ESHAPE, kw
    assert call(T=0) == 0


def test_layernorm_refuses(lib):
    fwd = lambda dtype=1, x=P, y=P + 4096, rows=5, cols=8, ldx=8, ldy=8, eps=1e-5: lib.revffn_op_layernorm_fwd(
        dtype, x, None, None, y, None, None, rows, cols, ldx, ldy, eps, None)
    assert fwd(x=None) == ENULL and fwd(y=None) == ENULL
    for kw in (dict(dtype=2), dict(rows=-1), dict(cols=0), dict(cols=2 ** 24 + 1, ldx=2 ** 25, ldy=2 ** 25), dict(eps=-1.0), dict(eps=float("nan")),
               dict(eps=float("inf"))):
        assert fwd(**kw) == EINVAL, kw
    for kw in (dict(ldx=7), dict(ldy=7), dict(x=P, y=P, ldx=9), dict(rows=2 ** 22)):
        assert fwd(**kw) == ESHAPE, kw
    assert fwd(rows=0) == 0
    need = lib.revffn_op_layernorm_workspace(5, 8)
    assert need >= 2 * 8 * 4 and lib.revffn_op_layernorm_workspace(-1, 8) == 0 and lib.revffn_op_layernorm_workspace(5, 0) == 0

    def bwd(dtype=1, dy=P, x=P + 4096, mean=P, rstd=P, dx=P + 8192, dgain=P, dbias=P, rows=5, cols=8, lddy=8, ldx=8, lddx=8, f32=0, work=P, n=need):
        return lib.revffn_op_layernorm_bwd(dtype, dy, x, P, mean, rstd, dx, dgain, dbias, rows, cols, lddy, ldx, lddx, f32, work, n, None)
    for name in ("dy", "x", "mean", "rstd", "dx", "work"):
        assert bwd(**{name: None}) == ENULL, name
    for kw in (dict(dtype=2), dict(rows=-1), dict(cols=0), dict(f32=2), dict(dx=P + 4096), dict(n=need - 1), dict(work=P + 4)):
        assert bwd(**kw) == EINVAL, kw
    for kw in (dict(lddy=7), dict(ldx=7), dict(lddx=7), dict(dx=P, lddx=9), dict(rows=2 ** 22)):
        assert bwd(**kw) == ESHAPE, kw


def test_tensors_that_no_gpu_may_read_are_refused():
    torch = pytest.importorskip("torch")
    t, f = torch.zeros(64, dtype=torch.bfloat16), torch.zeros(64)
    with pytest.raises(R.RevffnError, match="device"):
        R.revffn_op_layernorm_fwd(1, t, None, None, t, None, None, 1, 64, 64, 64, 1e-5, stream=0)
    with pytest.raises(R.RevffnError, match="device"):
        R.revffn_op_rotary(1, R.Rotary(dims=64, theta=1e4), t, t, None, 1, 1, 1, 64, 64, 64, stream=0)
    with pytest.raises(R.RevffnError, match="device"):
        R.revffn_op_attention_masked_fwd(desc(), R.AttnMask(P, P), P, P, P, P, f, None, stream=0)
    with pytest.raises(R.RevffnError, match="device"):
        R.revffn_op_attention_ranges(torch.zeros(3, dtype=torch.int32), None, None, 2, True, 0, 8, 8, P, P, stream=0)
    with pytest.raises(R.RevffnError, match="float32"):
        R.binding._refuse(t, torch.float32)


def test_arrays_with_strides_or_too_few_elements_are_refused():
    torch = pytest.importorskip("torch")
    dense = R.binding._dense
    table = torch.zeros(6, 2, dtype=torch.int32)
    assert dense(-1, torch.int32, 12, table, None, 4096) == [table.data_ptr(), None, 4096]
    with pytest.raises(R.RevffnError, match="strides"):
        dense(-1, torch.int32, 6, table[:, 0])
    with pytest.raises(R.RevffnError, match="12 elements"):
        dense(-1, torch.int32, 13, table)
    with pytest.raises(R.RevffnError, match="float32"):
        dense(-1, torch.float32, 1, table)
    with pytest.raises(R.RevffnError, match="device"):
        dense(0, torch.int32, 1, table)
    with pytest.raises(R.RevffnError, match="strides"):
        R.binding._work(-1, torch.zeros(8, 8, dtype=torch.uint8)[:, :4])


@pytest.mark.parametrize("cap,bias", [(0.0, False), (2.0, False), (0.0, True), (3.0, True)])
def test_reference_gradients_are_differences(cap, bias):
    """The gradients that the kernels are compared with, against central differences of the forward reference."""
    rng = np.random.default_rng(3)
    lo, hi, at = ref.ranges([4, 0, 3], [6, 2, 3], prefix=[3, 0, 0])
    q, k, v, do = (rng.standard_normal(s) for s in ((7, 4, 6), (11, 2, 6), (11, 2, 6), (7, 4, 6)))
    slopes = np.array([0.5, 0.25, 0.1, 0.7]) if bias else None
    out = ref.attention(q, k, v, lo, hi, at, cap=cap, slopes=slopes, do=do, dtype="f32")
    value = lambda: (ref.attention(q, k, v, lo, hi, at, cap=cap, slopes=slopes, dtype="f32")["o"][0] * do).sum()
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        for _ in range(12):
            i = tuple(rng.integers(0, n) for n in x.shape)
            keep, h = x[i], 1e-5
            x[i] = keep + h
            up = value()
            x[i] = keep - h
            down = value()
            x[i] = keep
            # second-order differences: off by h^2 times a third derivative of order one, and by 2^-53 / h of the value
            assert abs((up - down) / (2 * h) - out[name][0][i]) < 1e-7 + 1e-9 * abs(up)


def test_reference_layernorm_and_rotary_gradients():
    rng = np.random.default_rng(4)
    x, g, b, dy = rng.standard_normal((3, 9)), rng.standard_normal(9), rng.standard_normal(9), rng.standard_normal((3, 9))
    grads = dict(zip(("x", "g", "b"), ref.layernorm(x, g, b, 1e-5, dy)[3:]))
    for name, t in (("x", x), ("g", g), ("b", b)):
        for i in np.ndindex(*t.shape):
            keep, h = t[i], 1e-5
            t[i] = keep + h
            up = (ref.layernorm(x, g, b, 1e-5)[0] * dy).sum()
            t[i] = keep - h
            down = (ref.layernorm(x, g, b, 1e-5)[0] * dy).sum()
            t[i] = keep
            assert abs((up - down) / (2 * h) - grads[name][i]) < 1e-7
    x, dy = rng.standard_normal((4, 2, 10)), rng.standard_normal((4, 2, 10))
    pos, freq = [0, 3, -7, 100000], np.array([1.0, 0.3, 0.01])
    for inter in (False, True):       # the turn is linear: <turn x, dy> = <x, transposed turn dy>
        a = (ref.rotary(x, pos, freq, inter, 1.3) * dy).sum()
        assert abs(a - (x * ref.rotary(dy, pos, freq, inter, 1.3, True)).sum()) < 1e-9
