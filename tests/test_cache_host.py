"""Host-only checks of the paged cache, its attention and the integer products: what the calls refuse, before anything reaches a GPU; the
layout of the cache's struct; and the references in 64 bits against independent ones."""
import ctypes
import os
import re
import struct
import subprocess
import tempfile

import numpy as np
import pytest
import torch

import cache_reference as ref
import operators_reference
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


def cache(**kw):
    at = dict(k=P, v=2 * P, k_scale=3 * P, v_scale=4 * P, table=P, len=P, cu=P)
    sizes = dict(pages=10, page=64, max_pages=4, n_seqs=3, Hkv=2, dh=64)
    at.update({n: kw.pop(n) for n in list(kw) if n in at})
    c = R.Cache(*at.values(), **(sizes | kw))
    return c


def desc(**kw):
    return R.AttnDesc(**(dict(dtype=1, H=4, Hkv=2, dh=64, Tq=10) | kw))


BAD_CACHES = [(dict(page=0), EINVAL), (dict(page=8), EINVAL), (dict(page=48), EINVAL), (dict(page=256), EINVAL), (dict(pages=0), EINVAL), (dict(pages=-1), EINVAL),
              (dict(max_pages=0), EINVAL), (dict(max_pages=2 ** 30 // 64 + 1), EINVAL), (dict(n_seqs=-1), EINVAL), (dict(n_seqs=2 ** 20 + 1), EINVAL),
              (dict(Hkv=0), EINVAL), (dict(Hkv=65537), EINVAL), (dict(dh=8), EINVAL), (dict(dh=72), EINVAL), (dict(dh=272), EINVAL),
              (dict(dh=256, page=128), ESHAPE), (dict(pages=2 ** 30), ESHAPE), (dict(k=None), ENULL), (dict(v=None), ENULL), (dict(k_scale=None), ENULL),
              (dict(v_scale=None), ENULL), (dict(table=None), ENULL), (dict(len=None), ENULL), (dict(k=P + 8), EINVAL), (dict(v=P), EINVAL),
              (dict(v_scale=3 * P), EINVAL)]


def append(lib, c, dtype=1, r=None, pos=P, q=5 * P, q_out=6 * P, k=7 * P, v=8 * P, T=10, H=4, ldq=256, ldqo=256, ldk=128, ldv=128):
    return lib.revffn_op_cache_append(dtype, None if c is None else ctypes.byref(c), None if r is None else ctypes.byref(r), pos, q, q_out, k, v, T, H, ldq, ldqo,
                                      ldk, ldv, None)


def attend(lib, d, c, causal=1, window=0, q=5 * P, o=6 * P, lse=7 * P, work=8 * P, size=1 << 40):
    return lib.revffn_op_attention_cached(None if d is None else ctypes.byref(d), None if c is None else ctypes.byref(c), causal, window, q, o, lse, work, size, None)


def test_struct_layout_matches_header():
    header = open(os.path.join(ROOT, "include", "revffn.h")).read()
    body = re.sub(r"/\*.*?\*/", "", header[header.index("typedef struct revffn_cache {"):header.index("} revffn_cache;")], flags=re.S)
    fields = []
    for line in re.findall(r"(?:const\s+)?(?:int32_t|void|float)\s+([^;]+);", body):
        fields += [f.strip(" *") for f in line.split(",")]
    assert fields == [n for n, _ in R.Cache._fields_] and ctypes.sizeof(R.Cache) == 80


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_bad_caches_are_refused(lib, kw, code):
    c = cache(**kw)
    d = desc(dh=c.dh, Hkv=max(c.Hkv, 1), H=4 * max(c.Hkv, 1)) if c.Hkv <= 16384 else desc()
    assert append(lib, c, ldk=1 << 30, ldv=1 << 30, ldq=1 << 30, ldqo=1 << 30) == code
    assert attend(lib, d, c) == code
    assert lib.revffn_op_attention_cached_workspace(ctypes.byref(d), ctypes.byref(c)) == 0


def test_append_refuses(lib):
    c, r = cache(), R.Rotary(dims=64, theta=1e4)
    assert append(lib, None) == ENULL
    for kw in (dict(k=None), dict(v=None), dict(q_out=None)):
        assert append(lib, c, **kw) == ENULL
    for kw in (dict(dtype=2), dict(dtype=-1), dict(T=-1), dict(H=0), dict(H=65537), dict(r=R.Rotary(dims=72, theta=1e4)), dict(r=R.Rotary(dims=128, theta=1e4)),
               dict(r=R.Rotary(dims=64, theta=0.0)), dict(r=R.Rotary(dims=8, theta=1e4)), dict(k=c.k), dict(v=c.v), dict(q_out=7 * P), dict(q_out=c.k), dict(q_out=c.v_scale)):
        assert append(lib, c, **kw) == EINVAL, kw
    for kw in (dict(ldk=127), dict(ldv=0), dict(ldq=255), dict(ldqo=-1), dict(q_out=5 * P, ldqo=512), dict(T=2 ** 31 - 1)):
        assert append(lib, c, **kw) == ESHAPE, kw
    assert append(lib, c, T=0, k=None, v=None, q=None, q_out=None, r=r) == 0          # (nothing to do)
    assert append(lib, cache(n_seqs=0, table=None, len=None, cu=None)) == 0


def test_attention_refuses(lib):
    c, d = cache(max_pages=400), desc()
    assert attend(lib, None, c) == ENULL and attend(lib, d, None) == ENULL
    for kw in (dict(q=None), dict(o=None), dict(work=None)):
        assert attend(lib, d, c, **kw) == ENULL
    need = lib.revffn_op_attention_cached_workspace(ctypes.byref(d), ctypes.byref(c))
    assert need > 0
    for kw in (dict(causal=2), dict(causal=-1), dict(window=-1), dict(causal=0, window=5), dict(size=need - 1), dict(work=8 * P + 8), dict(o=5 * P), dict(lse=5 * P),
               dict(o=7 * P), dict(o=c.k), dict(lse=c.v_scale)):
        assert attend(lib, d, c, **kw) == EINVAL, kw
    for kw in (dict(Hkv=1), dict(dh=128), dict(kernel_mode=256), dict(kernel_mode=3), dict(dtype=2), dict(H=3), dict(Tq=-1), dict(softcap=-1.0)):
        assert attend(lib, desc(**kw), c) == EINVAL, kw
    for kw in (dict(ldq=255), dict(ldo=8), dict(Tq=2 ** 24)):
        assert attend(lib, desc(**kw), c) == ESHAPE, kw
    assert attend(lib, desc(kernel_mode=2), c, q=5 * P + 2) == EUNSUPPORTED and attend(lib, desc(kernel_mode=2, ldo=260), c) == EUNSUPPORTED
    assert attend(lib, desc(kernel_mode=2, dtype=0, dh=144), cache(dh=144)) == EUNSUPPORTED
    assert attend(lib, desc(Tq=0), c, q=None, o=None, lse=None, work=None, size=0) == 0


def test_workspaces_do_not_depend_on_addresses(lib):
    d = desc(Tq=300)
    sizes = {lib.revffn_op_attention_cached_workspace(ctypes.byref(d), ctypes.byref(cache(max_pages=99, **kw))) for kw in (dict(), dict(k=16 * P), dict(table=9 * P))}
    assert len(sizes) == 1 and min(sizes) > 0
    short = desc(Tq=3)                                       # (single tokens of short sequences need none)
    assert lib.revffn_op_attention_cached_workspace(ctypes.byref(short), ctypes.byref(cache())) == 0


def test_integer_products_refuse(lib):
    def quantize(dtype=1, x=P, codes=2 * P, scale=3 * P, rows=5, cols=64, ldx=64, ldc=64):
        return lib.revffn_op_quantize_rows(dtype, x, codes, scale, rows, cols, ldx, ldc, None)
    for kw in (dict(x=None), dict(codes=None), dict(scale=None)):
        assert quantize(**kw) == ENULL
    for kw in (dict(dtype=2), dict(rows=-1), dict(cols=0), dict(cols=2 ** 24 + 1, ldx=2 ** 25, ldc=2 ** 25), dict(codes=P), dict(scale=P)):
        assert quantize(**kw) == EINVAL, kw
    for kw in (dict(ldx=63), dict(ldc=63), dict(rows=2 ** 24)):
        assert quantize(**kw) == ESHAPE, kw
    assert quantize(rows=0, x=None, codes=None, scale=None) == 0

    def product(dtype=1, mode=0, a=P, sa=2 * P, b=3 * P, sb=4 * P, bias=5 * P, c=6 * P, M=5, N=7, K=64, lda=64, ldb=64, ldc=7):
        return lib.revffn_op_gemm_int(dtype, mode, a, sa, b, sb, bias, c, M, N, K, lda, ldb, ldc, None)
    for kw in (dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(c=None)):
        assert product(**kw) == ENULL
    for kw in (dict(dtype=2), dict(mode=3), dict(mode=-1), dict(mode=257), dict(mode=256 * 100), dict(M=-1), dict(N=-1), dict(K=0), dict(c=P), dict(c=3 * P), dict(c=5 * P)):
        assert product(**kw) == EINVAL, kw
    for kw in (dict(K=131072, lda=131072, ldb=131072), dict(lda=63), dict(ldb=48), dict(ldc=6), dict(M=2 ** 28, N=2 ** 10, ldc=2 ** 10)):
        assert product(**kw) == ESHAPE, kw
    for kw in (dict(lda=72), dict(ldb=72), dict(a=P + 8), dict(b=3 * P + 1)):
        assert product(mode=2, **kw) == EUNSUPPORTED and product(mode=256, **kw) == EUNSUPPORTED, kw
    assert product(M=0, a=None, sa=None, c=None) == 0 and product(N=0, b=None, sb=None, c=None) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    u8, f32, i32 = (lambda n, t=t: torch.zeros(n, dtype=t) for t in (torch.uint8, torch.float32, torch.int32))
    good = lambda **kw: dict(k=u8(2 * 2 * 16 * 16), v=u8(2 * 2 * 16 * 16), k_scale=f32(4), v_scale=f32(4), table=i32(3 * 5), len=i32(3), cu=i32(4)) | kw
    sizes = dict(pages=2, page=16, max_pages=5, n_seqs=3, Hkv=2, dh=16)
    R.Cache(**good(), **sizes)
    for kw in (dict(k=u8(1023)), dict(v=f32(1024)), dict(v_scale=f32(3)), dict(table=i32(14)), dict(len=i32(2)), dict(cu=i32(3)),
               dict(k=u8(2048)[::2]), dict(table=i32(30).reshape(3, 10)[:, :5])):
        with pytest.raises(R.RevffnError):
            R.Cache(**good(**kw), **sizes)


def test_eight_bit_numbers_of_the_reference():
    """Against torch's own conversion, every code and every border among the values."""
    codes = np.arange(256).astype(np.uint8)
    theirs = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.decode(codes), theirs, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([ref.VALUES, ref._BETWEEN, -ref._BETWEEN, rng.uniform(-448, 448, 5000), rng.standard_normal(5000) * 2.0 ** -7])
    assert np.array_equal(ref.nearest(x), torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy())
    assert np.isnan(ref.nearest([np.inf, -np.inf, np.nan])).all() and ref.nearest([1e9, -1e9]).tolist() == [448.0, -448.0]
    for m, want in ((448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (1e-40, 2.0 ** -96), (0.0, 2.0 ** -96), (3.4e38, 2.0 ** 119), (1.75, 2.0 ** -8)):
        assert ref.power_for(m) == want


def test_cache_of_the_reference_holds_what_was_appended():
    """Token by token or at once: the same numbers but for those below 2^-6 of a page's unit, and within half a step of what went in."""
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((2, 70, 2, 16))
    v[40:] *= 9
    table = np.array([[3, 0, 4, 1, -1]])
    once, each = ref.Cache(5, 16, 2, 16), ref.Cache(5, 16, 2, 16)
    once.append(table, [70], [70], k, v)
    for j in range(70):
        each.append(table, [j + 1], [1], k[j:j + 1], v[j:j + 1])
    for name, x in (("k", k), ("v", v)):
        a, b = once.rows(name, table, 0, 64), each.rows(name, table, 0, 64)
        unit = np.repeat(once.scale[name][table[0, :4]], 16, 0)[..., None]
        assert (np.abs(a - x[:64]) <= np.maximum(np.abs(x[:64]) * 2.0 ** -4, unit * 2.0 ** -10)).all()
        assert (np.abs(a - b) <= unit * 2.0 ** -9).all() and np.array_equal(a[np.abs(a) >= unit * 2.0 ** -6], b[np.abs(a) >= unit * 2.0 ** -6])
    assert np.isnan(once.rows("k", table, 0, 70)[64:]).all() and np.isnan(once.scale["k"][2]).all()


def test_attention_of_the_reference():
    """Against one dense softmax per row."""
    rng = np.random.default_rng(2)
    c, table = ref.Cache(6, 16, 1, 16), np.array([[5, 2], [0, 3]])
    c.append(table, [20, 31], [20, 31], rng.standard_normal((51, 1, 16)), rng.standard_normal((51, 1, 16)))
    q = rng.standard_normal((4, 2, 16))
    got = ref.attention(c, table, [20, 31], [3, 1], q, window=7, cap=2.0)
    for row, (s, at) in enumerate([(0, 17), (0, 18), (0, 19), (1, 30)]):
        k, v = c.rows("k", table, s, at + 1)[at - 6:, 0], c.rows("v", table, s, at + 1)[at - 6:, 0]
        for h in range(2):
            z = 2.0 * np.tanh(k @ q[row, h] / 4 / 2.0)
            p = np.exp(z)
            assert np.allclose(got["o"][0][row, h], p @ v / p.sum(), rtol=1e-12) and np.isclose(got["lse"][0][h, row], np.log(p.sum()), rtol=1e-12)
    assert operators_reference.outside(got["o"][0], got["o"][0], got["o"][1]) == 0


def test_integers_of_the_reference():
    x = np.array([[1.0, -127.0, 63.5, 2.5, -0.5], [0, 0, 0, 0, 0], [1e-40, 0, 0, 0, 0], [np.inf, 1, 1, 1, 1], [np.nan, 0, 0, 0, 0]])
    codes, scale = ref.quantized(x)
    assert codes[0].tolist() == [1, -127, 64, 2, 0] and scale[0] == 1.0 and scale[1] == scale[2] == 0 and np.isnan(scale[3:]).all() and not codes[1:].any()


# ---- results in the place of results, and calls at the ends of what is allowed -----------------------------------------
def test_rows_to_integers_refuse_codes_in_the_place_of_scales(lib):
    assert lib.revffn_op_quantize_rows(1, P, 3 * P, 3 * P, 5, 64, 64, 64, None) == EINVAL


@pytest.mark.parametrize("kw", [dict(Tk=-1), dict(Tk=2 ** 26), dict(ldk=64), dict(ldk=-5, ldv=1), dict(ldv=1)])
def test_attention_does_not_read_the_keys_fields(lib, kw):
    """The cache says where keys are: whatever the desc holds of them, it is the same call."""
    c = cache(max_pages=400)
    need = lib.revffn_op_attention_cached_workspace(ctypes.byref(desc()), ctypes.byref(c))
    assert lib.revffn_op_attention_cached_workspace(ctypes.byref(desc(**kw)), ctypes.byref(c)) == need > 0
    assert attend(lib, desc(Tq=0, **kw), c, q=None, o=None, lse=None, work=None, size=0) == 0


def test_attention_takes_every_call_that_a_launch_can_hold(lib):
    """Rows times heads, and sequences that have rows times key heads: as the header says, whatever the number of sequences without."""
    size = lambda d, c: lib.revffn_op_attention_cached_workspace(ctypes.byref(d), ctypes.byref(c))
    wide = cache(max_pages=400)
    assert size(desc(Tq=131072, H=128), wide) > 0 and size(desc(Tq=2 ** 19 - 100, H=128), wide) > 0
    many = dict(n_seqs=2 ** 20, Hkv=8, max_pages=400)
    assert size(desc(H=8, Hkv=8), cache(**many)) > 0 and size(desc(Tq=2 ** 20, H=8, Hkv=8), cache(**many)) > 0
    assert size(desc(Tq=2 ** 20, H=16, Hkv=16), cache(**many | dict(Hkv=16))) == 0
    assert attend(lib, desc(Tq=2 ** 20, H=16, Hkv=16), cache(**many | dict(Hkv=16))) == ESHAPE
    assert attend(lib, desc(Tq=2 ** 19, H=128), wide) == ESHAPE


def test_append_refuses_more_than_a_launch_can_hold(lib):
    """2^32 threads and more: for pages that get rows times key heads, for queries; of eight waves per page and head (and odd numbers of heads) too."""
    c = cache(n_seqs=2 ** 20, Hkv=64)
    assert append(lib, c, T=2 ** 20, ldk=4096, ldv=4096) == ESHAPE and append(lib, cache(), T=2 ** 26) == ESHAPE
    assert append(lib, cache(n_seqs=2 ** 20, Hkv=3, dh=128, page=128), T=2 ** 20, q=None, q_out=None, ldk=384, ldv=384) == ESHAPE


def test_integer_products_refuse_more_than_a_launch_can_hold(lib):
    def product(M, N, mode=0, lda=16):
        return lib.revffn_op_gemm_int(1, mode, P, 2 * P, 3 * P, 4 * P, None, 6 * P, M, N, 16, lda, lda, N, None)
    for M, N in ((2 ** 30, 1), (1, 2 ** 30), (2 ** 18, 2 ** 18), (2 ** 31 - 1, 2 ** 31 - 1)):
        for mode in (0, 1, 2, 256, 256 * 5):
            assert product(M, N, mode) == ESHAPE and (mode >= 2 or product(M, N, mode, lda=17) == ESHAPE)
    assert product(2 ** 17, 2 ** 17, 256 * 5) == ESHAPE and product(1, 2 ** 30 - 1, 256 * 4) == ESHAPE      # (more tiles than a launch can have)


def _kernels(path):
    """{name: (registers spilled, bytes of private memory)} of every kernel in a library built here."""
    data, out = open(path, "rb").read(), {}
    for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data):
        at = m.end() + 8
        for _ in range(struct.unpack_from("<Q", data, m.end())[0]):
            offset, size, length = struct.unpack_from("<3Q", data, at)
            target = data[at + 24:at + 24 + length]
            at += 24 + length
            if not target.endswith(b"gfx950"):
                continue
            with tempfile.NamedTemporaryFile(suffix=".elf") as f:
                f.write(data[m.start() + offset:m.start() + offset + size])
                f.flush()
                notes = subprocess.run(["/opt/rocm/llvm/bin/llvm-readelf", "--notes", f.name], capture_output=True, text=True, check=True).stdout
            for block in notes.split("  - .agpr_count:")[1:]:
                field = lambda n: re.search(rf"^ +\.{n}: +(\S+)", block, re.M).group(1)
                out[field("name")] = (int(field("vgpr_spill_count")), int(field("private_segment_fixed_size")))
    return out


def test_no_kernel_of_the_cache_spills_registers(lib):
    """A rule of those kernels: the first ones that spilled gave wrong results, and spills in their loops would cost more than the forms that do without."""
    kernels = {n: x for n, x in _kernels(R.library_path()).items() if "cached_" in n or "cache_append" in n or "gemm_i8" in n or "quantize_rows" in n}
    assert len(kernels) > 100 and not {n for n, x in kernels.items() if x != (0, 0)}
