"""Host checks of the backbone operators: what they refuse, their plan and struct layout.  No device calls: every
refused call returns before its first one."""
import ctypes
import subprocess

import numpy as np
import pytest
import torch
from torch.autograd import forward_ad

from paper_2607_14695_amd import reflex as R
from paper_2607_14695_amd.paged import PagedBatch, PagedCache, Rotary

from . import paged_reference as ref

A = 1 << 20  # an aligned address that is never read


def cache_c(**kw):
    f = dict(k=A, v=A, k_scale=None, v_scale=None, n_pages=4, page_size=16, n_kv_heads=2, head_dim=64,
             store=R.STORE_BF16, reserved=0)
    f.update(kw)
    return R.PagedCacheC(**f)


def batch_c(**kw):
    f = dict(cu_rows=A, lengths=A, page_table=A, n_seqs=2, max_pages=3, max_length=0, reserved=0)
    f.update(kw)
    return R.PagedBatchC(**f)


def rows_c(data=A, rs=128, hs=64):
    return R.RowsC(data, rs, hs)


def write(cache=None, batch=None, k=None, v=None, n=0, dtype=R.DTYPE_BF16, rotary=None, pos=None):
    b = ctypes.byref
    return R.load_library().reflex_paged_write(b(cache or cache_c()), b(batch or batch_c()), b(k or rows_c()),
                                               b(v or rows_c()), n, dtype, b(rotary) if rotary else None, pos, 0, None)


def read(cache=None, batch=None, k=None, v=None, n=0, dtype=R.DTYPE_BF16):
    b = ctypes.byref
    return R.load_library().reflex_paged_read(b(cache or cache_c()), b(batch or batch_c()), b(k or rows_c()),
                                              b(v or rows_c()), n, dtype, None)


def attend(cache=None, batch=None, q=None, o=None, n=0, heads=4, dtype=R.DTYPE_BF16, scale=0.125, window=0, ws=None,
           nb=0):
    b = ctypes.byref
    return R.load_library().reflex_paged_attention(b(cache or cache_c()), b(batch or batch_c()), b(q or rows_c()),
                                                   b(o or rows_c()), n, heads, dtype, scale, 1, window, ws, nb, None)


def plan(head_dim=64, sections=(32,)):
    return Rotary(head_dim, sections).c


def test_empty_calls_are_done():
    assert write() == read() == attend() == R.REFLEX_OK
    assert write(batch=batch_c(n_seqs=0), n=5) == R.REFLEX_OK
    r = rows_c()
    assert R.load_library().reflex_rotary_apply(ctypes.byref(plan()), None, 0, ctypes.byref(r), ctypes.byref(r), 0, 4,
                                                R.DTYPE_BF16, 0, None) == R.REFLEX_OK


@pytest.mark.parametrize("bad", [
    dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 2), dict(n_pages=0), dict(page_size=0), dict(page_size=24),
    dict(page_size=2048), dict(n_kv_heads=0), dict(n_kv_heads=1 << 17), dict(head_dim=96), dict(head_dim=512),
    dict(store=4), dict(store=-1), dict(store=R.STORE_FP8), dict(store=R.STORE_INT8, k_scale=A),
    dict(store=R.STORE_INT8, k_scale=A, v_scale=A + 2), dict(n_pages=1 << 26)])
def test_bad_caches(bad):
    for call in (write, read, attend):
        assert call(cache=cache_c(**bad), n=1) == R.REFLEX_EINVAL


@pytest.mark.parametrize("bad", [
    dict(cu_rows=None), dict(lengths=None), dict(page_table=None), dict(n_seqs=-1), dict(max_pages=-1),
    dict(max_length=-1), dict(max_pages=1 << 27)])
def test_bad_batches(bad):
    for call in (write, read, attend):
        assert call(batch=batch_c(**bad), n=1) == R.REFLEX_EINVAL


@pytest.mark.parametrize("r", [rows_c(data=None), rows_c(data=A + 8), rows_c(rs=129), rows_c(hs=4)])
def test_bad_rows(r):
    assert write(k=r, n=1) == write(v=r, n=1) == read(k=r, n=1) == read(v=r, n=1) == R.REFLEX_EINVAL
    assert attend(q=r, n=1) == attend(o=r, n=1) == R.REFLEX_EINVAL
    ok, p = rows_c(), plan()
    for x, y in ((r, ok), (ok, r)):
        assert R.load_library().reflex_rotary_apply(ctypes.byref(p), A, 0, ctypes.byref(x), ctypes.byref(y), 1, 2,
                                                    R.DTYPE_BF16, 0, None) == R.REFLEX_EINVAL


def test_bad_scalars_and_types():
    for call in (write, read, attend):
        assert call(n=-1) == call(n=(1 << 27) + 1) == call(n=1, dtype=2) == R.REFLEX_EINVAL
        assert call(n=1, dtype=R.DTYPE_F32) == R.REFLEX_EDTYPE
        assert call(cache=cache_c(store=R.STORE_F32), n=1) == R.REFLEX_EDTYPE
    for heads in (0, -2, 3, 1 << 25):
        assert attend(n=2, heads=heads) == R.REFLEX_EINVAL
    assert attend(n=1, scale=float("nan")) == attend(n=1, scale=float("inf")) == R.REFLEX_EINVAL
    assert attend(n=1, window=-1) == R.REFLEX_EINVAL
    assert write(n=1, rotary=plan(128, (64,))) == R.REFLEX_EINVAL  # another head_dim
    assert write(n=1, pos=A) == R.REFLEX_EINVAL  # positions without a plan
    broken = plan()
    broken.axis[3] = 7
    assert write(n=1, rotary=broken) == R.REFLEX_EINVAL


def test_null_structs():
    lib, b = R.load_library(), ctypes.byref
    c, q, r = cache_c(), batch_c(), rows_c()
    assert lib.reflex_paged_read(None, b(q), b(r), b(r), 1, 1, None) == R.REFLEX_EINVAL
    assert lib.reflex_paged_read(b(c), None, b(r), b(r), 1, 1, None) == R.REFLEX_EINVAL
    assert lib.reflex_paged_read(b(c), b(q), None, b(r), 1, 1, None) == R.REFLEX_EINVAL
    assert lib.reflex_paged_attention_workspace(b(c), b(q), 1, 4, 1, None) == R.REFLEX_EINVAL
    assert lib.reflex_rotary_apply(None, A, 0, b(r), b(r), 1, 1, 1, 0, None) == R.REFLEX_EINVAL
    assert lib.reflex_rotary_apply(b(plan()), None, 0, b(r), b(r), 1, 1, 1, 0, None) == R.REFLEX_EINVAL


def test_workspace_is_required_and_checked():
    """A single row over a long memory splits its keys: the call names its bytes and refuses less."""
    lib, b = R.load_library(), ctypes.byref
    c, q = cache_c(n_pages=4096), batch_c(max_pages=1024, n_seqs=1)
    need = ctypes.c_size_t(0)
    assert lib.reflex_paged_attention_workspace(b(c), b(q), 1, 4, R.DTYPE_BF16, b(need)) == R.REFLEX_OK
    assert need.value > 0
    for ws, nb in ((None, need.value), (A, need.value - 1), (A + 16, need.value)):
        assert attend(cache=c, batch=q, n=1, ws=ws, nb=nb) == R.REFLEX_EINVAL
    # a longer memory never needs less, and a huge batch needs no more than its rows' partials
    more = ctypes.c_size_t(0)
    assert lib.reflex_paged_attention_workspace(b(c), b(q), 4096, 4, R.DTYPE_BF16, b(more)) == R.REFLEX_OK
    assert more.value <= 4096 * 4 * 64 * (64 + 2) * 4


@pytest.mark.parametrize("args", [
    (60, (30,)), (0, (0,)), (272, (136,)), (64, (31,)), (64, (33,)), (64, (-1, 33)), (64, ()), (64, (8, 8, 8, 4, 4))])
def test_bad_rotary_plans(args):
    with pytest.raises(R.ReflexError):
        Rotary(*args)


def test_bad_rotary_options():
    with pytest.raises(ValueError):
        Rotary(64, ladder="interleaved")
    for theta in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(R.ReflexError):
            Rotary(64, theta=theta)


@pytest.mark.parametrize("ladder", ["shared", "per_axis"])
@pytest.mark.parametrize("dh,sections", [(64, (32,)), (80, (10, 15, 15)), (256, (32, 0, 48, 48))])
def test_rotary_plan_values(dh, sections, ladder):
    p = Rotary(dh, sections, theta=500.0, ladder=ladder).c
    # at position 1 on every axis the angle is 2 pi * turns
    ang = ref.rotary_angles(np.ones((len(sections), 1)), sections, 500.0, ladder, dh // 2)[0]
    np.testing.assert_allclose(np.array(p.turns[:dh // 2]) * 2 * np.pi, ang, rtol=4 * 2.0 ** -52)
    axis = np.repeat(np.arange(len(sections)), sections)
    assert list(p.axis[:dh // 2]) == axis.tolist()


def test_python_refusals():
    """The binding refuses tensors that are not what the call takes before it makes one."""
    t32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        PagedBatch(t32(3), t32(2), t32(2, 4))  # not on a GPU
    with pytest.raises(ValueError):
        PagedBatch(t32(3), t32(2), t32(8))
    with pytest.raises(ValueError):
        PagedCache(torch.zeros(2, 1, 16, 64), torch.zeros(2, 1, 16, 64))  # not on a GPU
    with pytest.raises(ValueError):
        PagedCache(torch.zeros(2, 1, 16, 64, dtype=torch.float16), torch.zeros(2, 1, 16, 64, dtype=torch.float16))
    with pytest.raises(ValueError):
        PagedCache(torch.zeros(2, 1, 16, 64, dtype=torch.int8), torch.zeros(2, 1, 16, 64, dtype=torch.int8))
    rot, pos = Rotary(64), torch.zeros(4, dtype=torch.int64)
    x = torch.zeros(4, 2, 64)
    for bad in (x[0], torch.zeros(4, 2, 128), x.half(), x.clone().requires_grad_(), x):
        with pytest.raises(ValueError):
            rot.apply(bad, pos)


def test_struct_sizes_match_c_layout(tmp_path):
    structs = {"reflex_rows": R.RowsC, "reflex_rotary": R.RotaryC, "reflex_paged_cache": R.PagedCacheC,
               "reflex_paged_batch": R.PagedBatchC}
    lines = ['#include <stddef.h>', '#include <stdio.h>', f'#include "{R.HEADER_PATH}"', "int main(void) {"]
    for cname, py in structs.items():
        lines.append(f'  printf("{cname} size %zu\\n", sizeof({cname}));')
        lines += [f'  printf("{cname} {f[0]} %zu\\n", offsetof({cname}, {f[0]}));' for f in py._fields_]
    lines += ["  return 0;", "}"]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines) + "\n")
    subprocess.run(["gcc", "-std=c99", "-o", str(exe), str(src)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    got = {tuple(line.split()[:2]): int(line.split()[2]) for line in out if line.strip()}
    for cname, py in structs.items():
        assert got[(cname, "size")] == ctypes.sizeof(py), cname
        for f in py._fields_:
            assert got[(cname, f[0])] == getattr(py, f[0]).offset, (cname, f[0])


def test_reference_quantiser_on_known_values():
    """The oracle itself, on rows worked out by hand."""
    v, s = ref.encode_row(np.array([127.0, 0.5, 1.5, -2.5, 0.0]), "int8")
    assert s == 1.0 and v.tolist() == [127, 0, 2, -2, 0]
    v, s = ref.encode_row(np.array([448.0, 17.0, 19.0, -0.001, 2.0 ** -10]), "fp8")
    assert s == 1.0 and v.tolist() == [448, 16, 20, -2.0 ** -9 * 1 if 0.001 > 2.0 ** -10 else 0, 0]
    assert ref.encode_row(np.array([449.0]), "fp8")[1] == 2.0
    assert np.isnan(ref.encode_row(np.array([1.0, np.inf]), "int8")[1])
    v, s = ref.encode_row(np.zeros(4), "fp8")
    assert s == 2.0 ** -126 and not v.any()


def test_scales_past_fp32_are_refused():
    """The scale enters the exponent times log2(e), which has to be finite in fp32 too."""
    for scale in (2.4e38, 3.4e38, -3.4e38):
        assert attend(n=0, scale=scale) == R.REFLEX_EINVAL
    for scale in (2.3e38, -2.3e38, 0.0, 1e-45):
        assert attend(n=0, scale=scale) == R.REFLEX_OK


def test_tangents_are_refused():
    """Forward-mode differentiation: a tangent would be dropped without a word, with gradients recorded or not."""
    rot, pos, x = Rotary(64), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 2, 64)
    with forward_ad.dual_level():
        d = forward_ad.make_dual(x, torch.ones_like(x))
        for call in (lambda: rot.apply(d, pos), lambda: rot.apply(x, pos, out=d)):
            with pytest.raises(ValueError, match="tangent"):
                call()
            with torch.no_grad(), pytest.raises(ValueError, match="tangent"):
                call()


def test_integers_that_do_not_fit_are_refused():
    """Python's integers are not cut to 32 bits on their way into the C structs."""
    with pytest.raises(ValueError, match="sections"):
        Rotary(64, (2 ** 32 + 32,))
    with pytest.raises(ValueError, match="head_dim"):
        Rotary(2 ** 32 + 64, (32,))
    t32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    for length in (2 ** 32, 2 ** 32 + 5, -2 ** 32):
        with pytest.raises(ValueError, match="max_length"):
            PagedBatch(t32(3), t32(2), t32(2, 4), length)


@pytest.mark.parametrize("rows,heads,dtype,store,max_length,splits", [
    # 128 keys at least to a split, at most 64 splits
    (1, 4, R.DTYPE_BF16, R.STORE_BF16, 128, 1), (1, 4, R.DTYPE_BF16, R.STORE_BF16, 129, 2),
    (1, 4, R.DTYPE_BF16, R.STORE_BF16, 8192, 64), (1, 4, R.DTYPE_BF16, R.STORE_BF16, 8193, 33),
    (1, 4, R.DTYPE_BF16, R.STORE_BF16, 0, 64), (1, 4, R.DTYPE_F32, R.STORE_F32, 16384, 64),
    # 4,096 rows of two heads on each of two K/V heads: 128 tiles of 128 rows, or 512 of 32 in fp32; 512 workgroups
    (4096, 4, R.DTYPE_BF16, R.STORE_BF16, 0, 4), (4096, 4, R.DTYPE_F32, R.STORE_F32, 0, 1),
    (4096, 4, R.DTYPE_BF16, R.STORE_INT8, 500, 4), (4096, 4, R.DTYPE_BF16, R.STORE_INT8, 300, 3)])
def test_workspace_bytes(rows, heads, dtype, store, max_length, splits):
    """Exactly the partial sums (head_dim and two fp32 a row, head and split) of the splits that a call makes.  A longer
    memory may need less: 64 splits of 128 keys hold 8,192, and 8,193 take 33 of 256."""
    need, b = ctypes.c_size_t(0), ctypes.byref
    scales = dict(k_scale=A, v_scale=A) if store == R.STORE_INT8 else {}
    c, q = cache_c(n_pages=4096, store=store, **scales), batch_c(max_pages=1024, n_seqs=1, max_length=max_length)
    assert R.load_library().reflex_paged_attention_workspace(b(c), b(q), rows, heads, dtype, b(need)) == R.REFLEX_OK
    assert need.value == (0 if splits == 1 else rows * heads * splits * (64 + 2) * 4)
