"""CPU-side checks of decoding from 8-bit pages: the oracle against closed forms, the refusals of the entry points."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from oracle import infoflow_oracle as O
from oracle import pages_oracle as P
from paper_2603_05353_amd import binding as B


# ---- the oracle -----------------------------------------------------------------------------------------------
def test_e4m3_is_torchs_float8():
    grid = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(P.E4M3, grid, equal_nan=True)
    # every number, every midpoint of neighbours (ties), and both sides of it
    pos = P.E4M3[:0x7F]
    mid = (pos[1:] + pos[:-1]) / 2
    x = np.concatenate([pos, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20)])
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(P.to_e4m3(x), want)
    assert np.array_equal(P.to_e4m3([np.nan, np.inf, -np.inf]), [0x7F] * 3)


def test_value_order_is_a_permutation():
    assert sorted(P.ORDER.tolist()) == list(range(64)) and tuple(P.ORDER) == B.VALUE_BYTE
    # the sixteen tokens of a lane group: four of each block of sixteen
    for g in range(4):
        assert {t for t in range(64) if P.ORDER[t] // 16 == g} == {16 * i + 4 * g + j for i in range(4) for j in range(4)}


@pytest.mark.parametrize("top,e", [(0.0, -100), (448.0, 0), (448.0001, 1), (447.0, 0), (224.0, -1), (224.5, 0), (1.0, -8),
                                   (1.75, -8), (1.7501, -7), (1e-45, -100), (2.0 ** -95, -100), (3.38e38, 120)])
def test_scale_is_the_smallest_power_of_two(top, e):
    assert P.scale_for([0.0, -top, np.nan, np.inf]) == 2.0 ** e


def test_equal_coordinates_are_the_one_axis_embedding():
    g = np.random.default_rng(3)
    x, pos, freq = g.standard_normal((5, 3, 64)), g.integers(0, 70000, 5), 1e4 ** (-np.arange(32) / 32)
    for pairing in ("half", "interleaved"):
        a = P.rope_rows_axes(x, np.stack([pos] * 3, 1), [j % 3 for j in range(32)], freq, pairing)
        b = P.rope_rows_axes(x, pos[:, None], [0] * 32, freq, pairing)
        assert np.array_equal(a, b)
        z = (x[..., :32] + 1j * x[..., 32:] if pairing == "half" else x[..., 0::2] + 1j * x[..., 1::2])
        z = z * np.exp(1j * pos[:, None] * freq)[:, None, :]
        got = a[..., :32] + 1j * a[..., 32:] if pairing == "half" else a[..., 0::2] + 1j * a[..., 1::2]
        assert np.abs(got - z).max() < 1e-12


def test_attention_over_pages_is_attention_over_rows():
    """Rows whose values e4m3 holds, stored in two steps, against the oracle of the dense path."""
    g = np.random.default_rng(4)
    n, hkv, hq, d = 150, 2, 6, 64
    k, v = (P.E4M3[P.to_e4m3(np.clip(g.standard_normal((n, hkv, d)), -4, 4))] for _ in range(2))
    k[0, :, 0], v[0, :, 0], k[100, :, 0], v[100, :, 0] = 4, 4, 4, 4         # the same scale in every page and both steps
    k[64, :, 0], v[64, :, 0], k[128, :, 0], v[128, :, 0] = 4, 4, 4, 4
    pool = dict(k=np.zeros((4, hkv, 64, d), np.uint8), v=np.zeros((4, hkv, d, 64), np.uint8), k_scale=np.ones((4, hkv)), v_scale=np.ones((4, hkv)))
    table = np.array([[2, 0, 3]])
    pool = P.store_pages(pool, table, [0], np.arange(100), k, v, row_start=[0, 100])
    pool = P.store_pages(pool, table, [100], np.arange(100, n), k[100:], v[100:], row_start=[0, 50])
    q, pos = g.standard_normal((4, hq, d)), np.array([0, 63, 64, 149])
    out, lse, _, _ = P.attend_pages(q, pos, pool, table, 0.2, row_start=[0, 4])
    ref, ref_lse = O.recompute_attention(q, pos, k, v, 0.2)
    # the first step's scale is that of its rows: values within half a step, 2^-4
    assert np.abs(out - ref).max() < 2.0 ** -4 * 4 and np.abs(lse - ref_lse).max() < 2.0 ** -4 * 0.2 * np.abs(q).sum(-1).max() * 4
    sizes = [P.scale_for(k[:, 0])]
    assert sizes[0] == 2.0 ** -6


# ---- the entry points -------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2603_05353_amd.build import build_library
        build_library()
    return B.load_library()


@pytest.fixture()
def layer(lib):
    L = B.Layer("bf16", 32, 8, 128, 5e5, max_ctx=4096, max_prompt=64)
    yield L
    L.close()


def fake(off=0):
    return C.c_void_p(4096 + off)


def desc(n_pages=8, **kw):
    d = B.PageCacheDesc(4096, 8192, 4096, 4096, n_pages)
    for k, v in kw.items():
        setattr(d, k, v)
    return C.byref(d)


def refused(layer, rc, code, *words):
    assert rc == code, (rc, layer._lib.ifkv_last_error(layer._ctx))
    for w in words:
        assert w in layer._lib.ifkv_last_error(layer._ctx).decode()


def test_store_pages_refusals(layer):
    f, call = fake(), layer._lib.ifkv_store_pages
    def store(pages=desc(), table=f, n_seqs=2, width=4, kv_len=f, start=f, pos=f, n=3, k=f, v=f, ks=0, vs=0):
        return call(layer._ctx, pages, table, n_seqs, width, kv_len, start, pos, n, k, v, ks, vs)
    E, S = B.IFKV_EINVAL, B.IFKV_ESHAPE
    assert call(None, desc(), f, 2, 4, f, f, f, 3, f, f, 0, 0) == E
    refused(layer, store(pages=None), E, "pages is NULL")
    refused(layer, store(pages=desc(-1)), E, "n_pages")
    refused(layer, store(pages=desc(1 << 31)), S, "too many pages")
    for name in ("k", "v", "k_scale", "v_scale"):
        refused(layer, store(pages=desc(**{name: None})), E, "NULL")
    refused(layer, store(pages=desc(v=8200)), E, "aligned")
    for kw in (dict(n_seqs=-1), dict(width=-1), dict(n=-1)):
        refused(layer, store(**kw), E, "negative")
    refused(layer, store(n=1 << 31), S, "too many rows")
    refused(layer, store(width=65), S, "max_ctx")            # 4096 tokens are 64 pages
    refused(layer, store(start=None), E, "row_start")        # three rows of two sequences
    for name in ("table", "kv_len", "pos", "k", "v"):
        refused(layer, store(**{name: None}), E, "NULL")
    refused(layer, store(k=fake(8)), E, "aligned")
    for kw in (dict(ks=1023), dict(vs=1020), dict(ks=1028), dict(vs=-1024), dict(ks=1 << 41)):
        refused(layer, store(**kw), E, "strides")
    assert store(n=0, k=None, v=None, kv_len=None) == 0
    assert store(n_seqs=0, k=None) == 0
    assert store(width=0, table=None) == 0 and store(pages=desc(0, k=None, v=None, k_scale=None, v_scale=None)) == 0   # no page: all rows dropped


def test_attend_pages_refusals(layer):
    f, call = fake(), layer._lib.ifkv_attend_pages
    def attend(pages=desc(), table=f, n_seqs=2, width=4, start=f, most=2, q=f, qs=0, pos=f, n=3, out=f, lse=None):
        return call(layer._ctx, pages, table, n_seqs, width, start, most, q, qs, pos, n, out, lse)
    E, S = B.IFKV_EINVAL, B.IFKV_ESHAPE
    assert call(None, desc(), f, 2, 4, f, 2, f, 0, f, 3, f, None) == E
    refused(layer, attend(pages=None), E, "pages is NULL")
    refused(layer, attend(pages=desc(k=4100)), E, "aligned")
    for kw in (dict(n_seqs=-1), dict(width=-1), dict(n=-1)):
        refused(layer, attend(**kw), E, "negative")
    refused(layer, attend(most=0), E, "max_rows")
    refused(layer, attend(width=65), S, "max_ctx")
    refused(layer, attend(start=None), E, "row_start")
    for name in ("table", "pos", "q", "out"):
        refused(layer, attend(**{name: None}), E, "NULL")
    refused(layer, attend(q=fake(4)), E, "aligned")
    refused(layer, attend(out=fake(2)), E, "aligned")
    for qs in (4095, 4092, 4100, -4096):
        refused(layer, attend(qs=qs), E, "q_stride")
    assert attend(n=0, q=None, out=None) == 0 and attend(n_seqs=0, q=None, out=None) == 0


def test_copy_pages_refusals(layer):
    call = layer._lib.ifkv_copy_pages
    arr = lambda *x: (C.c_int32 * len(x))(*x)   # noqa: E731
    E = B.IFKV_EINVAL
    assert call(None, desc(), 1, arr(0), arr(1)) == E
    refused(layer, call(layer._ctx, desc(), -1, arr(0), arr(1)), E, "negative")
    refused(layer, call(layer._ctx, desc(), 1, None, arr(1)), E, "NULL")
    refused(layer, call(layer._ctx, desc(), 1, arr(0), None), E, "NULL")
    for s, d in ((0, 8), (8, 0), (-1, 0), (0, -1)):
        refused(layer, call(layer._ctx, desc(), 1, arr(s), arr(d)), E, "outside")
    refused(layer, call(layer._ctx, desc(), 2, arr(0, 1), arr(3, 3)), E, "twice in dst")
    refused(layer, call(layer._ctx, desc(), 2, arr(0, 1), arr(1, 2)), E, "in src and in dst")
    refused(layer, call(layer._ctx, desc(), 1, arr(5), arr(5)), E, "in src and in dst")
    refused(layer, call(layer._ctx, desc(), 9, arr(*[0] * 9), arr(*range(9))), E, "twice")
    assert call(layer._ctx, desc(), 0, None, None) == 0


def test_rope_rows_axes_refusals(layer):
    call = layer._lib.ifkv_rope_rows_axes
    axes = (C.c_int32 * 64)(*[j % 3 for j in range(64)])
    ap, f, E = C.cast(axes, C.c_void_p), fake(), B.IFKV_EINVAL
    assert call(None, f, f, 3, ap, 4, 40, 0) == E
    refused(layer, call(layer._ctx, f, f, 2, ap, 4, 40, 0), E, "axis_of_pair[2]")
    axes[7] = -1
    refused(layer, call(layer._ctx, f, f, 3, ap, 4, 40, 0), E, "axis_of_pair[7]")
    axes[7] = 0
    for n_axes in (0, 9, -1):
        refused(layer, call(layer._ctx, f, f, n_axes, ap, 4, 40, 0), E, "n_axes")
    refused(layer, call(layer._ctx, f, f, 3, None, 4, 40, 0), E, "NULL")
    refused(layer, call(layer._ctx, None, f, 3, ap, 4, 40, 0), E, "NULL")
    refused(layer, call(layer._ctx, f, None, 3, ap, 4, 40, 0), E, "NULL")
    refused(layer, call(layer._ctx, fake(8), f, 3, ap, 4, 40, 0), E, "aligned")
    refused(layer, call(layer._ctx, f, f, 3, ap, -1, 40, 0), E, "n_rows")
    refused(layer, call(layer._ctx, f, f, 3, ap, 4, 0, 0), E, "n_heads")
    for stride in (40 * 128 - 8, 40 * 128 + 4, -1):
        refused(layer, call(layer._ctx, f, f, 3, ap, 4, 40, stride), E, "row_stride")
    refused(layer, call(layer._ctx, f, f, 3, ap, 1 << 31, 40, 0), B.IFKV_ESHAPE, "too many rows")
    assert call(layer._ctx, None, None, 3, ap, 0, 40, 0) == 0


def test_rope_rows_axes_refuses_rows_that_pass_32_bits(layer):
    axes = (C.c_int32 * 64)()
    rc = layer._lib.ifkv_rope_rows_axes(layer._ctx, fake(), fake(), 1, C.cast(axes, C.c_void_p), 4, 1 << 24, 0)
    refused(layer, rc, B.IFKV_ESHAPE, "too many heads")      # 2^24 heads of 128


def test_binding_takes_no_tensor_of_another_kind(layer):
    """What the C call cannot see: devices, types, shapes and layouts (CPU tensors stand for the wrong device)."""
    f8 = torch.float8_e4m3fn
    pool = B.PageCache(torch.zeros(2, 8, 64, 128).to(f8), torch.zeros(2, 8, 128, 64).to(f8), torch.ones(2, 8), torch.ones(2, 8))
    i = lambda *x: torch.zeros(*x, dtype=torch.int32)   # noqa: E731
    q = torch.zeros(1, 32, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="table"):
        layer.attend_pages(q, i(1), pool, i(1, 4), out=q)
    with pytest.raises(ValueError, match="table"):
        layer.store_pages(pool, i(1, 4), i(1), q[:, :8], q[:, :8], i(1))
    with pytest.raises(ValueError, match="pages.k"):
        layer.copy_pages(pool, [0], [1])
    with pytest.raises(ValueError, match="dst"):
        layer.copy_pages(pool, [0], [1, 0])
    with pytest.raises(ValueError, match="src"):
        layer.copy_pages(pool, i(1).long(), i(1))
    with pytest.raises(ValueError, match="axes"):
        layer.rope_rows_axes(q, i(1, 3), i(63))
    with pytest.raises(ValueError, match="pos"):
        layer.rope_rows_axes(q, i(1), i(64))
    with pytest.raises(ValueError, match="x:"):
        layer.rope_rows_axes(q, i(1, 3), i(64))
    assert B.IFKV_PAGE_TOKENS == 64
