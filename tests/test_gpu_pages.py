"""Decoding from 8-bit pages on the GPU against the fp64 oracle: rotary positions with several axes, rows into pages, attention
over pages, pages onto pages, and the four together."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as P
from paper_2603_05353_amd import IFKV_FLAG_FORCE_GENERIC, IFKV_FLAG_VALIDATE, IfkvError, Layer
from tests.helpers import DEV, to_host_f64
from tests.pages_helpers import (assert_attended, assert_same_pool, gen, i32, make_table, pool_to_device, pool_to_host,
                                 random_pool, stored)

pytestmark = pytest.mark.gpu

THETA = 1e6
SHAPES = [("bf16", 32, 8, 128), ("bf16", 28, 4, 128), ("bf16", 5, 5, 128), ("bf16", 16, 2, 64), ("f32", 8, 8, 64), ("f32", 12, 4, 128),
          ("bf16", 40, 1, 128)]


def layer(dtype, hq, hkv, d, max_ctx=1 << 20, **kw):
    return Layer(dtype, hq, hkv, d, THETA, max_ctx=max_ctx, max_prompt=1, **kw)


def parts_of(dtype, columns):
    """bf16 numbers that hold a weight in the second product."""
    return 3 if dtype == "f32" else 2 if columns <= 32 else 1


# ---- rotary positions ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("pairing", ["half", "interleaved"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("rows,heads,extra,n_axes", [(1, 1, 0, 3), (7, 5, 2, 3), (260, 3, 0, 2), (33, 40, 8, 8), (8200, 2, 1, 3)])
def test_rope_rows_axes(pairing, dtype, d, rows, heads, extra, n_axes):
    g = gen(rows * 131 + heads)
    x64, x = stored(g.standard_normal((rows, heads + extra, d)), dtype)
    pos = g.integers(-40, 1 << 17, (rows, n_axes))
    pos[0] = [0, 2 ** 31 - 1, -2 ** 31, 5, 6, 7, 8, 9][:n_axes]
    axes = g.integers(0, n_axes, d // 2)
    L = layer(dtype, 8, 8, d, pairing=pairing)
    before = x.clone()
    got = L.rope_rows_axes(x[:, :heads], i32(pos), torch.tensor(axes, dtype=torch.int32))
    assert got.data_ptr() == x.data_ptr()
    torch.cuda.synchronize()
    freq = THETA ** (-2.0 * np.arange(d // 2) / d)
    want = P.rope_rows_axes(x64[:, :heads], pos, axes, freq, pairing)
    assert torch.equal(x[:, heads:], before[:, heads:])                      # what lies between the rows is not touched
    # cos and sin rounded to fp32 (2^-24 each, after an fp64 angle below 2^31: 2^-22 of a turn), two fp32 operations, one rounding to storage
    size = np.abs(x64[:, :heads])
    pair = np.roll(size, d // 2, -1) if pairing == "half" else size.reshape(rows, heads, d // 2, 2)[..., ::-1].reshape(size.shape)
    tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want) + (4 * 2.0 ** -24 + 2.0 ** -21) * (size + pair)
    assert (np.abs(to_host_f64(x[:, :heads], dtype) - want) <= tol).all()
    L.close()


def test_rope_rows_axes_of_equal_coordinates_is_rope_rows():
    g = gen(5)
    L = layer("bf16", 8, 8, 128)
    _, x = stored(g.standard_normal((65, 8, 128)), "bf16")
    y, pos = x.clone(), i32(g.integers(0, 100000, 65))
    L.rope_rows(x, pos)
    L.rope_rows_axes(y, pos[:, None].repeat(1, 3).contiguous(), torch.arange(64, dtype=torch.int32) % 3)
    assert torch.equal(x, y)
    L.close()


# ---- rows into pages ------------------------------------------------------------------------------------------------
def store_case(dtype, hkv, d, lens, rows, seed, extra=0, flags=0, spoil=False):
    """Rows at given tokens of sequences that hold `lens` before; returns pools after, from device and oracle."""
    g = gen(seed)
    n_pages = sum(-(-max([n] + [p + 1 for p in ps if p >= 0]) // 64) for n, ps in zip(lens, rows)) + 3
    pool = random_pool(g, n_pages, hkv, d)
    tops = [max([n] + [p + 1 for p in ps]) for n, ps in zip(lens, rows)]
    table = make_table(g, tops, n_pages)
    start = np.concatenate([[0], np.cumsum([len(r) for r in rows])])
    pos = np.concatenate([np.asarray(r, dtype=np.int64) for r in rows] + [np.zeros(extra, dtype=np.int64)])
    n = len(pos)
    mag = 2.0 ** g.uniform(-12, 4, (n, hkv, 1))
    kx, vx = g.standard_normal((n, hkv, d)) * mag, g.standard_normal((n, hkv, d)) * mag[::-1]
    if spoil:
        kx[0, 0, 3], vx[n // 2, -1, 5], vx[0, 0, :] = np.nan, np.inf, 0.0
        kx[-1, 0, :] = -np.inf
    k64, k = stored(kx, dtype)
    v64, v = stored(vx, dtype)
    L = layer(dtype, hkv, hkv, d, flags=flags)
    pages = pool_to_device(pool)
    args = (pages, i32(table), i32(lens), k, v, i32(pos))
    L.store_pages(*args, row_start=i32(start))
    torch.cuda.synchronize()
    want = P.store_pages(pool, table, lens, pos, k64, v64, row_start=start)
    return L, pages, args, start, want


@pytest.mark.parametrize("dtype,hkv,d", [("bf16", 8, 128), ("bf16", 3, 64), ("f32", 2, 128), ("f32", 4, 64)])
@pytest.mark.parametrize("lens,rows", [
    ([0], [[0]]), ([63], [[63]]), ([64], [[64]]), ([100], [[100]]),                      # one token: first of a cache, last and first of a page, inside
    ([0], [list(range(200))]), ([37], [list(range(37, 165))]),                            # a context; the rest of one
    ([300, 0, 64, 0, 129], [[5, 6, 70, 299], [], list(range(64)), list(range(70)), [0, 63, 64, 127, 128, 129]]),
    ([128], [list(range(64, 128))]),                                                      # every token of a page replaced
    ([128], [list(range(0, 128, 2))]),                                                    # every second
    ([130], [[-1, -1, 40, 129]]), ([130], [[40, 129, -1]]),                               # rows that go nowhere
])
def test_store_pages(dtype, hkv, d, lens, rows):
    L, pages, args, start, want = store_case(dtype, hkv, d, lens, rows, len(rows) * 7 + lens[0], extra=2)
    assert_same_pool(pool_to_host(pages), want)
    L.store_pages(*args, row_start=i32(start))                                            # again: the same
    torch.cuda.synchronize()
    assert_same_pool(pool_to_host(pages), want)
    L.close()


def test_store_pages_many_rows_and_elements_that_are_not_finite():
    g = gen(9)
    lens = [3000, 0, 700]
    rows = [sorted(g.choice(3000, 900, replace=False).tolist()), list(range(2111)), sorted(g.choice(900, 500, replace=False).tolist())]
    for dtype, spoil in (("bf16", False), ("f32", False), ("bf16", True), ("f32", True)):
        L, pages, _, _, want = store_case(dtype, 2, 128, lens, rows, 10, spoil=spoil, flags=IFKV_FLAG_VALIDATE)
        assert_same_pool(pool_to_host(pages), want)
        L.close()


def test_store_pages_one_row_a_sequence_strided_and_without_a_page():
    g = gen(11)
    hkv, d, n = 8, 128, 70
    lens = g.integers(0, 500, n)
    pool = random_pool(g, 700, hkv, d)
    table = make_table(g, [int(x) + 1 for x in lens], 700, width=9)
    pos = lens.copy()
    pos[3], pos[4] = -1, 9 * 64                       # a padded row; one behind the table
    table[5, :], table[6, :] = -1, 700                # sequences whose pages are none
    qkv64, qkv = stored(g.standard_normal((n, 32 + 16, d)), "bf16")
    L = layer("bf16", 32, hkv, d)
    pages = pool_to_device(pool)
    L.store_pages(pages, i32(table), i32(lens), qkv[:, 32:40], qkv[:, 40:], i32(pos))
    want = P.store_pages(pool, table, lens, pos, qkv64[:, 32:40], qkv64[:, 40:])
    assert_same_pool(pool_to_host(pages), want)
    L.close()


def test_store_pages_scale_rises_token_by_token_and_a_page_comes_back():
    """Tokens that grow by steps of two: the page's bytes are rounded again each time, down to subnormals; then its page is given to
    another sequence and forgets all of it."""
    hkv, d = 2, 64
    pool = random_pool(gen(12), 2, hkv, d)
    L = layer("f32", 4, hkv, d)
    pages, table = pool_to_device(pool), np.array([[1]])
    g = gen(13)
    for j in range(70):
        at = j % 64 if j < 64 else j - 64
        x64, x = stored(g.standard_normal((1, hkv, d)) * 2.0 ** (j // 2 if j < 64 else -3), "f32")
        pool = P.store_pages(pool, table, [at], [at], x64, x64 * 0.5)
        L.store_pages(pages, i32(table), i32([at]), x, x * 0.5, i32([at]))
        assert_same_pool(pool_to_host(pages), pool)
    L.close()


def test_store_pages_validate_names_the_row():
    L = layer("bf16", 8, 8, 64, flags=IFKV_FLAG_VALIDATE)
    pages = pool_to_device(random_pool(gen(1), 4, 8, 64))
    _, x = stored(np.zeros((4, 8, 64)), "bf16")
    with pytest.raises(IfkvError, match="index 3"):
        L.store_pages(pages, i32([[0, 1], [2, 3]]), i32([0, 0]), x, x, i32([4, 5, 9, 9]), row_start=i32([0, 2, 4]))
    L.store_pages(pages, i32([[0, 1], [2, 3]]), i32([0, 0]), x, x, i32([4, 5, 3, 9]), row_start=i32([0, 2, 4]))
    L.close()


# ---- pages onto pages -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,hkv,d,n,n_pages", [("bf16", 8, 128, 1, 2), ("f32", 3, 64, 5, 30), ("bf16", 1, 64, 1000, 2100), ("bf16", 5, 128, 449, 900)])
def test_copy_pages(dtype, hkv, d, n, n_pages):
    g = gen(n)
    pool = random_pool(g, n_pages, hkv, d)
    dst = g.permutation(n_pages)[:n]
    left = np.setdiff1d(np.arange(n_pages), dst)
    src = g.choice(left, n)                            # some pages go to many
    L = layer(dtype, hkv, hkv, d)
    pages = pool_to_device(pool)
    L.copy_pages(pages, src.tolist(), torch.tensor(dst, dtype=torch.int32))
    got, want = pool_to_host(pages), P.copy_pages(pool, src, dst)
    assert all(np.array_equal(got[name], want[name]) for name in want)
    L.close()


# ---- attention ----------------------------------------------------------------------------------------------------------
def attend_case(shape, lens, rows, seed, flags=0, lse=True, extra=0, width=None, spread=3, tweak=None, scale=1.0, sm_scale=0.0, max_rows=None,
                columns=None):
    dtype, hq, hkv, d = shape
    g = gen(seed)
    n_pages = sum(-(-n // 64) for n in lens) + 2
    pool = random_pool(g, n_pages, hkv, d, spread)
    table = make_table(g, lens, n_pages, width)
    start = np.concatenate([[0], np.cumsum([len(r) for r in rows])])
    pos = np.concatenate([np.asarray(r, dtype=np.int64) for r in rows] + [np.zeros(extra, dtype=np.int64)])
    q64, q = stored(scale * g.standard_normal((len(pos), hq, d)), dtype)
    if tweak is not None:
        q64, q = tweak(pool, table, pos, q64, q)
    L = layer(dtype, hq, hkv, d, flags=flags, sm_scale=sm_scale)
    out = torch.full((len(pos), hq, d), 7.0, dtype=q.dtype, device=DEV)
    most = max([len(r) for r in rows] + [1])
    got, got_lse = L.attend_pages(q, i32(pos), pool_to_device(pool), i32(table), row_start=i32(start), max_rows=max_rows or most,
                                  out=out, return_lse=True)
    torch.cuda.synchronize()
    ref = P.attend_pages(q64, pos, pool, table, sm_scale or d ** -0.5, row_start=start)
    parts = 3 if flags & IFKV_FLAG_FORCE_GENERIC else parts_of(dtype, most * hq // hkv)
    if extra:
        assert (out[-extra:] == 7.0).all()             # rows behind the last sequence are left as they were
    assert_attended(to_host_f64(got, dtype), got_lse.cpu().numpy().astype(np.float64), ref, dtype, max(lens + [1]), parts)
    L.close()
    return got, got_lse, ref


CASES = [
    ([1], [[0]]), ([64], [[63]]), ([65], [[64]]), ([300], [[299]]),
    ([1, 700, 64, 128, 65, 33], [[0], [699], [63], [127], [64], [32]]),
    ([500, 90, 200], [[495, 496, 497, 498, 499], [], [199]]),                             # proposed tokens of one sequence, none of another
    ([260], [list(range(200, 260))]),                                                     # the end of a prompt
    ([513, 40], [[0, 512, 7, 300, 64], [39, -1, 0]]),                                     # any rows, any order, rows that see nothing
]


@pytest.mark.parametrize("flags", [0, IFKV_FLAG_FORCE_GENERIC], ids=["", "generic"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attend_pages(shape, case, flags):
    lens, rows = CASES[case]
    attend_case(shape, lens, rows, 100 + case, flags=flags, extra=3 if case % 2 else 0, width=None if case % 3 else 40)


@pytest.mark.parametrize("shape", [("bf16", 32, 8, 128), ("f32", 8, 8, 64), ("bf16", 14, 2, 64)], ids=lambda s: "-".join(map(str, s)))
def test_attend_pages_long_and_uneven(shape):
    """Sequences that are cut along the cache beside ones that are not, logits of all sizes."""
    lens = [9001, 1, 63, 2500, 4096, 130]
    attend_case(shape, lens, [[n - 1] for n in lens], 31, scale=3.0)
    attend_case(shape, [20011], [[20010]], 32)


@pytest.mark.parametrize("shape", [("bf16", 32, 8, 128), ("bf16", 28, 4, 128), ("bf16", 16, 2, 64), ("f32", 12, 4, 128)], ids=lambda s: "-".join(map(str, s)))
def test_attend_pages_many_rows(shape):
    """Pieces of prompts: whole blocks of query columns, a diagonal through pages, uneven sequences, the rows of one in the middle."""
    attend_case(shape, [700, 10, 1500], [list(range(450, 700)), list(range(10)), list(range(3, 1500, 9))], 41, extra=1)


def test_attend_pages_of_one_row_a_sequence_without_row_start():
    g = gen(51)
    lens = [5, 900, 64, 1, 333]
    pool, hq = random_pool(g, 40, 2, 128), 8
    table = make_table(g, lens, 40)
    q64, qkv = stored(g.standard_normal((5, hq + 4, 128)), "bf16")
    pos = np.array(lens) - 1
    pos[2] = -1
    L = layer("bf16", hq, 2, 128)
    out, lse = L.attend_pages(qkv[:, :hq], i32(pos), pool_to_device(pool), i32(table), return_lse=True)
    ref = P.attend_pages(q64[:, :hq], pos, pool, table, 128 ** -0.5)
    assert_attended(to_host_f64(out, "bf16"), lse.cpu().numpy().astype(np.float64), ref, "bf16", 900, 2)
    assert (out[2] == 0).all() and torch.isneginf(lse[2]).all()
    L.close()


@pytest.mark.parametrize("flags", [0, IFKV_FLAG_FORCE_GENERIC], ids=["", "generic"])
@pytest.mark.parametrize("shape,rows", [(("bf16", 8, 2, 128), 1), (("bf16", 8, 2, 128), 40), (("f32", 4, 4, 64), 3)], ids=str)
def test_attend_pages_missing_pages(shape, rows, flags):
    """Pages that the table does not name are not seen; a sequence without any gives zeros."""
    lens = [640, 200, 64 * 12]
    def tweak(pool, table, pos, q64, q):
        table[0, 2], table[0, 9], table[1, :], table[2, :11] = -1, 1 << 30, -5, pool["k"].shape[0]
        return q64, q
    got, lse, _ = attend_case(shape, lens, [list(range(n - rows, n)) for n in lens], 61, flags=flags, tweak=tweak)
    assert (got[rows:2 * rows] == 0).all() and torch.isneginf(lse[rows:2 * rows]).all()


@pytest.mark.parametrize("flags", [0, IFKV_FLAG_FORCE_GENERIC], ids=["", "generic"])
@pytest.mark.parametrize("shape,rows", [(("bf16", 8, 2, 128), 1), (("bf16", 8, 2, 128), 4), (("bf16", 8, 2, 128), 40), (("bf16", 8, 1, 64), 33),
                                        (("f32", 4, 4, 64), 3)], ids=str)
def test_attend_pages_nan_behind_a_row_does_not_show(shape, rows, flags):
    """The last page of a sequence holds NaN behind the last row, and behind the rows before it: each row sees its own tokens only.
    NaN that a row does see makes it NaN: a key all of it, a value its column."""
    n = 130 + rows
    def tweak(pool, table, pos, q64, q):
        for j in range(n, 192 + (n > 192) * 64):
            page = table[0, j // 64]
            pool["k"][page, :, j % 64], pool["v"][page, :, :, P.value_byte(j % 64)] = 0x7F, 0xFF
        return q64, q
    attend_case(shape, [n], [list(range(n - rows, n))], 71, flags=flags, tweak=tweak)

    dtype, hq, hkv, d = shape
    g = gen(72)
    pool = random_pool(g, 5, hkv, d)
    table = make_table(g, [n], 5)
    bad = n - 1 - rows // 2                             # the rows from this token on see it
    page, byte = table[0, bad // 64], P.value_byte(bad % 64)
    pos = np.arange(n - rows, n)
    _, q = stored(g.standard_normal((rows, hq, d)), dtype)
    L = layer(dtype, hq, hkv, d, flags=flags)
    args = dict(row_start=i32([0, rows]), max_rows=rows)
    clean = L.attend_pages(q, i32(pos), pool_to_device(pool), i32(table), **args)
    sees = torch.tensor(pos >= bad, device=DEV)
    with_v = dict(pool, v=pool["v"].copy())
    with_v["v"][page, 0, 9, byte] = 0x7F
    got = L.attend_pages(q, i32(pos), pool_to_device(with_v), i32(table), **args)
    grp = hq // hkv
    assert torch.isnan(got[sees][:, :grp, 9]).all()
    hurt = torch.zeros_like(got, dtype=torch.bool)
    hurt[:, :grp, 9] = sees[:, None]
    assert torch.equal(got[~hurt], clean[~hurt])
    with_k = dict(pool, k=pool["k"].copy())
    with_k["k"][page, 0, bad % 64, 3] = 0x7F
    got = L.attend_pages(q, i32(pos), pool_to_device(with_k), i32(table), **args)
    assert torch.isnan(got[sees][:, :grp]).all()
    assert torch.equal(got[~sees], clean[~sees]) and torch.equal(got[:, grp:], clean[:, grp:])
    L.close()


@pytest.mark.parametrize("flags", [0, IFKV_FLAG_FORCE_GENERIC], ids=["", "generic"])
def test_attend_pages_queries_that_are_not_finite(flags):
    """A logit of +infinity or NaN makes its row NaN, and no other."""
    g = gen(75)
    pool = random_pool(g, 6, 2, 128)
    table = make_table(g, [300], 6)
    for rows in (2, 40):
        _, q = stored(g.standard_normal((rows, 8, 128)), "bf16")
        L = layer("bf16", 8, 2, 128, flags=flags)
        pos = i32(np.arange(300 - rows, 300))
        args = (pos, pool_to_device(pool), i32(table), i32([0, rows]), rows)
        clean = L.attend_pages(q, *args)
        spoiled = q.clone()
        spoiled[0, 1, 5], spoiled[1, 6, 0] = float("inf"), float("nan")
        got = L.attend_pages(spoiled, *args)
        assert torch.isnan(got[0, 1]).all() and torch.isnan(got[1, 6]).all()
        ok = torch.ones(rows, 8, dtype=torch.bool)
        ok[0, 1], ok[1, 6] = False, False
        assert torch.equal(got[ok], clean[ok])
        L.close()


@pytest.mark.parametrize("rows", [1, 40])
def test_attend_pages_scales_far_apart(rows):
    """Pages whose scales lie 2^60 apart, a large one that no row attends to among them, and logits of hundreds."""
    def tweak(pool, table, pos, q64, q):
        pool["v_scale"][table[0, 0]] = 2.0 ** 40
        pool["v_scale"][table[0, 2]] = 2.0 ** -20
        pool["k_scale"][table[0, 1]] = 2.0 ** -3
        return q64, q
    n = 64 * 5 + 3
    attend_case(("bf16", 8, 2, 128), [n], [list(range(n - rows, n))], 81, tweak=tweak, spread=0)
    attend_case(("f32", 4, 2, 64), [n], [list(range(n - min(rows, 3), n))], 82, tweak=tweak, spread=0)


def test_attend_pages_max_rows_bounds_what_is_computed():
    g = gen(85)
    pool, table = random_pool(g, 6, 2, 128), np.array([[0, 1, 2], [3, 4, 5]])
    q64, q = stored(g.standard_normal((9, 8, 128)), "bf16")
    pos, start = np.array([150, 151, 152, 153, 154, 155, 100, 101, 102]), [0, 6, 9]
    L = layer("bf16", 8, 2, 128)
    full = L.attend_pages(q, i32(pos), pool_to_device(pool), i32(table), row_start=i32(start))
    out = torch.full_like(full, 3.0)
    L.attend_pages(q, i32(pos), pool_to_device(pool), i32(table), row_start=i32(start), max_rows=6, out=out)
    ref = P.attend_pages(q64, pos, pool, table, 128 ** -0.5, row_start=start)
    for o, rows in ((full, 9), (out, 6)):            # 36 columns: a weight is one bf16 number, 2^-8 of the mass; 24: two, 2^-16
        assert_attended(to_host_f64(o, "bf16"), None, ref, "bf16", 192, parts_of("bf16", rows * 4))
    L.close()


def test_attend_pages_same_results_every_time():
    """No atomics on results: the same call gives the same bits."""
    g = gen(87)
    lens = [3001, 70, 9000]
    pool, hkv = random_pool(g, 200, 8, 128), 8
    table = make_table(g, lens, 200)
    _, q = stored(g.standard_normal((3, 32, 128)), "bf16")
    L = layer("bf16", 32, hkv, 128)
    pages, t, pos = pool_to_device(pool), i32(table), i32(np.array(lens) - 1)
    first = L.attend_pages(q, pos, pages, t).clone()
    for _ in range(20):
        assert torch.equal(L.attend_pages(q, pos, pages, t), first)
    L.close()


# ---- together --------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", [("bf16", 28, 4, 128), ("f32", 8, 8, 64)], ids=lambda s: "-".join(map(str, s)))
def test_decoding_with_a_fork_eager_and_replayed(shape):
    """A context goes into pages; two answers to it are decoded step by step, the second forked from the first in the middle of a page; the
    step is captured once and replayed, lengths and rows living in device memory.  Every step against the oracle."""
    dtype, hq, hkv, d = shape
    g = gen(91)
    n0, steps, n_pages = 130, 5, 12
    L = layer(dtype, hq, hkv, d, max_ctx=1024)
    axes = torch.tensor([j % 3 for j in range(d // 2)], dtype=torch.int32)
    freq = THETA ** (-2.0 * np.arange(d // 2) / d)
    pool = {n: np.zeros_like(a) for n, a in random_pool(g, n_pages, hkv, d).items()}
    pages = pool_to_device(pool)
    # the context, its keys turned on three axes
    k64, k = stored(g.standard_normal((n0, hkv, d)), dtype)
    v64, v = stored(g.standard_normal((n0, hkv, d)), dtype)
    where = np.stack([np.arange(n0), np.arange(n0) // 8, np.arange(n0) % 8], 1)
    L.rope_rows_axes(k, i32(where), axes)
    kr = to_host_f64(k, dtype)
    want_k = P.rope_rows_axes(k64, where, axes.tolist(), freq)
    tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * np.abs(want_k) + 2.0 ** -20 * 8
    assert (np.abs(kr - want_k) <= tol).all()
    table = np.array([[7, 2, 9, 4], [7, 2, 5, 6]])
    L.store_pages(pages, i32(table[:1]), i32([0]), k, v, i32(np.arange(n0)), row_start=i32([0, n0]))
    pool = P.store_pages(pool, table[:1], [0], np.arange(n0), kr, v64, row_start=[0, n0])
    L.copy_pages(pages, [9], [5])                       # the fork: full pages shared, the last one copied
    pool = P.copy_pages(pool, [9], [5])
    assert_same_pool(pool_to_host(pages), pool)

    t = i32(table)
    qkv = torch.empty(2, hq + 2 * hkv, d, dtype=k.dtype, device=DEV)
    pos3, kv_len, row_pos = i32(np.zeros((2, 3))), i32([0, 0]), i32([0, 0])
    out = torch.empty(2, hq, d, dtype=k.dtype, device=DEV)

    def step():
        L.rope_rows_axes(qkv[:, : hq + hkv], pos3, axes)
        L.store_pages(pages, t, kv_len, qkv[:, hq: hq + hkv], qkv[:, hq + hkv:], row_pos)
        L.attend_pages(qkv[:, :hq], row_pos, pages, t, out=out)

    graph = None
    for i in range(steps):
        x64, x = stored(g.standard_normal((2, hq + 2 * hkv, d)), dtype)
        at = n0 + i
        qkv.copy_(x)
        pos3.copy_(i32([[at, 17, 3], [at, 18 + i, 4]]))
        kv_len.fill_(at)
        row_pos.fill_(at)
        torch.cuda.synchronize()
        if i == 0:
            step()
        elif i == 1:
            s = torch.cuda.Stream()
            # a context belongs to a stream: a second one for the captured step, warmed up on an idle pool first
            L2 = layer(dtype, hq, hkv, d, max_ctx=1024, stream=s.cuda_stream)
            with torch.cuda.stream(s):
                spare = pool_to_device(pool)
                L2.rope_rows_axes(qkv.clone()[:, : hq + hkv], pos3, axes)
                L2.attend_pages(qkv[:, :hq], row_pos, spare, t, out=out)
                s.synchronize()
                eager, L = L, L2
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=s):
                    step()
            torch.cuda.synchronize()
            graph.replay()
        else:
            graph.replay()
        torch.cuda.synchronize()
        rot = to_host_f64(qkv, dtype)
        pool = P.store_pages(pool, table, [at, at], [at, at], rot[:, hq: hq + hkv], rot[:, hq + hkv:])
        assert_same_pool(pool_to_host(pages), pool)
        ref = P.attend_pages(rot[:, :hq], np.array([at, at]), pool, table, d ** -0.5)
        assert_attended(to_host_f64(out, dtype), None, ref, dtype, at + 1, parts_of(dtype, hq // hkv))
        assert np.array_equal(rot[:, hq + hkv:], x64[:, hq + hkv:])
    L.close()
    eager.close()
