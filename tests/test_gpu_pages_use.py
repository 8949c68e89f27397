"""Calls on 8-bit pages as programs make them: rows of uneven batches, every number of query columns, calls that are repeated, several contexts at
once, and both ways of the binding."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as P
from paper_2603_05353_amd import IFKV_FLAG_FORCE_GENERIC, IFKV_FLAG_VALIDATE, IfkvError
from tests.helpers import DEV, to_host_f64
from tests.pages_helpers import assert_attended, assert_same_pool, gen, i32, make_table, pool_to_device, pool_to_host, random_pool, stored
from tests.test_gpu_marshalling import Served
from tests.test_gpu_pages import attend_case, layer

pytestmark = pytest.mark.gpu


# ---- rows into pages ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,hkv,d", [("bf16", 8, 128), ("f32", 2, 64)])
def test_store_pages_uneven_batch(dtype, hkv, d):
    """A prompt among single tokens, sequences without rows, rows before the first sequence and behind the last, long runs of rows that name
    no token: a workgroup finds the first rows of pages among many."""
    g = gen(101)
    held = g.integers(0, 200, 90)
    rows = [[int(n)] for n in held]
    for s in (0, 7, 8, 40, 89):
        rows[s] = []
    rows[20] = list(range(int(held[20]), int(held[20]) + 700))            # a prompt
    rows[21] = [-1] * 130 + list(range(int(held[21]), int(held[21]) + 9))  # padded in front, farther than a wavefront looks
    rows[60] = list(range(5, 150)) + [-1] * 70                             # and behind
    rows[61] = sorted(g.choice(400, 60, replace=False).tolist())
    tops = [max([int(n)] + [p + 1 for p in ps]) for n, ps in zip(held, rows)]
    n_pages = sum(-(-n // 64) for n in tops) + 2
    pool = random_pool(g, n_pages, hkv, d)
    table = make_table(g, tops, n_pages)
    start = 5 + np.concatenate([[0], np.cumsum([len(r) for r in rows])])
    pos = np.concatenate([np.arange(5)] + [np.asarray(r, dtype=np.int64) for r in rows] + [np.arange(70)]).astype(np.int64)
    k64, k = stored(g.standard_normal((len(pos), hkv, d)) * 3, dtype)
    v64, v = stored(g.standard_normal((len(pos), hkv, d)), dtype)
    L = layer(dtype, hkv, hkv, d, flags=IFKV_FLAG_VALIDATE)
    pages = pool_to_device(pool)
    L.store_pages(pages, i32(table), i32(held), k, v, i32(pos), row_start=i32(start))
    want = P.store_pages(pool, table, held, pos, k64, v64, row_start=start)
    assert_same_pool(pool_to_host(pages), want)
    L.close()


@pytest.mark.parametrize("n", [1500, 5000])
def test_store_pages_one_sequence_of_scattered_rows(n):
    g = gen(n)
    hkv, d, top = 8, 64, 3 * n
    pos = np.sort(g.choice(top, n, replace=False))
    n_pages = -(-top // 64) + 1
    pool, table = random_pool(g, n_pages, hkv, d), make_table(g, [top], n_pages)
    k64, k = stored(g.standard_normal((n, hkv, d)), "bf16")
    L = layer("bf16", hkv, hkv, d)
    pages = pool_to_device(pool)
    L.store_pages(pages, i32(table), i32([top]), k, k, i32(pos), row_start=i32([0, n]))
    assert_same_pool(pool_to_host(pages), P.store_pages(pool, table, [top], pos, k64, k64, row_start=[0, n]))
    L.close()


def test_store_pages_validate_sees_rows_behind_an_end():
    L = layer("bf16", 8, 8, 64, flags=IFKV_FLAG_VALIDATE)
    pages = pool_to_device(random_pool(gen(1), 4, 8, 64))
    _, x = stored(np.zeros((6, 8, 64)), "bf16")
    args = pages, i32([[0, 1], [2, 3]]), i32([0, 0]), x, x
    with pytest.raises(IfkvError, match="index 4"):
        L.store_pages(*args, i32([4, 5, -1, -1, 9, 10]), row_start=i32([0, 5, 6]))
    L.store_pages(*args, i32([-1, 4, 5, -1, -1, 10]), row_start=i32([0, 5, 6]))
    L.close()


# ---- attention ----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", [("bf16", 8, 8, 128), ("bf16", 4, 4, 64), ("f32", 4, 4, 128)], ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("rows", [15, 16, 17, 32, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129])
def test_attend_pages_numbers_of_columns(shape, rows):
    """As many rows as a kernel takes and one more, one of them in the sequence's middle; cut along the cache, and whole."""
    for lens in ([1500, 130], [300, 130]):
        first = lens[0] - rows
        attend_case(shape, lens, [[5] + list(range(first + 1, lens[0])), [129]], 200 + rows)


@pytest.mark.parametrize("shape", [("bf16", 12, 1, 128), ("bf16", 20, 2, 64)], ids=lambda s: "-".join(map(str, s)))
def test_attend_pages_columns_that_split_a_row(shape):
    """Groups of query heads that do not divide a tile: a row's heads lie in two tiles, or in two blocks of columns."""
    attend_case(shape, [2000, 70], [list(range(1985, 2000)), [69, 3]], 231)
    attend_case(shape, [700], [list(range(650, 700))], 232)


@pytest.mark.parametrize("width,longest", [(22, 1400), (70, 130)])
def test_attend_pages_more_sequences_than_a_plan_holds(width, longest):
    g = gen(width)
    lens = [int(x) for x in g.integers(1, 100, 1100)]
    lens[3], lens[700], lens[1099] = longest, longest - 64, longest
    attend_case(("bf16", 2, 1, 64), lens, [[n - 1] for n in lens], 240 + width, width=width)


@pytest.mark.parametrize("flags", [0, IFKV_FLAG_FORCE_GENERIC], ids=["", "generic"])
def test_attend_pages_without_any_page(flags):
    L = layer("bf16", 8, 2, 64, flags=flags)
    _, q = stored(np.ones((3, 8, 64)), "bf16")
    some, none = pool_to_device(random_pool(gen(2), 2, 2, 64)), L.empty_pages(0)
    for pages, table in ((some, i32(np.zeros((3, 0)))), (none, i32(np.zeros((3, 4)))), (some, i32(np.full((3, 30), 2)))):
        L.store_pages(pages, table, i32([0, 0, 0]), q[:, :2], q[:, :2], i32([0, 1, 2]))
        for kw in ({}, dict(row_start=i32([0, 0, 3, 3]), max_rows=3)):
            out, lse = L.attend_pages(q, i32([0, 1, 2]), pages, table, return_lse=True, out=torch.full_like(q, 5.0), **kw)
            assert (out == 0).all() and torch.isneginf(lse).all()
    L.close()


def test_attend_pages_contexts_at_the_same_time():
    """Two streams, a context each, the pool shared: as one after the other."""
    g = gen(250)
    lens = [9000, 4000, 70]
    pool = random_pool(g, 220, 8, 128)
    pages, table, pos = pool_to_device(pool), i32(make_table(g, lens, 220)), i32(np.array(lens) - 1)
    qs = [stored(g.standard_normal((3, 32, 128)), "bf16")[1] for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in qs]
    layers = [layer("bf16", 32, 8, 128, stream=s.cuda_stream) for s in streams]
    want = [L.attend_pages(q, pos, pages, table) for L, q in zip(layers, qs)]
    torch.cuda.synchronize()
    outs = [[torch.empty_like(q) for _ in range(10)] for q in qs]
    torch.cuda.synchronize()
    for i in range(10):
        for L, q, out in zip(layers, qs, outs):
            L.attend_pages(q, pos, pages, table, out=out[i])
    torch.cuda.synchronize()
    for w, out in zip(want, outs):
        assert all(torch.equal(o, w) for o in out)
    for L in layers:
        L.close()


# ---- both ways of the binding, repeated calls ---------------------------------------------------------------------------------
def a_step(L, seed, out=None):
    """Every call on pages; all that they write."""
    g = gen(seed)
    hq, hkv, d, dtype = L.n_q_heads, L.n_kv_heads, L.head_dim, L.dtype
    held = [130, 64, 5]
    pool = random_pool(g, 20, hkv, d)
    pages, table = pool_to_device(pool), i32(make_table(g, [n + 8 for n in held], 18))
    _, qkv = stored(g.standard_normal((6, hq + 2 * hkv, d)), dtype)
    start, pos = i32([0, 3, 4, 6]), i32([130, 131, 132, 64, 5, 6])
    axes = torch.arange(d // 2, dtype=torch.int32) % 3
    L.rope_rows_axes(qkv[:, : hq + hkv], pos[:, None].repeat(1, 3).contiguous(), axes)
    L.store_pages(pages, table, i32(held), qkv[:, hq: hq + hkv], qkv[:, hq + hkv:], pos, row_start=start)
    free = [p for p in range(20) if p not in set(table.flatten().tolist())][:2]
    L.copy_pages(pages, torch.tensor([int(table[0, 0])] * 2, dtype=torch.int32), torch.tensor(free, dtype=torch.int32))
    o, lse = L.attend_pages(qkv[:, :hq], pos, pages, table, row_start=start, max_rows=3, return_lse=True)
    return [qkv, *(t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in pages), o, lse]


@pytest.mark.parametrize("shape", [("bf16", 16, 4, 128), ("f32", 6, 2, 64)], ids=lambda s: "-".join(map(str, s)))
def test_native_and_ctypes_calls_agree_on_pages(shape):
    native, plain = layer(*shape), layer(*shape)
    plain._native = None
    native._native = served = Served(native._native)
    a, b = a_step(native, 260), a_step(plain, 260)
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    assert [name for name, _ in served.returned] == ["rope_rows_axes", "store_pages", "copy_pages", "attend_pages"]
    assert all(r == 0 for _, r in served.returned)
    native.close(), plain.close()


def test_native_calls_leave_what_they_do_not_take_to_the_checks():
    """Tensors that a call must not read: refused with a name by a layer that has both ways."""
    L = layer("bf16", 8, 2, 64)
    pages, table, pos = pool_to_device(random_pool(gen(3), 4, 2, 64)), i32([[0, 1], [2, 3]]), i32([3, 3])
    _, q = stored(np.ones((2, 8, 64)), "bf16")
    bad = [("q", lambda: L.attend_pages(q.float(), pos, pages, table)), ("q", lambda: L.attend_pages(q[:, :, ::2], pos, pages, table)),
           ("q", lambda: L.attend_pages(q[:, ::2], pos, pages, table)), ("row_pos", lambda: L.attend_pages(q, pos[:1], pages, table)),
           ("row_pos", lambda: L.attend_pages(q, pos.long(), pages, table)), ("table", lambda: L.attend_pages(q, pos, pages, table.t())),
           ("row_start", lambda: L.attend_pages(q, pos, pages, table, row_start=i32([0, 2]))),
           ("out", lambda: L.attend_pages(q, pos, pages, table, out=torch.empty(2, 16, 64, dtype=q.dtype, device=DEV)[:, ::2])),
           ("pages.v", lambda: L.attend_pages(q, pos, pages._replace(v=pages.v[:3]), table)),
           ("pages.k_scale", lambda: L.attend_pages(q, pos, pages._replace(k_scale=pages.k_scale.double()), table)),
           ("pages.k", lambda: L.store_pages(pages._replace(k=pages.k.view(torch.uint8)), table, pos, q[:, :2], q[:, 2:4], pos)),
           ("v_new", lambda: L.store_pages(pages, table, pos, q[:, :2], q[:1, 2:4], pos)),
           ("k_new", lambda: L.store_pages(pages, table, pos, q[:, :3], q[:, :2], pos)),
           ("kv_len", lambda: L.store_pages(pages, table, pos[:1], q[:, :2], q[:, 2:4], pos)),
           ("x", lambda: L.rope_rows_axes(q.half(), pos[:, None].contiguous(), torch.zeros(32, dtype=torch.int32))),
           ("src", lambda: L.copy_pages(pages, i32([0]), i32([1])))]
    for name, call in bad:
        with pytest.raises(ValueError, match=f"^{name}:"):
            call()
    L.close()


def test_bound_calls_on_pages_repeat():
    """bind() of each call, repeated eagerly and captured: lengths, rows and queries live in device memory."""
    g = gen(270)
    s = torch.cuda.Stream()
    L = layer("bf16", 8, 2, 128, stream=s.cuda_stream)
    held, n_pages = np.array([2000, 70]), 48
    pool = random_pool(g, n_pages, 2, 128)
    host_table = make_table(g, [2050, 120], n_pages - 4)
    pages, table = pool_to_device(pool), i32(host_table)
    spare = [p for p in range(n_pages) if p not in set(host_table.flatten().tolist())][0]
    kv_len, pos = i32(held), i32(held)
    qkv = torch.empty(2, 12, 128, dtype=torch.bfloat16, device=DEV)
    out = torch.empty(2, 8, 128, dtype=torch.bfloat16, device=DEV)
    axes = torch.zeros(64, dtype=torch.int32)
    turn = i32(np.zeros((2, 1)))
    qkv.zero_()
    scratch = pool_to_device(pool)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        first = (L.bind("rope_rows_axes", qkv[:, :10], turn, axes), L.bind("store_pages", scratch, table, kv_len, qkv[:, 8:10], qkv[:, 10:], pos),
                 L.bind("attend_pages", qkv[:, :8], pos, scratch, table, out=out), L.bind("copy_pages", scratch, [int(host_table[0, 0])], [spare]))
        s.synchronize()
        for n in ("k", "v", "k_scale", "v_scale"):
            getattr(scratch, n).copy_(getattr(pages, n))
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            for call in first:
                call()
        want = pool
        for i in range(5):
            at = held + i
            x64, x = stored(g.standard_normal((2, 12, 128)), "bf16")
            qkv.copy_(x), kv_len.copy_(i32(at)), pos.copy_(i32(at)), turn.copy_(i32(at[:, None]))
            torch.cuda.synchronize()
            if i % 2:
                graph.replay()
            else:
                for call in first:
                    call()
            torch.cuda.synchronize()
            rot = to_host_f64(qkv, "bf16")
            want = P.store_pages(want, host_table, at, at, rot[:, 8:10], rot[:, 10:])
            ref = P.attend_pages(rot[:, :8], at, want, host_table, 128 ** -0.5)
            want = P.copy_pages(want, [int(host_table[0, 0])], [spare])
            assert_same_pool(pool_to_host(scratch), want)
            assert_attended(to_host_f64(out, "bf16"), None, ref, "bf16", int(at.max()) + 1, 2)
    L.close()
