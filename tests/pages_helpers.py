"""Plumbing of the tests on 8-bit pages: pools on both sides, page tables, error bounds."""
import numpy as np
import torch

from oracle import pages_oracle as P
from tests.helpers import DEV
from workloads import to_f64, to_storage

F8 = torch.float8_e4m3fn


def gen(seed):
    return np.random.Generator(np.random.Philox(key=[seed, 83]))


def stored(x, dtype):
    """float64 -> (what the storage type holds, as float64; its device tensor)."""
    bits = to_storage(np.asarray(x, dtype=np.float64), dtype)
    if dtype == "bf16":
        return to_f64(bits, dtype), torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16).to(DEV)
    return bits.astype(np.float64), torch.from_numpy(np.ascontiguousarray(bits)).to(DEV)


def random_pool(g, n_pages, heads, d, spread=3):
    """Bytes of Gaussian numbers, scales that differ from page to page and head to head by up to 2^spread."""
    def one(a, b):
        x = np.clip(g.standard_normal((n_pages, heads, a, b)) * 100.0, -448, 448)
        return P.to_e4m3(x), 2.0 ** (-7 + g.integers(0, spread + 1, (n_pages, heads)))
    k, ks = one(P.PAGE, d)
    v, vs = one(d, P.PAGE)
    return dict(k=k, v=v, k_scale=ks, v_scale=vs)


def pool_to_device(pool):
    from paper_2603_05353_amd import PageCache
    return PageCache(*(torch.from_numpy(pool[n].copy()).view(F8).to(DEV) for n in ("k", "v")),
                     *(torch.from_numpy(pool[n].astype(np.float32)).to(DEV) for n in ("k_scale", "v_scale")))


def pool_to_host(pages):
    return dict(k=pages.k.view(torch.uint8).cpu().numpy(), v=pages.v.view(torch.uint8).cpu().numpy(),
                k_scale=pages.k_scale.cpu().numpy().astype(np.float64), v_scale=pages.v_scale.cpu().numpy().astype(np.float64))


def same_numbers(a, b):
    """Bytes that stand for the same numbers (all NaN are one; zeros of either sign too)."""
    x, y = P.E4M3[a], P.E4M3[b]
    return np.array_equal(x, y, equal_nan=True)


def assert_same_pool(got, want):
    for n in ("k_scale", "v_scale"):
        assert np.array_equal(got[n], want[n]), n
    for n in ("k", "v"):
        assert same_numbers(got[n], want[n]), n


def make_table(g, lens, n_pages, width=None):
    """Pages of sequences with so many tokens, all over the pool; -1 behind the last."""
    need = [-(-n // P.PAGE) for n in lens]
    width = width or max(need + [1])
    free = list(g.permutation(n_pages))
    table = np.full((len(lens), width), -1, dtype=np.int32)
    for s, n in enumerate(need):
        for i in range(n):
            table[s, i] = free.pop()
    return table


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def attend_bounds(ref, mass, size, n, d, dtype, parts):
    """What |out - ref| and |lse - lse_ref| cannot exceed, element by element.

    A logit is a sum of d exact products in fp32 (d + 1 roundings of at most 2^-24 of sum |q k| each), scaled, moved by the maximum and
    brought to base 2: three more on numbers of at most 2 * size.  So weights move by the factor exp(e), e <= 2^-24 (d + 8) size,
    and the exponential itself by 2^-22; both enter twice, over numerator and sum.  Sums over n tokens are chains of n / 16 matrix
    instructions and joins, 2^-24 each.  Weights are then held in `parts` bf16 numbers (2^-8, 2^-16, 2^-24), and the result is
    rounded once."""
    e = 2.0 ** -24 * (d + 8) * size
    chain = 2.0 ** -24 * (n / 16 + 96)
    w = 2 * np.expm1(e) + 2.0 ** -21 + 2 * chain + 2.0 ** -(8 * parts)
    rounding = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    return w[..., None] * mass * (1 + rounding) + rounding * np.abs(ref) + 1e-37, e + 2.0 ** -21 + chain + 2.0 ** -22 * (1 + size)


def assert_attended(out, lse, ref, dtype, n, parts):
    """out, lse: float64 from the device; ref: what the oracle returned for all rows of the tensors (NaN: not to be looked at)."""
    want, want_lse, mass, size = ref
    rows = ~np.isnan(size[:, 0])
    bound, bound_lse = attend_bounds(want, mass, size, n, want.shape[-1], dtype, parts)
    err = np.abs(out - want)[rows]
    worst = (err - bound[rows]).max() if err.size else 0.0
    assert worst <= 0, f"output off by {err.max()}, {worst} beyond the bound"
    if lse is not None:
        empty = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(lse)[rows], empty[rows])
        ok = rows[:, None] & ~empty
        off = np.abs(lse[ok] - want_lse[ok])
        assert (off <= bound_lse[ok]).all(), off.max()
