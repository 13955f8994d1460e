"""Pins of the oracles of pages, rotations and latent attention: closed forms, invariants, the expanded form."""
import numpy as np
import pytest

from oracle import latent_attn as LA
from oracle import pages as PG
from oracle import rope_append as RA


def test_extend_hands_out_pages_in_order():
    table = [[7, -1, -1], [-1, -1, -1]]
    t, slots, pos, cu, lens, n = PG.extend(table, 4, [3, 0], [3, 5], [9, 8, 5, 6], 4, 10)
    assert t == [[7, 6, -1], [5, 8, -1]] and n == 1 and lens == [6, 5] and cu == [0, 3, 8]
    assert slots == [31, 24, 25, 20, 21, 22, 23, 32, -1, -1] and pos == [3, 4, 5, 0, 1, 2, 3, 4, 0, 0]


@pytest.mark.parametrize("n_free,max_tokens,admitted", [(3, 99, [4, 4]), (2, 8, [4, 4]), (1, 99, [4, 0]),
                                                        (0, 99, [0, 0]), (9, 7, [4, 0]), (9, 3, [0, 0])])
def test_extend_refuses_from_the_first_that_does_not_fit(n_free, max_tokens, admitted):
    _, slots, _, cu, lens, n = PG.extend([[-1] * 4, [-1] * 4], 4, [0, 0], [4, 4], list(range(9)), n_free, max_tokens)
    assert cu == [0, 4, 8] and lens == admitted and n == n_free - sum(admitted) // 4
    assert sum(s >= 0 for s in slots) == sum(admitted)


def test_release_undoes_extend():
    rng = np.random.default_rng(3)
    ps, table = 4, [[i * 8 + c if c < 2 else -1 for c in range(8)] for i in range(4)]
    lens, new, free = [5, 8, 7, 6], [9, 1, 0, 20], [int(x) for x in rng.permutation(40) + 100]
    t, _, _, _, grown, n = PG.extend(table, ps, lens, new, free, len(free), 64)
    back, kept, m = PG.release(t, ps, grown, lens, [-1] * 40, 0)
    assert kept == lens and n + m == len(free) and sorted(back[:m]) == sorted(free[n:])


def test_rotation_is_a_rotation():
    rng = np.random.default_rng(0)
    x, f = rng.standard_normal((3, 2, 10)), np.array([1.0, 0.25, 0.01])
    pos = np.array([[0, 5, 1000], [4, 4, 4]])
    for inter in (False, True):
        y = RA.rotate(x, pos, f, None, inter)
        assert np.allclose(y[0], x[0]) and np.allclose(y[..., 6:], x[..., 6:])
        assert np.allclose((y**2).sum(-1), (x**2).sum(-1))
        # scores depend on differences of positions only
        z = RA.rotate(x, pos + 7, f, None, inter)
        assert np.allclose((y[1, 0, :6] * y[2, 1, :6]).sum(), (z[1, 0, :6] * z[2, 1, :6]).sum())
    y = RA.rotate(x, pos, f, [1, 1, 1])
    assert np.allclose(y, RA.rotate(x, pos[1:], f))


def test_norm():
    x = np.array([[3.0, 4.0]])
    assert np.allclose(RA.rms(x, np.array([1.0, 2.0]), 0.0), [[3 / np.sqrt(12.5), 8 / np.sqrt(12.5)]])
    assert RA.rms(x, None, 0.0) is not None and np.allclose(RA.rms(x, None, 0.0), x)


def test_absorbed_is_expanded():
    rng = np.random.default_rng(1)
    Hq, Dn, Dr, Dc, Dv, n, k = 3, 6, 4, 16, 5, 11, 2
    w_k, w_v = rng.standard_normal((Hq, Dn, Dc)), rng.standard_normal((Hq, Dv, Dc))
    rows = rng.standard_normal((1, n, Dc + Dr))
    qn, qr = rng.standard_normal((k + 1, Hq, Dn)), rng.standard_normal((k + 1, Hq, Dr))
    q = np.concatenate([np.einsum("ihd,hdc->ihc", qn, w_k), qr], -1)[None]
    out, _, _ = LA.verify(q, rows, [n], k, 0.3, Dc)
    for i in range(k + 1):
        want = LA.expanded(qn[i], qr[i], rows[0], n - k + i, w_k, w_v, 0.3)
        assert np.allclose(np.einsum("hc,hvc->hv", out[0, i], w_v), want)


def test_empty_rows_and_paging():
    rng = np.random.default_rng(2)
    cache, q = rng.standard_normal((6, 4, 12)), rng.standard_normal((2, 3, 2, 12))
    table = np.array([[5, 0, 3], [2, -1, 99]])
    out, lse, _ = LA.verify(q, cache, [10, 2], 2, 0.5, 8, table)
    flat = np.concatenate([cache[5], cache[0], cache[3]])[None]
    o2, l2, _ = LA.verify(q[:1], flat, [10], 2, 0.5, 8)
    assert np.allclose(out[0], o2[0]) and np.allclose(lse[0], l2[0])
    assert np.all(out[1, 0] == 0) and np.all(np.isneginf(lse[1, 0])) and np.all(np.isfinite(lse[1, 1:]))
