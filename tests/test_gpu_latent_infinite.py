"""Infinite latents: the same element is part of a key and a value.  A key whose score is -inf weighs zero, and 0 * inf
makes its dimension NaN in the rows that see it, however the sequence is shared out; a row whose visible scores are all
-inf is an empty row of zeros."""
import numpy as np
import pytest
import torch

from tests.test_gpu_latent_attn import Inp

pytestmark = pytest.mark.gpu


def inputs(lens, kv, Hq, k, Dc, ps):
    inp = Inp(lens, Hq, k, Dc=Dc, kv=kv, ps=ps, seed=41)
    inp.q[..., 0] = 1
    return inp


def rows(inp, b, keys):
    for j in keys:
        yield inp.cache[int(inp.table[b, j // inp.ps]), j % inp.ps] if inp.ps else inp.cache[b, j]


def compare(inp, kernel, want=None):
    out, lse = (x.double().cpu().numpy() for x in inp.run("f32", kernel))
    o, l, size = want or inp.oracle()
    assert np.array_equal(np.isnan(out), np.isnan(o)) and np.array_equal(np.isneginf(lse), np.isneginf(l))
    fine = np.isfinite(o)
    c = 2.0**-15 + (2.0**-8 if kernel == 0 and inp.kv == "bf16" else 0)
    assert np.all(np.abs(out - o)[fine] <= (c * size + 2.0**-24)[fine])
    f = np.isfinite(l)
    assert np.all(np.abs(lse[f] - l[f]) <= 2.0**-15 + 2.0**-22 * np.abs(l[f]))
    return o, l


FORMS = pytest.mark.parametrize("kv,kernel", [("bf16", 0), ("bf16", 1), ("f32", 0)])


@FORMS
@pytest.mark.parametrize("Hq,k,Dc,ps", [(16, 0, 512, 16), (16, 1, 256, 0), (48, 2, 512, 16), (128, 0, 256, 16)])
def test_rows_of_nothing_but_infinite_keys(kv, kernel, Hq, k, Dc, ps):
    inp = inputs([3, 70, 9, 40], kv, Hq, k, Dc, ps)
    for b, n in ((0, 3), (1, 70)):
        for r in rows(inp, b, range(n)):
            r[0] = -float("inf")
    o, l = compare(inp, kernel)
    assert np.isneginf(l[:2]).all() and (o[:2] == 0).all() and np.isfinite(o[2:, k]).all()


@FORMS
@pytest.mark.parametrize("lens", [[6000], [70, 200] * 150, [4000] * 40, [3000, 5] * 30])
def test_infinite_keys_among_others(kv, kernel, lens):
    """One workgroup a sequence, a few, many: the first 64 keys (whole tiles, and whole shares of long sequences)."""
    inp = inputs(lens, kv, 16, 0, 256, 64)
    for b in range(0, len(lens), 2):
        for r in rows(inp, b, range(min(64, lens[b] - 1))):
            r[0] = -float("inf")
    o, l = compare(inp, kernel)
    assert np.isnan(o[::2, 0, :, 0]).all() and np.isfinite(o[::2, 0, :, 1:]).all() and np.isfinite(l).all()


@FORMS
def test_long_sequences_of_nothing_but_infinite_keys(kv, kernel):
    inp = inputs([6000, 300], kv, 16, 1, 256, 64)
    for r in rows(inp, 0, range(6000)):
        r[0] = -float("inf")
    o, l = compare(inp, kernel)
    assert np.isneginf(l[0]).all() and (o[0] == 0).all()
