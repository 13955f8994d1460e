"""Attention over a latent cache in every shape of its kernels: one to eight blocks of 16 rows a workgroup on both widths,
units whose last blocks are not there, storage orders on each of them, and the fp32 kernel on contiguous storage and pages
off its tile of 32 keys.  Tolerances and inputs of the parity tests."""
import pytest
import torch

from tests.test_gpu_latent_attn import LENS, Inp, check

pytestmark = pytest.mark.gpu


def shape(Hq, k):
    """(blocks, units, blocks a unit) of the matrix kernel."""
    blocks = (k + 1) * -(-Hq // 16)
    units = -(-blocks // 8)
    return blocks, units, -(-blocks // units)


def run(inp, kernel=0):
    want = inp.oracle()
    a, b = inp.run("f32", kernel), inp.run("f32", kernel)
    assert torch.equal(a[0].isnan(), b[0].isnan()) and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    check(inp, "f32", kernel, want)
    check(inp, "bf16", kernel, want)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("Dc", [256, 512])
@pytest.mark.parametrize("nb,Hq,k", [(n, 16, n - 1) for n in range(1, 9)] + [(n, 16 * n, 0) for n in range(2, 8)] +
                         [(7, 100, 0), (6, 20, 2), (8, 30, 3)])
def test_blocks_of_a_workgroup(kv, Dc, nb, Hq, k):
    assert shape(Hq, k)[1:] == (1, nb)
    run(Inp(LENS, Hq, k, Dc=Dc, kv=kv, seed=nb + k))


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("Dc", [256, 512])
@pytest.mark.parametrize("Hq,k", [(64, 4), (16, 10), (16, 12), (48, 2), (80, 4), (80, 10)])
def test_units_with_missing_blocks(kv, Dc, Hq, k):
    blocks, units, nb = shape(Hq, k)
    assert units * nb > blocks
    run(Inp([0, 1, 3, 7, 16, 33, 65, 300, 5000], Hq, k, Dc=Dc, kv=kv, ps=64, seed=blocks))


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("Dc", [256, 512])
@pytest.mark.parametrize("ps", [0, 7, 64, 100])
@pytest.mark.parametrize("Hq,k", [(16, 1), (16, 3), (16, 4), (16, 5), (16, 6), (16, 7), (64, 4)])
def test_storage_of_split_sequences(kv, Dc, ps, Hq, k):
    """A few long sequences on all workgroups, and a short one between them."""
    run(Inp([3001, 5, 2500, 64], Hq, k, Dc=Dc, kv=kv, ps=ps, seed=ps + k))


@pytest.mark.parametrize("kv,kernel", [("f32", 0), ("bf16", 1), ("fp8", 1)])
@pytest.mark.parametrize("Dc", [256, 512])
@pytest.mark.parametrize("ps", [0, 1, 3, 7, 33, 100, 256])
def test_pages_of_the_fp32_kernel(kv, kernel, Dc, ps):
    run(Inp([0, 1, 31, 32, 33, 65, 190, 513], 8, 2, Dc=Dc, kv=kv, ps=ps, seed=ps), kernel)


@pytest.mark.parametrize("kv,kernel", [("f32", 0), ("bf16", 1), ("fp8", 1)])
@pytest.mark.parametrize("Dc", [256, 512])
@pytest.mark.parametrize("lens,Hq,k,ps", [([9000], 16, 0, 0), ([4000, 3, 0, 2500], 16, 4, 64), ([1500] * 3, 128, 0, 7),
                                          ([40] * 300, 8, 1, 16), ([64] * 600, 16, 0, 0), ([2000] + [10] * 40, 32, 1, 100)])
def test_split_sequences_of_the_fp32_kernel(kv, kernel, Dc, lens, Hq, k, ps):
    run(Inp(lens, Hq, k, Dc=Dc, kv=kv, ps=ps, seed=len(lens)), kernel)


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("Hq,k", [(16, 6), (112, 0), (64, 4), (16, 1)])
def test_hidden_keys_on_contiguous_storage(kv, Hq, k):
    """NaN behind every length of a contiguous cache changes nothing."""
    lens = [1, 5, 64, 65, 130, 0]
    for Dc in (256, 512):
        inp = Inp(lens, Hq, k, Dc=Dc, kv=kv, ps=0, seed=3)
        clean = inp.run()
        bits = inp.cache.view(torch.uint8) if kv == "fp8" else inp.cache
        for b, n in enumerate(lens):
            bits[b, n:] = 0x7F if kv == "fp8" else float("nan")
        got = inp.run()
        assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
