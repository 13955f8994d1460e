"""Many small weights behind one large one: the first key's weight is 1, every other one's 2^-e.

Tolerance: a probability is off by half a step of fp16 (fp8 rows, 2^-11 of it, or half of the smallest step, 2^-25 on the
lifted scale and so 2^-32 of the largest) or of bf16 (2^-8 of it; its range is that of fp32), or not at all (fp32 path),
besides the parity tests' 2^-15.  A lane's part of the sum is 1 plus up to n / 4 weights, so it loses up to 2^-24 of 1 with
each addition (4 keys): n 2^-28 of the largest, which the outputs' small weights feel relative to 1 only."""
import numpy as np
import pytest
import torch

from tests.test_gpu_latent_attn import SCALE, Inp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e", [10, 16, 24, 26, 28])
@pytest.mark.parametrize("kv,kernel", [("fp8", 0), ("bf16", 0), ("fp8", 1)])
@pytest.mark.parametrize("lens,Hq,k,Dc", [([4096, 700] * 150, 4, 0, 512), ([4096, 900], 16, 1, 512),
                                          ([4096, 700] * 150, 4, 0, 256), ([3000, 4000], 128, 0, 256)])
def test_small_weights(kv, kernel, e, lens, Hq, k, Dc):
    inp = Inp(lens[:2], Hq, k, Dc=Dc, kv=kv, ps=64, seed=e)
    unit = SCALE if kv == "fp8" else 1.0
    inp.q.zero_()
    inp.q[..., Dc] = 1
    rows = torch.randint(1, 9, inp.cache.shape, generator=torch.Generator().manual_seed(e)).to(inp.cache.device).float()
    rows[..., Dc:] = 0
    inp.cache.copy_(rows.to(inp.cache.dtype))
    first = [inp.cache[int(inp.table[b, 0]), 0] for b in range(2)]
    for r in first:
        r.zero_()
        r[Dc:Dc + 1] = torch.full((1,), 16.0, device=r.device).to(r.dtype)
    inp.sm = e * np.log(2.0) / (16.0 * unit)
    o, l, size = inp.oracle()
    reps = len(lens) // 2                    # the same two sequences, as often as makes them one workgroup's or many's
    inp.q, inp.dl = inp.q.repeat(reps, 1, 1, 1), inp.dl.repeat(reps)
    inp.table, inp.lens = inp.table.repeat(reps, 1).contiguous(), lens
    out, lse = (x.double().cpu().numpy().reshape((reps, 2) + x.shape[1:]) for x in inp.run("f32", kernel))
    n = np.array(lens[:2]).reshape(2, 1, 1, 1)
    c = 2.0**-15 + (0 if kernel == 1 else 2.0**-11 if kv == "fp8" else 2.0**-8)
    tiny = 2.0**-32 if kv == "fp8" and kernel == 0 else 0
    tol = (c + n * 2.0**-28) * size + n * tiny * 8 * unit
    err = np.abs(out - o)
    assert np.all(err <= tol), (err / tol).max()
    assert np.all(np.abs(lse - l) <= 2.0**-15 + 2.0**-22 * np.abs(l) + n[..., 0] * 2.0**-28)
