"""Lengths and tables at the end of 32-bit key numbers.

Every page of the table is the same one, so a softmax over r repetitions of it has the page's output and its log-sum-exp
plus ln r.  Tolerances: a lane adds at most 2^19 times to its part of a row's sum (2^31 keys over 256 workgroups and 4
lanes, 4 keys a time), an accumulator 2^18 times (32 keys a time), each addition off by at most 2^-24 of the sum so far:
2^-5 and 2^-6 of the whole, besides the parity tests' own."""
import numpy as np
import pytest
import torch

from oracle import latent_attn as LA
from paper_2504_06419_amd import spire

pytestmark = pytest.mark.gpu
DEV = "cuda"
PS, DC, DR = 1024, 256, 64
MOST = 2**31 - 8192                    # a multiple of the page


def page_of(kv, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(1, PS, DC + DR, generator=g, device=DEV)
    return x.to(torch.bfloat16) if kv == "bf16" else (x * 50).clamp(-448, 448).to(torch.float8_e4m3fn)


@pytest.mark.parametrize("kv", ["fp8", "bf16"])
def test_latent(kv):
    cache = page_of(kv, 1)
    scale = torch.full((1,), 0.02, device=DEV) if kv == "fp8" else None
    table = torch.zeros(1, 2**31 // PS + 2, dtype=torch.int32, device=DEV)   # room for more than 2^31 keys
    q = torch.randn(1, 1, 16, DC + DR, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(torch.bfloat16)
    rows = cache.double().cpu().numpy() * (0.02 if kv == "fp8" else 1.0)
    want, lse, size = LA.verify(q.double().cpu().numpy(), rows, [PS], 0, 0.07, DC)
    for n in (2**31 - 1, MOST):          # the first is clamped to the second
        lens = torch.tensor([n], dtype=torch.int32, device=DEV)
        out, l = spire.latent_verify_attn(q, spire.latent_view(cache, DC, table, scale), lens, 0, 0.07)
        torch.cuda.synchronize()
        err = np.abs(out.double().cpu().numpy() - want)
        assert np.all(err <= (2.0**-8 + 2.0**-15 + 2.0**-5 + 2.0**-6) * size), err.max()
        assert np.all(np.abs(l.double().cpu().numpy() - lse - np.log(MOST // PS)) <= 2.0**-5 + 2.0**-15)


def test_many_sequences_of_any_length():
    """Lengths that would pass the prefix sums' 32 bits are clamped; the short ones beside them are right."""
    cache = page_of("bf16", 3)[:, :16].contiguous()
    B = 64
    table = torch.zeros(B, 4, dtype=torch.int32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(4)
    q = torch.randn(B, 1, 16, DC + DR, generator=g, device=DEV).to(torch.bfloat16)
    lens = torch.tensor([2**31 - 1 if b % 2 else b for b in range(B)], dtype=torch.int32, device=DEV)
    out, l = spire.latent_verify_attn(q, spire.latent_view(cache, DC, table), lens, 0, 0.07)
    torch.cuda.synchronize()
    rows = np.repeat(cache.double().cpu().numpy(), 4, 0).reshape(1, 64, DC + DR)
    want, lse, size = LA.verify(q.double().cpu().numpy(), np.repeat(rows, B, 0), lens.tolist(), 0, 0.07, DC)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= (2.0**-8 + 2.0**-15) * size + 2.0**-24)


def test_verify():
    g = torch.Generator(device=DEV).manual_seed(5)
    k = torch.randn(1, 1, PS, 128, generator=g, device=DEV).to(torch.bfloat16)
    v = torch.randn(1, 1, PS, 128, generator=g, device=DEV).to(torch.bfloat16)
    q = torch.randn(1, 1, 8, 128, generator=g, device=DEV).to(torch.bfloat16)
    table = torch.zeros(1, 2**31 // PS + 2, dtype=torch.int32, device=DEV)
    s = (q[0, 0].double() @ k[0, 0].double().T * 0.09).cpu()
    p = torch.softmax(s, -1)
    want, size = (p @ v[0, 0].double().cpu()), p @ v[0, 0].double().cpu().abs()
    lens = torch.tensor([2**31 - 1], dtype=torch.int32, device=DEV)
    out, l = spire.verify_attn(q, spire.kv_view(k, v, table), lens, 1, 0, 0.09)
    torch.cuda.synchronize()
    assert torch.all((out[0, 0].double().cpu() - want).abs() <= (2.0**-8 + 2.0**-15 + 2.0**-5 + 2.0**-6) * size)
    assert torch.all((l[0, 0].double().cpu() - torch.logsumexp(s, -1) - np.log(MOST // PS)).abs() <= 2.0**-5 + 2.0**-15)
