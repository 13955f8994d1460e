"""The operators as a serving loop uses them together: pages and slots, projections into the cache, attention over it,
pages of what was not accepted given back, on grouped heads and on a latent cache, over several rounds with ragged prompts
first.  The oracle keeps every sequence's rows in plain arrays and never sees a page."""
import numpy as np
import pytest
import torch

from oracle import latent_attn as LA
from oracle import rope_append as RA
from paper_2504_06419_amd import spire

pytestmark = pytest.mark.gpu
DEV = "cuda"
PS, POOL, MAXB, B, K = 16, 80, 20, 5, 2


class Pages:
    def __init__(self):
        self.table = torch.full((B, MAXB), -1, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(B, dtype=torch.int32, device=DEV)
        self.free = torch.randperm(POOL, generator=torch.Generator().manual_seed(1)).to(torch.int32).to(DEV)
        self.n = torch.tensor([POOL], dtype=torch.int32, device=DEV)

    def extend(self, new, pad=3):
        N = int(sum(new)) + pad
        slots = torch.empty(N, dtype=torch.int64, device=DEV)
        pos, cu = torch.empty(N, dtype=torch.int32, device=DEV), torch.empty(B + 1, dtype=torch.int32, device=DEV)
        spire.page_extend(self.table, PS, self.lens, torch.tensor(new, dtype=torch.int32, device=DEV), self.free, self.n,
                          slots, pos, cu)
        return N, slots, pos

    def release(self, keep):
        spire.page_release(self.table, PS, self.lens, torch.tensor(keep, dtype=torch.int32, device=DEV), self.free, self.n)


def rounds(append, attend, check):
    """append(N, slots, pos, new) -> rows kept by the oracle; attend(lens) after every round of K + 1 tokens."""
    pg, rng, lens = Pages(), np.random.default_rng(0), [0] * B
    new = [1, 40, 17, 0, 100]
    append(*pg.extend(new), new)
    lens = [a + b for a, b in zip(lens, new)]
    for _ in range(4):
        append(*pg.extend([K + 1] * B), [K + 1] * B)
        attend(pg, lens)
        lens = [n + int(rng.integers(1, K + 2)) for n in lens]
        check(lens)
        pg.release(lens)
        torch.cuda.synchronize()
        assert pg.lens.tolist() == lens
        held = [-(-n // PS) for n in lens]
        assert int(pg.n) == POOL - sum(held)
        ids = pg.free[:int(pg.n)].tolist() + [x for b in range(B) for x in pg.table[b, :held[b]].tolist()]
        assert sorted(ids) == list(range(POOL))  # no page lost, none twice


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_latent(kv):
    Hq, Dc, Dr = 16, 512, 64
    g = torch.Generator(device=DEV).manual_seed(2)
    dt = torch.bfloat16 if kv == "bf16" else torch.float8_e4m3fn
    scale = torch.full((1,), 0.02, device=DEV) if kv == "fp8" else None
    cache = torch.zeros(POOL, PS, Dc + Dr, device=DEV).to(dt)
    w = torch.rand(Dc, generator=g, device=DEV) + 0.5
    freq = (1e4 ** (-torch.arange(Dr // 2, device=DEV) * 2.0 / Dr))
    rows, last = [np.zeros((0, Dc + Dr)) for _ in range(B)], {}
    u, sc = (2.0**-8, 1.0) if kv == "bf16" else (2.0**-4, 0.02)

    def append(N, slots, pos, new):
        proj = torch.randn(N, Dc + Dr, generator=g, device=DEV).to(torch.bfloat16)
        qp = torch.randn(N, Hq, Dr, generator=g, device=DEV).to(torch.bfloat16)
        q = torch.randn(N, Hq, Dc + Dr, generator=g, device=DEV).to(torch.bfloat16)
        latent = q[..., :Dc].double().cpu().numpy()
        rope = spire.rope_view(pos, freq)
        spire.latent_append(spire.latent_view(cache, Dc, scale=scale), proj[:, :Dc], proj[:, Dc:], slots, rope, w, q_rope=qp, q=q)
        torch.cuda.synchronize()
        x, at = proj.double().cpu().numpy(), 0
        p = pos.cpu().numpy()[None]
        f = freq.double().cpu().numpy()
        full = np.concatenate([RA.rms(x[:, :Dc], w.double().cpu().numpy(), 1e-6), RA.rotate(x[:, None, Dc:], p, f)[:, 0]], 1)
        qs = np.concatenate([latent, RA.rotate(qp.double().cpu().numpy(), p, f)], -1)
        for b, m in enumerate(new):
            assert p[0, at:at + m].tolist() == list(range(len(rows[b]), len(rows[b]) + m))
            rows[b] = np.concatenate([rows[b], full[at:at + m]])
            at += m
        last.update(q=q, qs=qs)

    def attend(pg, lens):
        q = last["q"][:B * (K + 1)].view(B, K + 1, Hq, Dc + Dr)
        out, _ = spire.latent_verify_attn(q, spire.latent_view(cache, Dc, pg.table, scale=scale), pg.lens, K, 0.07)
        torch.cuda.synchronize()
        for b in range(B):
            c = rows[b][None]
            want, _, size = LA.verify(last["qs"][b * (K + 1):(b + 1) * (K + 1)][None], c, [len(rows[b])], K, 0.07, Dc)
            # rounded rows: u of each value directly, and through scores, whose error is a sum of 576 independent ones
            # of up to u 0.07 |q c|: 0.07 * 24 * u, six deviations of it at most
            tol = (u + 6 * 0.07 * 24 * u) * size + 2.0**-8 * size + 2.0**-10 * sc
            assert np.all(np.abs(out[b:b + 1].double().cpu().numpy() - want) <= tol)

    def check(lens):
        for b in range(B):
            rows[b] = rows[b][:lens[b]]

    rounds(append, attend, check)


def test_grouped_heads():
    Hq, Hkv, D = 8, 2, 128
    g = torch.Generator(device=DEV).manual_seed(3)
    kc = torch.zeros(POOL, Hkv, PS, D, device=DEV, dtype=torch.bfloat16)
    vc = torch.zeros_like(kc)
    wq, wk = torch.rand(D, generator=g, device=DEV) + 0.5, torch.rand(D, generator=g, device=DEV) + 0.5
    freq = 1e4 ** (-torch.arange(D // 2, device=DEV) * 2.0 / D)
    ks, vs, last = [np.zeros((0, Hkv, D)) for _ in range(B)], [np.zeros((0, Hkv, D)) for _ in range(B)], {}

    def append(N, slots, pos, new):
        x = torch.randn(N, Hq + 2 * Hkv, D, generator=g, device=DEV).to(torch.bfloat16)
        view = spire.kv_view(kc, vc, torch.zeros(1, 1, dtype=torch.int32, device=DEV), PS)
        q = spire.qkv_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], view, slots, spire.rope_view(pos, freq), wq, wk)
        torch.cuda.synchronize()
        y, p, f, at = x.double().cpu().numpy(), pos.cpu().numpy()[None], freq.double().cpu().numpy(), 0
        k = RA.rotate(RA.rms(y[:, Hq:Hq + Hkv], wk.double().cpu().numpy(), 1e-6), p, f)
        qs = RA.rotate(RA.rms(y[:, :Hq], wq.double().cpu().numpy(), 1e-6), p, f)
        for b, m in enumerate(new):
            ks[b], vs[b] = np.concatenate([ks[b], k[at:at + m]]), np.concatenate([vs[b], y[at:at + m, Hq + Hkv:]])
            at += m
        last.update(q=q, qs=qs)

    def attend(pg, lens):
        q = last["q"][:B * (K + 1)].view(B, K + 1, Hq, D)
        out, _ = spire.verify_attn(q, spire.kv_view(kc, vc, pg.table, PS), pg.lens, Hkv, K, 0.088)
        torch.cuda.synchronize()
        for b in range(B):
            for i in range(K + 1):
                n = len(ks[b]) - K + i
                for h in range(Hq):
                    s = ks[b][:n, h // 4] @ last["qs"][b * (K + 1) + i, h] * 0.088
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    v = vs[b][:n, h // 4]
                    # rounded queries and keys (u = 2^-8 each): scores off by 0.088 sqrt(128) u sqrt(2), six deviations
                    tol = (6 * 0.088 * 11.4 * 1.5 + 2) * 2.0**-8 * (p @ np.abs(v)) + 1e-6
                    assert np.all(np.abs(out[b, i, h].double().cpu().numpy() - p @ v) <= tol)

    def check(lens):
        for b in range(B):
            ks[b], vs[b] = ks[b][:lens[b]], vs[b][:lens[b]]

    rounds(append, attend, check)
