"""The operators between a layer's projections and its attention over a paged cache, in plain torch and as this
library's kernels: page tables and slot maps, norms and rotations of queries and keys on their way into the cache,
and attention over a cache of one shared latent per token.

`own` false: run() computes the plain form, elementary operations in 32 bits (64 for angles), rounded once at the
end; `own` true: run() makes the calls a serving program makes.

Ranges: batch 1..256; contexts 1..65536 tokens, log-uniform within a batch; k 0..7; 4..128 query heads on a latent of
256 or 512 and 64 rotated dimensions; f32, bf16 and fp8 caches, pages of 16..256 tokens or contiguous; appends of
1..16384 tokens, 1..64 query and 1..8 KV heads of 64..256, one to three position axes, both pair orders.
"""
import math

import torch

own = False

DEV = "cuda"
ES = {"f32": 4, "bf16": 2, "fp8": 1}
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
DR = 64       # rotated dimensions of a latent cache
EPS = 1e-6
KV_SCALE = 0.02


def _attn(name, B, Hq, k, Dc, lo, hi, kv, page, out):
    return dict(name=name, kind="attn", B=B, Hq=Hq, k=k, Dc=Dc, lo=lo, hi=hi, kv=kv, page=page, out=out)


def listed():
    return [
        # target verification on one of eight devices that share 128 heads: bound by the cache's bytes
        _attn("latent_verify_bf16_B64_h16_k4", 64, 16, 4, 512, 512, 16384, "bf16", 64, "bf16"),
        # one new token of a large batch with every head on one device: bytes and products about even
        _attn("latent_decode_bf16_B128_h128", 128, 128, 0, 512, 1024, 16384, "bf16", 64, "bf16"),
        # target verification with every head on one device: bound by the matrix products
        _attn("latent_verify_bf16_B32_h128_k3", 32, 128, 3, 512, 2048, 16384, "bf16", 16, "bf16"),
        # one new token of one long request: the cache's length split over the device and joined
        _attn("latent_decode_bf16_B1_h16_L65536", 1, 16, 0, 512, 65536, 65536, "bf16", 64, "bf16"),
        # target verification on an fp8 cache, long contexts
        _attn("latent_verify_fp8_B64_h32_k2", 64, 32, 2, 512, 1024, 32768, "fp8", 64, "bf16"),
        # the smallest call: a full-precision check run of a small model
        _attn("latent_verify_f32_B4_h8_k4", 4, 8, 4, 256, 512, 512, "f32", 0, "f32"),
        # a round's new tokens of 64 requests, 128 heads: latent normed, key and queries rotated, cache written
        dict(name="latent_append_N320_h128", kind="lappend", N=320, Hq=128, Dc=512, kv="bf16", page=64, inter=True),
        # prompts, 16 heads of a device
        dict(name="latent_append_N8192_h16", kind="lappend", N=8192, Hq=16, Dc=512, kv="bf16", page=64, inter=True),
        # a round's new tokens of 64 requests on grouped heads: per-head norms, rotation, cache write
        dict(name="qkv_append_N320_bf16", kind="qkv", N=320, Hq=32, Hkv=8, D=128, rot=128, axes=1, inter=False,
             new="bf16", kv="bf16", page=16, norm=True),
        # prompts with images: positions of time, height and width, an fp8 cache
        dict(name="qkv_append_N8192_axes_fp8", kind="qkv", N=8192, Hq=32, Hkv=8, D=128, rot=128, axes=3, inter=False,
             new="bf16", kv="fp8", page=16, norm=True),
        # a round of a large batch: k + 1 tokens get pages and slots, what was not accepted goes back
        dict(name="pages_round_B256_k4", kind="pages", B=256, page=16, lo=512, hi=65536, nlo=5, nhi=5, back=True),
        # admission of 64 prompts
        dict(name="pages_prompts_B64", kind="pages", B=64, page=64, lo=1, hi=4096, nlo=16, nhi=16384, back=False),
    ]


# ---- drawing -----------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_attn(rng):
    kv = rng.choice(["bf16", "bf16", "bf16", "fp8", "fp8", "f32"])
    Dc, k = rng.choice([512, 512, 256]), rng.choice([0, 0, 1, 2, 3, 4, 5, 7])
    Hq = rng.choice([4, 8, 16, 16, 20, 32, 64, 128, 128])
    hi = _log(rng, 1, 65536)
    c = dict(kind="attn", B=_log(rng, 1, 256), Hq=Hq, k=k, Dc=Dc, lo=_log(rng, max(1, hi // 64), hi), hi=hi, kv=kv,
             page=rng.choice([0, 16, 64, 64, 128, 256]), out="f32" if kv == "f32" else "bf16")
    most = 0.02 if kv == "f32" else 1.0  # full precision belongs to check runs
    while True:
        w = work(c)
        if w["bytes"] <= 8e8 * most and w["flops"] <= 2.4e11 * most and c["B"] * c["hi"] <= 2e6:
            return c
        if c["B"] > 1:
            c["B"] = (c["B"] + 1) // 2
        else:
            c["hi"] = max(1, c["hi"] // 2)
            c["lo"] = min(c["lo"], c["hi"])


def draw(rng):
    kind = rng.choice(["attn"] * 5 + ["lappend", "lappend", "qkv", "qkv", "pages", "pages"])
    if kind == "attn":
        return _draw_attn(rng)
    N = _log(rng, 1, 16384)
    if kind == "lappend":
        Hq = rng.choice([4, 16, 16, 20, 32, 128])
        return dict(kind=kind, N=min(N, 131072 // Hq), Hq=Hq, Dc=rng.choice([512, 512, 256]),
                    kv=rng.choice(["bf16", "bf16", "fp8", "f32"]), page=rng.choice([16, 64, 64, 256]),
                    inter=rng.choice([True, False]))
    if kind == "qkv":
        Hkv = rng.choice([1, 2, 8, 8])
        Hq, D = Hkv * rng.choice([1, 4, 4, 8]), rng.choice([64, 128, 128, 256])
        return dict(kind=kind, N=min(N, 8192 * 48 * 128 // ((Hq + 2 * Hkv) * D)), Hq=Hq, Hkv=Hkv, D=D,
                    rot=rng.choice([D, D, D // 2]), axes=rng.choice([1, 1, 2, 3]), inter=rng.choice([True, False]),
                    new=rng.choice(["bf16", "bf16", "f32"]), kv=rng.choice(["bf16", "bf16", "fp8", "f32"]),
                    page=rng.choice([16, 16, 64, 256]), norm=rng.choice([True, True, False]))
    if rng.random() < 0.5:
        k = rng.randint(1, 8)
        return dict(kind="pages", B=_log(rng, 1, 256), page=rng.choice([1, 16, 16, 64]), lo=1,
                    hi=_log(rng, 64, 65536), nlo=k, nhi=k, back=True)
    nhi = _log(rng, 16, 16384)
    return dict(kind="pages", B=_log(rng, 1, 64), page=rng.choice([16, 16, 64, 128]), lo=1, hi=_log(rng, 16, 4096),
                nlo=_log(rng, 1, nhi), nhi=nhi, back=rng.choice([True, False]))


# ---- inputs ------------------------------------------------------------------------
def _spread(lo, hi, B):
    """B lengths at the quantiles of a log-uniform distribution: the same for every seed."""
    return [int(round(lo * (hi / lo) ** ((b + 0.5) / B))) for b in range(B)]


def _gens(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    h = torch.Generator()
    h.manual_seed(seed)
    return g, h


def _shuffled(values, h):
    return torch.tensor(values, dtype=torch.int32)[torch.randperm(len(values), generator=h)]


def _norm(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.bfloat16 if dtype is torch.bfloat16 else torch.float32)


def _cache(g, kv, *shape):
    """A cache's content: unit variance, in fp8 as multiples of the scale."""
    x = _norm(g, *shape, dtype=DT[kv])
    return (x / KV_SCALE).clamp_(-448, 448).to(DT[kv]) if kv == "fp8" else x


def _freq(rot, g):
    i = torch.arange(rot // 2, device=DEV, dtype=torch.float64)
    return (1e6 ** (-2.0 * i / rot)).float()


def _prepare_attn(c, seed):
    g, h = _gens(seed)
    B, Dk, ps = c["B"], c["Dc"] + DR, c["page"]
    lens = _shuffled(_spread(c["lo"], c["hi"], B), h)
    s = dict(q=_norm(g, B, c["k"] + 1, c["Hq"], Dk, dtype=DT["f32" if c["kv"] == "f32" else "bf16"]),
             lens=lens.to(DEV), sm=1.0 / math.sqrt(128 + DR), table=None, scale=None)
    if c["kv"] == "fp8":
        s["scale"] = torch.full((1,), KV_SCALE, device=DEV)
    if ps:
        need = (lens + ps - 1) // ps
        total = int(need.sum())
        perm = torch.randperm(total, generator=h).to(torch.int32)
        table = torch.zeros(B, int(need.max()), dtype=torch.int32)
        at = torch.arange(table.shape[1])[None] < need[:, None]
        table[at] = perm
        s["table"] = table.to(DEV)
        s["cache"] = _cache(g, c["kv"], total, ps, Dk)
    else:
        s["cache"] = _cache(g, c["kv"], B, max(1, c["hi"]), Dk)
    return s


def _positions(axes, N, g):
    """Runs of text, and of patches with their row and column."""
    t = torch.arange(N, device=DEV) + int(torch.randint(0, 100000, (1,), generator=g, device=DEV))
    i = torch.arange(N, device=DEV)
    return torch.stack([t, t - i % 256 + (i // 16) % 16, t - i % 256 + i % 16][:axes]).to(torch.int32)


def _slots(N, ps, h):
    """Token t at its place in shuffled pages; the last few are padding and have none."""
    pages = (N + ps - 1) // ps + 2
    perm = torch.randperm(pages, generator=h)
    t = torch.arange(N)
    s = perm[t // ps] * ps + t % ps
    if N >= 16:
        s[N - N // 16:] = -1
    return s.to(DEV), pages


def _prepare_lappend(c, seed):
    g, h = _gens(seed)
    N, Hq, Dc = c["N"], c["Hq"], c["Dc"]
    new = DT["f32" if c["kv"] == "f32" else "bf16"]
    slots, pages = _slots(N, c["page"], h)
    return dict(proj=_norm(g, N, Dc + DR, dtype=new), qproj=_norm(g, N, Hq, 128 + DR, dtype=new), slots=slots,
                cache=_cache(g, c["kv"], pages, c["page"], Dc + DR), q=torch.zeros(N, Hq, Dc + DR, device=DEV, dtype=new),
                w=1 + 0.1 * _norm(g, Dc), freq=_freq(DR, g), pos=_positions(1, N, g),
                scale=torch.full((1,), KV_SCALE, device=DEV) if c["kv"] == "fp8" else None)


def _prepare_qkv(c, seed):
    g, h = _gens(seed)
    N, Hq, Hkv, D, rot = c["N"], c["Hq"], c["Hkv"], c["D"], c["rot"]
    slots, pages = _slots(N, c["page"], h)
    axis = torch.arange(rot // 2, device=DEV, dtype=torch.int32) * c["axes"] // (rot // 2)
    scale = torch.full((Hkv,), KV_SCALE, device=DEV) * (1 + torch.arange(Hkv, device=DEV) / 8)
    return dict(proj=_norm(g, N, (Hq + 2 * Hkv) * D, dtype=DT[c["new"]]), slots=slots,
                kc=_cache(g, c["kv"], pages, Hkv, c["page"], D), vc=_cache(g, c["kv"], pages, Hkv, c["page"], D),
                table=torch.zeros(1, 1, device=DEV, dtype=torch.int32), q=torch.zeros(N, Hq, D, device=DEV, dtype=DT[c["new"]]),
                qw=1 + 0.1 * _norm(g, D) if c["norm"] else None, kw=1 + 0.1 * _norm(g, D) if c["norm"] else None,
                freq=_freq(rot, g), axis=axis if c["axes"] > 1 else None, pos=_positions(c["axes"], N, g),
                scale=scale if c["kv"] == "fp8" else None)


def _prepare_pages(c, seed):
    g, h = _gens(seed)
    B, ps = c["B"], c["page"]
    lens, new = _shuffled(_spread(c["lo"], c["hi"], B), h), _shuffled(_spread(c["nlo"], c["nhi"], B), h)
    held = (lens + ps - 1) // ps
    pool = int(held.sum() + ((new + ps - 1) // ps).sum()) + B  # enough, and the same for every seed
    perm = torch.randperm(pool, generator=h).to(torch.int32)
    maxb = -(-(c["hi"] + c["nhi"]) // ps) + 1
    table = torch.full((B, maxb), -1, dtype=torch.int32)
    used = int(held.sum())
    table[torch.arange(maxb)[None] < held[:, None]] = perm[:used]
    free = torch.full((pool,), -1, dtype=torch.int32)
    free[:pool - used] = perm[used:]
    total = int(new.sum())
    keep = lens + (torch.rand(B, generator=h) * (new + 1)).to(torch.int32).clamp_(max=new)
    d = dict(table=table, lens=lens, new=new, free=free, nfree=torch.tensor([pool - used], dtype=torch.int32),
             back=torch.full((pool,), -1, dtype=torch.int32), nback=torch.zeros(1, dtype=torch.int32), keep=keep)
    s = {k: v.to(DEV) for k, v in d.items()}
    s.update(tokens=total + total // 32, after=torch.empty_like(s["lens"]), nleft=torch.empty_like(s["nfree"]),
             slots=torch.empty(total + total // 32, device=DEV, dtype=torch.int64),
             pos=torch.empty(total + total // 32, device=DEV, dtype=torch.int32),
             cu=torch.empty(B + 1, device=DEV, dtype=torch.int32), kept=torch.empty_like(s["lens"]),
             nb=torch.empty_like(s["nback"]))
    return s


def prepare(case, seed):
    s = {"attn": _prepare_attn, "lappend": _prepare_lappend, "qkv": _prepare_qkv, "pages": _prepare_pages}[case["kind"]](case, seed)
    s["c"] = dict(case)
    return s


# ---- plain forms -------------------------------------------------------------------
def _plain_attn(s):
    c, Dc = s["c"], s["c"]["Dc"]
    B, nq, Hq, Dk = s["q"].shape
    kk = s["cache"] if s["table"] is None else s["cache"].view(torch.uint8 if c["kv"] == "fp8" else s["cache"].dtype)[s["table"].long()].view(s["cache"].dtype)
    kk = kk.reshape(B, -1, Dk).float()
    if s["scale"] is not None:
        kk = kk * s["scale"]
    sc = torch.matmul(s["q"].float().view(B, nq * Hq, Dk), kk.transpose(1, 2)) * s["sm"]
    lim = s["lens"][:, None] - c["k"] + torch.arange(nq, device=DEV)
    seen = torch.arange(kk.shape[1], device=DEV) < lim.repeat_interleave(Hq, 1)[:, :, None]
    sc = torch.where(seen, sc, torch.full_like(sc, -math.inf))
    m = sc.amax(2, keepdim=True)
    p = torch.exp(sc - torch.where(m == -math.inf, torch.zeros_like(m), m))
    l = p.sum(2, keepdim=True)
    out = torch.matmul(p, kk[:, :, :Dc]) / torch.where(l > 0, l, torch.ones_like(l))
    return out.view(B, nq, Hq, Dc).to(DT[c["out"]]), (m + torch.log(l)).view(B, nq, Hq)


def _rms(x, w):
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w


def _angles(s):
    """[N, rot/2] in 64 bits: far positions."""
    pos = s["pos"][0][:, None] if s.get("axis") is None else s["pos"].t()[:, s["axis"].long()]
    return pos.double() * s["freq"].double()


def _rotate(x, cos, sin, rot, inter):
    """x [N, heads, D]: the first `rot` elements in pairs, neighbours or halves."""
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if inter else (r[..., :rot // 2], r[..., rot // 2:])
    cos, sin = cos[:, None], sin[:, None]
    u, v = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([u, v], -1).flatten(-2) if inter else torch.cat([u, v], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _stored(x, kv, scale):
    return (x / scale).clamp(-448, 448).to(DT[kv]) if kv == "fp8" else x.to(DT[kv])


def _write(cache, slots, rows):
    """rows [N, ...] to cache[page, token, ...] at their slots."""
    live = (slots >= 0).nonzero()[:, 0]
    at = slots[live]
    bits = torch.uint8 if cache.dtype is torch.float8_e4m3fn else cache.dtype
    cache.view(bits)[at // cache.shape[1], at % cache.shape[1]] = rows.view(bits)[live]


def _plain_lappend(s):
    c, Dc = s["c"], s["c"]["Dc"]
    ang = _angles(s)
    cos, sin = ang.cos().float(), ang.sin().float()
    x = s["proj"].float()
    row = torch.cat([_rms(x[:, :Dc], s["w"]), _rotate(x[:, None, Dc:], cos, sin, DR, c["inter"])[:, 0]], 1)
    _write(s["cache"], s["slots"], _stored(row, c["kv"], s["scale"]))
    s["q"][..., Dc:] = _rotate(s["qproj"][..., 128:].float(), cos, sin, DR, c["inter"]).to(s["q"].dtype)
    return s["q"][..., Dc:], s["cache"]


def _plain_qkv(s):
    c = s["c"]
    N, Hq, Hkv, D = c["N"], c["Hq"], c["Hkv"], c["D"]
    ang = _angles(s)
    cos, sin = ang.cos().float(), ang.sin().float()
    x = s["proj"].float().view(N, Hq + 2 * Hkv, D)
    s["q"].copy_(_rotate(_rms(x[:, :Hq], s["qw"]), cos, sin, c["rot"], c["inter"]))
    k = _rotate(_rms(x[:, Hq:Hq + Hkv], s["kw"]), cos, sin, c["rot"], c["inter"])
    scale = None if s["scale"] is None else s["scale"][:, None]
    _write(s["kc"].transpose(1, 2), s["slots"], _stored(k, c["kv"], scale))
    _write(s["vc"].transpose(1, 2), s["slots"], _stored(x[:, Hq + Hkv:], c["kv"], scale))
    return s["q"], s["kc"], s["vc"]


def _plain_pages(s):
    c, ps, lens, new = s["c"], s["c"]["page"], s["lens"].long(), s["new"].long()
    B, maxb = s["table"].shape
    held, want = (lens + ps - 1) // ps, (lens + new + ps - 1) // ps
    need, cu = (want - held).cumsum(0), new.cumsum(0)
    n = s["nfree"].long()
    ok = (need <= n) & (cu <= s["tokens"])
    given = torch.where(ok, want - held, 0)
    first = given.cumsum(0) - given
    col = torch.arange(maxb, device=DEV)[None]
    nth = first[:, None] + col - held[:, None]
    fresh = (col >= held[:, None]) & (col < (held + given)[:, None])
    page = s["free"].long()[(n - 1 - nth).clamp(0, s["free"].shape[0] - 1)]
    s["table"].copy_(torch.where(fresh, page, s["table"].long()))
    i = torch.arange(s["tokens"], device=DEV)
    b = torch.searchsorted(cu, i, right=True).clamp(max=B - 1)
    pos = lens[b] + i - (cu - new)[b]
    live = (i < cu[-1]) & ok[b]
    slot = s["table"].long()[b, (pos // ps).clamp(max=maxb - 1)] * ps + pos % ps
    s["slots"].copy_(torch.where(live, slot, -1))
    s["pos"].copy_(torch.where(live, pos, 0))
    s["cu"].copy_(torch.cat([cu.new_zeros(1), cu]))
    s["after"].copy_(torch.where(ok, lens + new, lens))
    s["nleft"].copy_(n - given.sum())
    if not c["back"]:
        return s["table"], s["slots"], s["pos"], s["cu"], s["after"], s["nleft"]
    after, keep = s["after"].long(), torch.minimum(s["keep"].long(), s["after"].long())
    h0, h1 = (keep + ps - 1) // ps, (after + ps - 1) // ps
    at = s["nback"].long() + (h1 - h0).cumsum(0) - (h1 - h0)
    gone = (col >= h0[:, None]) & (col < h1[:, None])
    to = (at[:, None] + col - h0[:, None])[gone]
    s["back"][to] = s["table"][gone]
    s["kept"].copy_(keep)
    s["nb"].copy_(s["nback"] + (h1 - h0).sum())
    return s["table"], s["slots"], s["pos"], s["cu"], s["after"], s["nleft"], s["back"], s["kept"], s["nb"]


# ---- the library's calls -----------------------------------------------------------
def _own_attn(s):
    from paper_2504_06419_amd import spire
    c = s["c"]
    if "ws" not in s:  # a serving program keeps its workspace
        s["ws"] = spire.workspace(spire.latent_workspace_size(c["B"], c["Hq"], c["k"], c["Dc"], DR))
    view = spire.latent_view(s["cache"], c["Dc"], s["table"], scale=s["scale"])
    return spire.latent_verify_attn(s["q"], view, s["lens"], c["k"], s["sm"], ws=s["ws"], out_dtype=DT[c["out"]])


def _own_lappend(s):
    from paper_2504_06419_amd import spire
    c, Dc = s["c"], s["c"]["Dc"]
    view = spire.latent_view(s["cache"], Dc, s["table"] if "table" in s else None, scale=s["scale"])
    rope = spire.rope_view(s["pos"], s["freq"], interleaved=c["inter"])
    spire.latent_append(view, s["proj"][:, :Dc], s["proj"][:, Dc:], s["slots"], rope, s["w"], EPS,
                        q_rope=s["qproj"][..., 128:], q=s["q"])
    return s["q"][..., Dc:], s["cache"]


def _own_qkv(s):
    from paper_2504_06419_amd import spire
    c = s["c"]
    N, Hq, Hkv, D = c["N"], c["Hq"], c["Hkv"], c["D"]
    x = s["proj"].view(N, Hq + 2 * Hkv, D)
    view = spire.kv_view(s["kc"], s["vc"], s["table"], c["page"], s["scale"], s["scale"])
    rope = spire.rope_view(s["pos"], s["freq"], s["axis"], c["inter"])
    spire.qkv_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], view, s["slots"], rope, s["qw"], s["kw"], EPS, q_out=s["q"])
    return s["q"], s["kc"], s["vc"]


def _own_pages(s):
    from paper_2504_06419_amd import spire
    c = s["c"]
    if "ws" not in s:
        s["ws"] = spire.workspace(spire.page_workspace_size(c["B"]))
    spire.page_extend(s["table"], c["page"], s["lens"], s["new"], s["free"], s["nfree"], s["slots"], s["pos"], s["cu"],
                      lens_out=s["after"], n_free_out=s["nleft"], ws=s["ws"])
    if not c["back"]:
        return s["table"], s["slots"], s["pos"], s["cu"], s["after"], s["nleft"]
    spire.page_release(s["table"], c["page"], s["after"], s["keep"], s["back"], s["nback"], lens_out=s["kept"],
                       n_free_out=s["nb"], ws=s["ws"])
    return s["table"], s["slots"], s["pos"], s["cu"], s["after"], s["nleft"], s["back"], s["kept"], s["nb"]


def run(state):
    kind = state["c"]["kind"]
    if own:
        return {"attn": _own_attn, "lappend": _own_lappend, "qkv": _own_qkv, "pages": _own_pages}[kind](state)
    return {"attn": _plain_attn, "lappend": _plain_lappend, "qkv": _plain_qkv, "pages": _plain_pages}[kind](state)


# ---- work --------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "attn":
        es, qs, Dk, rows = ES[c["kv"]], 4 if c["kv"] == "f32" else 2, c["Dc"] + DR, c["B"] * (c["k"] + 1) * c["Hq"]
        lens = _spread(c["lo"], c["hi"], c["B"])
        pairs = sum(max(0, n - i) for n in lens for i in range(c["k"] + 1))
        return {"bytes": sum(lens) * Dk * es + rows * (Dk * qs + c["Dc"] * ES[c["out"]] + 4),
                "flops": 2.0 * pairs * c["Hq"] * (Dk + c["Dc"])}
    if c["kind"] == "lappend":
        new, Dk = 4 if c["kv"] == "f32" else 2, c["Dc"] + DR
        return {"bytes": c["N"] * (Dk * (new + ES[c["kv"]]) + 2 * c["Hq"] * DR * new + 12),
                "flops": c["N"] * (4 * c["Dc"] + 3 * DR * (1 + c["Hq"]))}
    if c["kind"] == "qkv":
        new, D = ES[c["new"]], c["D"]
        return {"bytes": c["N"] * (((c["Hq"] + 2 * c["Hkv"]) + c["Hq"]) * D * new + 2 * c["Hkv"] * D * ES[c["kv"]] + 8 + 4 * c["axes"]),
                "flops": c["N"] * 7 * (c["Hq"] + c["Hkv"]) * D}
    new = _spread(c["nlo"], c["nhi"], c["B"])
    pages = sum(-(-n // c["page"]) for n in new)
    return {"bytes": 12 * sum(new) + 8 * pages * (2 if c["back"] else 1) + 28 * c["B"], "flops": 4.0 * sum(new)}


# ---- the definitions in 64 bits ----------------------------------------------------
def _exact_attn(c, seed):
    s = _prepare_attn(c, seed)
    B, k, Hq, Dc = c["B"], c["k"], c["Hq"], c["Dc"]
    out = torch.zeros(B, k + 1, Hq, Dc, dtype=torch.float64, device=DEV)
    lse = torch.full((B, k + 1, Hq), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["lens"].tolist()):
        if s["table"] is None:
            keys = s["cache"][b].double()
        else:
            ids = s["table"][b, :-(-n // c["page"])].tolist()
            keys = torch.stack([s["cache"][i] for i in ids]).double().flatten(0, 1)
        keys = keys[:n] * (1.0 if s["scale"] is None else s["scale"].double())
        for i in range(k + 1):
            if n - k + i > 0:
                seen = keys[:n - k + i]
                z = s["q"][b, i].double() @ seen.t().contiguous() * s["sm"]
                lse[b, i] = torch.logsumexp(z, 1)
                out[b, i] = torch.exp(z - lse[b, i][:, None]) @ seen[:, :Dc].contiguous()
    return out, lse


def _turn(x, ang, inter):
    """Complex numbers: pairs times e^(i angle)."""
    half = x.shape[-1] // 2
    z = torch.view_as_complex(x.reshape(*x.shape[:-1], half, 2).contiguous()) if inter else torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous())
    z = z * torch.polar(torch.ones_like(ang), ang)[:, None]
    return torch.view_as_real(z).reshape(x.shape) if inter else torch.cat([z.real, z.imag], -1)


def _place(cache, slots, rows, kv, scale):
    if kv == "fp8":
        rows = (rows / scale).clamp(-448, 448)
    flat = cache.reshape(-1, *cache.shape[2:])
    keep = slots >= 0
    flat[slots[keep]] = rows[keep]
    return flat.view(cache.shape)


def _exact_lappend(c, seed):
    s, Dc = _prepare_lappend(c, seed), c["Dc"]
    ang = torch.outer(s["pos"][0].double(), s["freq"].double())
    x = s["proj"].double()
    lat = x[:, :Dc] / (x[:, :Dc].pow(2).sum(1, keepdim=True) / Dc + EPS).sqrt() * s["w"].double()
    rows = torch.cat([lat, _turn(x[:, None, Dc:], ang, c["inter"])[:, 0]], 1)
    scale = None if s["scale"] is None else s["scale"].double()
    return _turn(s["qproj"][..., 128:].double(), ang, c["inter"]), _place(s["cache"].double(), s["slots"], rows, c["kv"], scale)


def _exact_qkv(c, seed):
    s = _prepare_qkv(c, seed)
    N, Hq, Hkv, D, rot = c["N"], c["Hq"], c["Hkv"], c["D"], c["rot"]
    axis = [0] * (rot // 2) if s["axis"] is None else s["axis"].tolist()
    ang = torch.stack([s["pos"][a].double() * f for a, f in zip(axis, s["freq"].double().tolist())], 1)
    x = s["proj"].double().view(N, Hq + 2 * Hkv, D)

    def through(y, w):
        if w is not None:
            y = y / (y.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * w.double()
        return torch.cat([_turn(y[..., :rot], ang, c["inter"]), y[..., rot:]], -1)

    scale = None if s["scale"] is None else s["scale"].double()[:, None]
    kc = _place(s["kc"].double().transpose(1, 2), s["slots"], through(x[:, Hq:Hq + Hkv], s["kw"]), c["kv"], scale)
    vc = _place(s["vc"].double().transpose(1, 2), s["slots"], x[:, Hq + Hkv:], c["kv"], scale)
    return through(x[:, :Hq], s["qw"]), kc.transpose(1, 2), vc.transpose(1, 2)


def exact(case, seed):
    if case["kind"] == "pages":
        return None  # whole numbers
    return {"attn": _exact_attn, "lappend": _exact_lappend, "qkv": _exact_qkv}[case["kind"]](case, seed)
