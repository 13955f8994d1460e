"""Refusals of the page, append and latent entry points: decided on the host, nothing enqueued, no device pointer
read."""
import ctypes as C

import pytest

from paper_2504_06419_amd import spire

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE = 0x10000


def msg():
    return spire.load().spire_last_error().decode()


def extend(**kw):
    a = dict(table=FAKE, ps=16, maxb=8, lens=FAKE, new=FAKE, B=4, free=FAKE, pool=10, n=FAKE, slots=FAKE, pos=FAKE,
             mt=64, cu=FAKE, lo=FAKE, no=FAKE, ws=FAKE, wb=1 << 20)
    a.update(kw)
    return spire.load().spire_page_extend(a["table"], a["ps"], a["maxb"], a["lens"], a["new"], a["B"], a["free"], a["pool"],
                                          a["n"], a["slots"], a["pos"], a["mt"], a["cu"], a["lo"], a["no"], a["ws"],
                                          a["wb"], None)


def release(**kw):
    a = dict(table=FAKE, ps=16, maxb=8, lens=FAKE, keep=FAKE, B=4, free=FAKE, pool=10, n=FAKE, lo=FAKE, no=FAKE, ws=FAKE,
             wb=1 << 20)
    a.update(kw)
    return spire.load().spire_page_release(a["table"], a["ps"], a["maxb"], a["lens"], a["keep"], a["B"], a["free"],
                                           a["pool"], a["n"], a["lo"], a["no"], a["ws"], a["wb"], None)


COMMON = [(dict(B=-1), INVALID), (dict(B=8193), UNSUPPORTED), (dict(pool=-1), INVALID), (dict(ps=0), INVALID),
          (dict(maxb=0), INVALID), (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(free=None), INVALID),
          (dict(n=None), INVALID), (dict(lo=None), INVALID), (dict(no=None), INVALID), (dict(lens=FAKE + 2), INVALID),
          (dict(ws=None), WORKSPACE), (dict(ws=FAKE + 4), WORKSPACE), (dict(wb=100), WORKSPACE)]


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(new=None), INVALID), (dict(mt=-1), INVALID), (dict(mt=(1 << 30) + 1), INVALID), (dict(slots=None), INVALID),
    (dict(pos=None), INVALID), (dict(cu=None), INVALID), (dict(slots=FAKE + 4), INVALID)])
def test_extend_refusals(kw, status):
    assert extend(**kw) == status and msg()


@pytest.mark.parametrize("kw,status", COMMON + [(dict(keep=None), INVALID)])
def test_release_refusals(kw, status):
    assert release(**kw) == status and msg()


def rope(rot=128, axes=1, inter=0, reserved=0, pos=FAKE, freq=FAKE, axis=None):
    r = spire.Rope()
    r.positions, r.inv_freq, r.axis = pos, freq, axis
    r.axes, r.rot_dim, r.interleaved, r.reserved = axes, rot, inter, reserved
    return r


def kv(dtype=spire.BF16, scales=False, **kw):
    d = spire.KV()
    d.k, d.v, d.block_table = FAKE, FAKE, FAKE
    d.k_scale = d.v_scale = FAKE if scales else None
    d.s_blk, d.s_head, d.s_tok = 8 * 16 * 128, 16 * 128, 128
    d.dtype, d.page_size, d.max_blocks, d.num_blocks = dtype, 16, 4, 16
    for n, x in kw.items():
        setattr(d, n, x)
    return d


def qkv(**kw):
    a = dict(q=FAKE, qs=4096, k=FAKE, ks=4096, v=FAKE, vs=4096, dt=spire.BF16, qw=FAKE, kw=FAKE, eps=1e-6, rope=rope(),
             kv=kv(), slots=FAKE, N=4, Hq=8, Hkv=2, D=128, out=FAKE, od=spire.BF16)
    a.update(kw)
    ref = lambda s: None if s is None else C.byref(s)  # noqa: E731
    return spire.load().spire_qkv_append(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["dt"], a["qw"], a["kw"],
                                         a["eps"], ref(a["rope"]), ref(a["kv"]), a["slots"], a["N"], a["Hq"], a["Hkv"],
                                         a["D"], a["out"], a["od"], None)


ROPES = [(dict(rope=rope(rot=3)), INVALID), (dict(rope=rope(rot=-2)), INVALID), (dict(rope=rope(rot=130)), INVALID),
         (dict(rope=rope(axes=0)), UNSUPPORTED), (dict(rope=rope(axes=9)), UNSUPPORTED),
         (dict(rope=rope(inter=2)), INVALID), (dict(rope=rope(reserved=1)), INVALID), (dict(rope=rope(pos=None)), INVALID),
         (dict(rope=rope(freq=None)), INVALID), (dict(rope=rope(pos=FAKE + 2)), INVALID),
         (dict(rope=rope(axis=FAKE + 1)), INVALID)]


@pytest.mark.parametrize("kw,status", ROPES + [
    (dict(N=-1), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=0), INVALID), (dict(Hq=4095), UNSUPPORTED),
    (dict(D=0), UNSUPPORTED), (dict(D=1025), UNSUPPORTED), (dict(dt=spire.FP8), UNSUPPORTED),
    (dict(od=spire.FP8), UNSUPPORTED), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(out=None), INVALID),
    (dict(slots=None), INVALID), (dict(slots=FAKE + 4), INVALID), (dict(q=FAKE + 1), INVALID),
    (dict(qw=FAKE + 2), INVALID), (dict(qs=-1), INVALID), (dict(kv=None), INVALID), (dict(kv=kv(dtype=5)), INVALID),
    (dict(kv=kv(dtype=spire.FP8)), INVALID), (dict(kv=kv(reserved=1)), INVALID), (dict(kv=kv(k=FAKE + 1)), INVALID),
    (dict(kv=kv(page_size=0, num_blocks=-1)), INVALID)])
def test_qkv_append_refusals(kw, status):
    assert qkv(**kw) == status and msg()


def test_no_tokens_is_a_no_op():
    assert qkv(N=0, q=None, k=None, v=None, out=None, slots=None) == OK
    assert lappend(N=0, c=None, k=None, q=None, out=None, slots=None) == OK
    assert lattn(B=0, q=None, out=None, ws=None, lens=None) == OK


def latent(dtype=spire.BF16, **kw):
    d = spire.Latent()
    d.c, d.block_table, d.scale = FAKE, FAKE, None
    d.s_blk, d.s_tok, d.dtype, d.Dc, d.Dr = 16 * 576, 576, dtype, 512, 64
    d.page_size, d.max_blocks, d.num_blocks, d.capacity = 16, 4, 16, 0
    for n, x in kw.items():
        setattr(d, n, x)
    return d


def lappend(**kw):
    a = dict(c=FAKE, cs=576, k=FAKE, ks=576, q=FAKE, qs=1000, qh=192, dt=spire.BF16, w=FAKE, eps=1e-6,
             rope=rope(rot=64), lat=latent(), slots=FAKE, N=4, Hq=16, out=FAKE, od=spire.BF16)
    a.update(kw)
    ref = lambda s: None if s is None else C.byref(s)  # noqa: E731
    return spire.load().spire_latent_append(a["c"], a["cs"], a["k"], a["ks"], a["q"], a["qs"], a["qh"], a["dt"], a["w"],
                                            a["eps"], ref(a["rope"]), ref(a["lat"]), a["slots"], a["N"], a["Hq"],
                                            a["out"], a["od"], None)


VIEWS = [(dict(lat=None), INVALID), (dict(lat=latent(c=None)), INVALID), (dict(lat=latent(dtype=9)), INVALID),
         (dict(lat=latent(reserved=1)), INVALID), (dict(lat=latent(Dc=0)), UNSUPPORTED), (dict(lat=latent(Dr=0)), UNSUPPORTED),
         (dict(lat=latent(s_tok=-1)), INVALID), (dict(lat=latent(dtype=spire.FP8)), INVALID),
         (dict(lat=latent(page_size=-1)), INVALID), (dict(lat=latent(c=FAKE + 1)), INVALID)]


@pytest.mark.parametrize("kw,status", VIEWS + [
    (dict(N=-1), INVALID), (dict(Hq=-1), INVALID), (dict(Hq=5000), UNSUPPORTED), (dict(rope=rope(rot=32)), INVALID),
    (dict(rope=rope(rot=66)), INVALID), (dict(c=None), INVALID), (dict(k=None), INVALID), (dict(q=None), INVALID),
    (dict(out=None), INVALID), (dict(slots=None), INVALID), (dict(dt=spire.FP8), UNSUPPORTED), (dict(eps=-1.0), INVALID),
    (dict(cs=-1), INVALID), (dict(qh=-1), INVALID), (dict(c=FAKE + 1), INVALID), (dict(w=FAKE + 1), INVALID)])
def test_latent_append_refusals(kw, status):
    assert lappend(**kw) == status and msg()


def lattn(**kw):
    a = dict(q=FAKE, qd=spire.BF16, lat=latent(), lens=FAKE, B=2, Hq=16, k=4, sm=0.1, out=FAKE, od=spire.BF16, lse=None,
             ws=FAKE, wb=1 << 30, opts=None)
    a.update(kw)
    ref = lambda s: None if s is None else C.byref(s)  # noqa: E731
    return spire.load().spire_latent_verify_attn_ex(a["q"], a["qd"], ref(a["lat"]), a["lens"], a["B"], a["Hq"], a["k"],
                                                    a["sm"], a["out"], a["od"], a["lse"], a["ws"], a["wb"], None,
                                                    ref(a["opts"]))


def options(**kw):
    o = spire.LaunchOpts()
    for n, x in kw.items():
        setattr(o, n, x)
    return o


@pytest.mark.parametrize("kw,status", VIEWS + [
    (dict(B=-1), INVALID), (dict(B=8193), UNSUPPORTED), (dict(Hq=0), INVALID), (dict(Hq=129), UNSUPPORTED),
    (dict(k=-1), UNSUPPORTED), (dict(k=16), UNSUPPORTED), (dict(qd=spire.FP8), UNSUPPORTED),
    (dict(od=spire.FP8), UNSUPPORTED), (dict(sm=0.0), INVALID), (dict(sm=float("inf")), INVALID),
    (dict(lat=latent(Dc=128)), UNSUPPORTED), (dict(lat=latent(Dr=32)), UNSUPPORTED),
    (dict(lat=latent(block_table=None)), INVALID), (dict(lat=latent(max_blocks=0)), INVALID),
    (dict(lat=latent(num_blocks=0)), INVALID), (dict(lat=latent(page_size=0, capacity=0)), INVALID),
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(lens=None), INVALID), (dict(q=FAKE + 2), INVALID),
    (dict(lse=FAKE + 2), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=FAKE + 16), WORKSPACE),
    (dict(opts=options(kernel=4)), INVALID), (dict(opts=options(reserved=1)), INVALID),
    (dict(opts=options(max_launches=1)), INVALID)])
def test_latent_attention_refusals(kw, status):
    assert lattn(**kw) == status and msg()


def test_workspace_of_invalid_sizes():
    L = spire.load()
    for a in [(-1, 16, 0, 512, 64), (1, 0, 0, 512, 64), (1, 129, 0, 512, 64), (1, 16, 16, 512, 64), (1, 16, 0, 128, 64),
              (9000, 16, 0, 512, 64), (1, 16, 0, 512, 32)]:
        assert L.spire_latent_workspace_size(*a) == 0
    assert L.spire_page_workspace_size(-1) == 0 and L.spire_page_workspace_size(8193) == 0
    assert L.spire_page_workspace_size(0) > 0
