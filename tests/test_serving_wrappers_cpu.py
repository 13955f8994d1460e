"""The Python calls of the serving operators refuse arrays that do not have the sizes, types and order their kernels read
and write: the check comes before the library is called, on tensors without a GPU."""
import pytest
import torch

from paper_2504_06419_amd import spire

B, K, HQ, DC, DR = 3, 2, 4, 256, 64
I32 = torch.int32


@pytest.fixture
def called(monkeypatch):
    """Stands in for the library: counts the calls that reach it."""
    class Lib:
        calls = 0

        def __getattr__(self, name):
            def call(*args):
                Lib.calls += 1
                return 0
            return call
    lib = Lib()
    monkeypatch.setattr(spire, "load", lambda *a: lib)
    monkeypatch.setattr(spire, "_stream", lambda: 0)
    return Lib


def refused(called, call):
    before = called.calls
    with pytest.raises((AssertionError, ValueError)):
        call()
    assert called.calls == before


def attention(**kw):
    a = dict(q=torch.zeros(B, K + 1, HQ, DC + DR), cache=torch.zeros(6, 16, DC + DR), table=torch.zeros(B, 2, dtype=I32),
             scale=None, capacity=None, lens=torch.zeros(B, dtype=I32), out=torch.zeros(B, K + 1, HQ, DC),
             lse=torch.zeros(B, K + 1, HQ), ws=torch.zeros(256, dtype=torch.uint8))
    a.update(kw)
    view = spire.latent_view(a["cache"], DC, a["table"], a["scale"], a["capacity"])
    return spire.latent_verify_attn(a["q"], view, a["lens"], K, 0.1, out=a["out"], lse=a["lse"], ws=a["ws"])


def test_latent_attention_is_called(called):
    attention()
    attention(table=None)
    attention(table=None, capacity=16)
    attention(lens=torch.zeros(B, dtype=torch.int64))
    attention(lens=torch.zeros(2 * B, dtype=torch.int64)[::2])  # converted, and so in order
    attention(scale=torch.ones(1))
    attention(lens=torch.zeros(B + 5, dtype=I32), table=torch.zeros(B + 5, 2, dtype=I32))  # of the largest batch
    assert called.calls == 7


@pytest.mark.parametrize("kw", [
    dict(lens=torch.zeros(B - 1, dtype=I32)), dict(lens=torch.zeros(B - 1, dtype=torch.int64)),
    dict(lens=torch.zeros(2 * B, dtype=I32)[::2]),
    dict(lse=torch.zeros(B, K + 1, HQ, dtype=torch.float64)), dict(lse=torch.zeros(B, K + 1, HQ, dtype=torch.bfloat16)),
    dict(lse=torch.zeros(B, K, HQ)), dict(lse=torch.zeros(B, HQ, K + 1).transpose(1, 2)),
    dict(table=torch.zeros(B - 1, 2, dtype=I32)), dict(table=torch.zeros(2 * B, dtype=I32)),
    dict(table=torch.zeros(B, 2, dtype=torch.int64)), dict(table=None, cache=torch.zeros(B - 1, 16, DC + DR)),
    dict(table=None, capacity=17), dict(scale=torch.ones(1, dtype=torch.float64)), dict(scale=torch.ones(0))])
def test_latent_attention_refuses(called, kw):
    refused(called, lambda: attention(**kw))


def ints(n):
    return torch.zeros(n, dtype=I32)


def extend(**kw):
    a = dict(table=torch.zeros(B, 4, dtype=I32), lens=ints(B), new=ints(B), free=ints(9), n=ints(1),
             slots=torch.zeros(7, dtype=torch.int64), pos=ints(7), cu=ints(B + 1), lens_out=None, n_out=None)
    a.update(kw)
    spire.page_extend(a["table"], 16, a["lens"], a["new"], a["free"], a["n"], a["slots"], a["pos"], a["cu"],
                      a["lens_out"], a["n_out"], torch.zeros(4096, dtype=torch.uint8))


def release(**kw):
    a = dict(table=torch.zeros(B, 4, dtype=I32), lens=ints(B), new=ints(B), free=ints(9), n=ints(1), lens_out=None,
             n_out=None)
    a.update(kw)
    spire.page_release(a["table"], 16, a["lens"], a["new"], a["free"], a["n"], a["lens_out"], a["n_out"],
                       torch.zeros(4096, dtype=torch.uint8))


def test_pages_are_called(called):
    extend()
    extend(n_out=ints(1), lens_out=ints(B))
    release()
    release(n_out=ints(1), lens_out=ints(B), free=ints(0))
    assert called.calls == 4


@pytest.mark.parametrize("call", [extend, release])
@pytest.mark.parametrize("kw", [
    dict(n=ints(0)), dict(n_out=ints(0)), dict(n=torch.zeros(1, dtype=torch.int64)), dict(lens=ints(B - 1)),
    dict(new=ints(B - 1)), dict(lens_out=ints(B - 1)), dict(free=torch.zeros(9, dtype=torch.int64)),
    dict(lens=ints(2 * B)[::2])])
def test_pages_refuse(called, call, kw):
    refused(called, lambda: call(**kw))


@pytest.mark.parametrize("kw", [dict(slots=torch.zeros(6, dtype=torch.int64)), dict(slots=ints(7)), dict(cu=ints(B))])
def test_extend_refuses(called, kw):
    refused(called, lambda: extend(**kw))


def append(cache=(4, 2, 16, 64), **kw):
    x = torch.zeros(5, 12, 64)
    a = dict(q=x[:, :8], k=x[:, 8:10], v=x[:, 10:], slots=torch.zeros(5, dtype=torch.int64), qw=None)
    a.update(kw)
    k = torch.zeros(cache)
    view = spire.kv_view(k, torch.zeros_like(k), torch.zeros(1, 1, dtype=I32))
    return spire.qkv_append(a["q"], a["k"], a["v"], view, a["slots"], q_weight=a["qw"])


def test_append_is_called(called):
    append()
    append(cache=(4, 3, 16, 64))   # into the first heads of a cache of more
    assert called.calls == 2


@pytest.mark.parametrize("kw", [
    dict(cache=(4, 1, 16, 64)), dict(cache=(4, 2, 16, 32)), dict(slots=torch.zeros(4, dtype=torch.int64)),
    dict(slots=torch.zeros(5, dtype=I32)), dict(qw=torch.ones(32)), dict(q=torch.zeros(5, 64, 8).transpose(1, 2))])
def test_append_refuses(called, kw):
    refused(called, lambda: append(**kw))


def verify(noalloc=False, **kw):
    a = dict(lens=torch.zeros(B, dtype=I32), out=torch.zeros(B, K + 1, HQ, 64), lse=torch.zeros(B, K + 1, HQ))
    a.update(kw)
    q, cache = torch.zeros(B, K + 1, HQ, 64), torch.zeros(B, 2, 16, 64)
    view = spire.kv_view(cache, torch.zeros_like(cache))
    if noalloc:
        return spire.verify_attn_noalloc(q, view, a["lens"], 2, K, 0.1, a["out"], a["lse"])
    return spire.verify_attn(q, view, a["lens"], 2, K, 0.1, out=a["out"], lse=a["lse"],
                             ws=torch.zeros(256, dtype=torch.uint8))


@pytest.mark.parametrize("noalloc", [False, True])
def test_verify_is_called(called, noalloc):
    verify(noalloc)
    verify(noalloc, lens=torch.zeros(B + 2, dtype=torch.int64))
    verify(noalloc, lens=torch.zeros(2 * B, dtype=torch.int64)[::2])
    verify(noalloc, out=torch.zeros(B, K + 1, HQ, 64, dtype=torch.bfloat16))
    assert called.calls == 4


@pytest.mark.parametrize("noalloc", [False, True])
@pytest.mark.parametrize("kw", [
    dict(lens=torch.zeros(B - 1, dtype=I32)), dict(lens=torch.zeros(2 * B, dtype=I32)[::2]),
    dict(lse=torch.zeros(B, K + 1, HQ, dtype=torch.float64)), dict(lse=torch.zeros(B, K, HQ)),
    dict(lse=torch.zeros(B, HQ, K + 1).transpose(1, 2)), dict(out=torch.zeros(B, K, HQ, 64)),
    dict(out=torch.zeros(B, K + 1, HQ, 128)[..., :64])])
def test_verify_refuses(called, noalloc, kw):
    refused(called, lambda: verify(noalloc, **kw))
