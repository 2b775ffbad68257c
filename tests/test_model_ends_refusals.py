"""Host-side refusals of the entry points of a model's ends (no GPU: arguments are checked before any CUDA call)."""
import ctypes as C

import pytest

from paper_2506_03077_b200 import binding as B
from paper_2506_03077_b200 import build as build_mod

P = 0x10000     # an aligned address that is never read: every call here is refused on the host
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return B.lib()


def call(lib, name, defaults, kw):
    unknown = set(kw) - set(defaults)
    assert not unknown
    return getattr(lib, name)(*{**defaults, **kw}.values())


def cfg(kw):
    c = dict(k=4, tail=0, temperature=1.0)
    c.update(kw.pop("cfg", {}))
    return C.byref(B.DistillCfgC(**c))


SCORE = dict(logits=P, ld=100, rows=3, vocab=100, dtype=0, tokens=P, ignore=-100, temperature=1.0, k=4, logp=P, lse=P, entropy=P,
             top_logp=P, top_ids=P, ws=P, ws_bytes=4096, stream=None)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), B.E_NULL), (dict(ws=None), B.E_NULL), (dict(tokens=None), B.E_NULL),
    (dict(logp=None, lse=None, entropy=None, top_logp=None, top_ids=None), B.E_NULL),
    (dict(logp=None, lse=None, entropy=None, k=0), B.E_NULL), (dict(dtype=2), B.E_DTYPE), (dict(rows=0), B.E_SHAPE),
    (dict(rows=2 ** 27 + 1), B.E_SHAPE), (dict(vocab=0), B.E_SHAPE), (dict(vocab=2 ** 27 + 1, ld=2 ** 28), B.E_SHAPE), (dict(ld=99), B.E_SHAPE),
    (dict(k=-1), B.E_SHAPE), (dict(k=129, vocab=200, ld=200), B.E_SHAPE), (dict(k=101), B.E_SHAPE), (dict(temperature=0.0), B.E_SHAPE),
    (dict(temperature=-1.0), B.E_SHAPE), (dict(temperature=NAN), B.E_SHAPE), (dict(temperature=INF), B.E_SHAPE), (dict(temperature=2.0 ** 21), B.E_SHAPE),
    (dict(logits=P + 2), B.E_ALIGN), (dict(logits=P + 1, dtype=1), B.E_ALIGN), (dict(tokens=P + 4), B.E_ALIGN), (dict(logp=P + 2), B.E_ALIGN),
    (dict(lse=P + 2), B.E_ALIGN), (dict(entropy=P + 1), B.E_ALIGN), (dict(top_logp=P + 2), B.E_ALIGN), (dict(top_ids=P + 4), B.E_ALIGN),
    (dict(ws=P + 128), B.E_ALIGN), (dict(ws_bytes=255), B.E_WORKSPACE)])
def test_token_logprobs(lib, kw, status):
    assert call(lib, "streambp_token_logprobs", SCORE, kw) == status


SCORE_GRAD = dict(logits=P, ld=100, rows=3, vocab=100, dtype=0, tokens=P, ignore=-100, temperature=1.0, lse=P, entropy=P, d_logp=P, d_lse=P,
                  d_entropy=P, d_logits=2 * P, ldd=100, stream=None)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), B.E_NULL), (dict(lse=None), B.E_NULL), (dict(d_logits=None), B.E_NULL), (dict(entropy=None), B.E_NULL),
    (dict(tokens=None), B.E_NULL), (dict(dtype=-1), B.E_DTYPE), (dict(rows=0), B.E_SHAPE), (dict(ld=99), B.E_SHAPE), (dict(ldd=99), B.E_SHAPE),
    (dict(d_logits=P, ldd=101), B.E_SHAPE), (dict(temperature=NAN), B.E_SHAPE), (dict(d_logits=P + 2), B.E_ALIGN), (dict(d_lse=P + 2), B.E_ALIGN)])
def test_token_logprobs_backward(lib, kw, status):
    assert call(lib, "streambp_token_logprobs_backward", SCORE_GRAD, kw) == status


DISTILL = dict(cfg=None, logits=P, ld=100, rows=3, vocab=100, dtype=1, ids=P, values=P, weight=P, row_loss=P, d_logits=2 * P, ldd=100, ws=P,
               ws_bytes=4096, stream=None)


@pytest.mark.parametrize("kw,status", [
    (dict(cfg=dict(k=0)), B.E_SHAPE), (dict(cfg=dict(k=129)), B.E_SHAPE), (dict(cfg=dict(tail=2)), B.E_SHAPE), (dict(cfg=dict(tail=-1)), B.E_SHAPE),
    (dict(cfg=dict(temperature=0.0)), B.E_SHAPE), (dict(cfg=dict(temperature=NAN)), B.E_SHAPE), (dict(logits=None), B.E_NULL),
    (dict(ids=None), B.E_NULL), (dict(values=None), B.E_NULL), (dict(ws=None), B.E_NULL), (dict(row_loss=None, d_logits=None), B.E_NULL),
    (dict(dtype=3), B.E_DTYPE), (dict(rows=0), B.E_SHAPE), (dict(vocab=B.DISTILL_MAX_VOCAB + 1, ld=10 ** 6, ldd=10 ** 6), B.E_SHAPE),
    (dict(ld=99), B.E_SHAPE), (dict(ldd=99), B.E_SHAPE), (dict(d_logits=P, ldd=101), B.E_SHAPE), (dict(logits=P + 1), B.E_ALIGN),
    (dict(d_logits=P + 1), B.E_ALIGN), (dict(ids=P + 4), B.E_ALIGN), (dict(values=P + 2), B.E_ALIGN), (dict(weight=P + 2), B.E_ALIGN),
    (dict(row_loss=P + 2), B.E_ALIGN), (dict(ws=P + 8), B.E_ALIGN), (dict(ws_bytes=0), B.E_WORKSPACE)])
def test_distill_topk(lib, kw, status):
    kw = dict(kw)
    kw["cfg"] = cfg(kw)
    assert call(lib, "streambp_distill_topk", DISTILL, kw) == status
    assert call(lib, "streambp_distill_topk", DISTILL, {}) == B.E_NULL


def head(**kw):
    c = dict(d_model=64, vocab=500, rms_eps=1e-6, ignore_index=-100, dtype=1)
    c.update(kw)
    return C.byref(B.HeadCfgC(**c))


HEAD_SCORE = dict(cfg=head(), g=P, w=P, H=P, tokens=P, T=10, chunk=4, temperature=1.0, k=4, logp=P, lse=P, entropy=P, top_logp=P, top_ids=P, ws=P,
                  ws_bytes=1 << 30, stream=None)
HEAD_DISTILL = dict(cfg=head(), distill=C.byref(B.DistillCfgC(4, 0, 1.0)), g=P, w=P, H=P, ids=P, values=P, weight=P, T=10, chunk=4, group=1, accumulate=0,
                    loss=P, row_loss=P, dH=P, dw=P, dg=P, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,status", [
    (dict(cfg=None), B.E_NULL), (dict(cfg=head(d_model=12)), B.E_SHAPE), (dict(g=None), B.E_NULL), (dict(H=None), B.E_NULL), (dict(T=0), B.E_SHAPE),
    (dict(chunk=0), B.E_SHAPE), (dict(k=129), B.E_SHAPE), (dict(tokens=None), B.E_NULL), (dict(temperature=0.0), B.E_SHAPE), (dict(w=P + 8), B.E_ALIGN),
    (dict(logp=None, lse=None, entropy=None, top_logp=None, top_ids=None), B.E_NULL), (dict(top_ids=P + 4), B.E_ALIGN), (dict(ws_bytes=4096), B.E_WORKSPACE)])
def test_lmhead_logprobs(lib, kw, status):
    assert call(lib, "streambp_lmhead_logprobs", HEAD_SCORE, kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(cfg=None), B.E_NULL), (dict(distill=None), B.E_NULL), (dict(distill=C.byref(B.DistillCfgC(200, 0, 1.0))), B.E_SHAPE),
    (dict(cfg=head(vocab=B.DISTILL_MAX_VOCAB + 8)), B.E_SHAPE), (dict(weight=None), B.E_NULL), (dict(loss=None), B.E_NULL), (dict(dw=None), B.E_NULL),
    (dict(T=0), B.E_SHAPE), (dict(chunk=0), B.E_SHAPE), (dict(group=0), B.E_SHAPE), (dict(dH=P + 8), B.E_ALIGN), (dict(values=P + 2), B.E_ALIGN),
    (dict(row_loss=P + 2), B.E_ALIGN), (dict(ws_bytes=4096), B.E_WORKSPACE)])
def test_lmhead_distill_backward(lib, kw, status):
    assert call(lib, "streambp_lmhead_distill_backward", HEAD_DISTILL, kw) == status


NORM = dict(x=P, ldx=64, gain=P, bias=P, eps=1e-5, rows=3, d=64, dtype=1, y=2 * P, ldy=64, mean=P, rstd=P, stream=None)
NORM_GRAD = dict(dy=P, lddy=64, x=P, ldx=64, gain=P, mean=P, rstd=P, add=P, ldadd=64, rows=3, d=64, dtype=1, dx=2 * P, lddx=64, dg=P, db=P,
                 accumulate=0, ws=P, ws_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), B.E_NULL), (dict(y=None), B.E_NULL), (dict(dtype=9), B.E_DTYPE), (dict(rows=0), B.E_SHAPE), (dict(d=0), B.E_SHAPE),
    (dict(d=2 ** 20 + 1, ldx=2 ** 21, ldy=2 ** 21), B.E_SHAPE), (dict(eps=-1.0), B.E_SHAPE), (dict(eps=NAN), B.E_SHAPE), (dict(eps=INF), B.E_SHAPE),
    (dict(ldx=63), B.E_SHAPE), (dict(ldy=63), B.E_SHAPE), (dict(y=P, ldy=65), B.E_SHAPE), (dict(x=P + 1), B.E_ALIGN), (dict(gain=P + 1), B.E_ALIGN),
    (dict(mean=P + 2), B.E_ALIGN)])
def test_layernorm_forward(lib, kw, status):
    assert call(lib, "streambp_layernorm_forward", NORM, kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dy=None), B.E_NULL), (dict(x=None), B.E_NULL), (dict(mean=None), B.E_NULL), (dict(rstd=None), B.E_NULL), (dict(ws=None), B.E_NULL),
    (dict(dx=None, dg=None, db=None), B.E_NULL), (dict(dtype=9), B.E_DTYPE), (dict(rows=0), B.E_SHAPE), (dict(d=0), B.E_SHAPE), (dict(lddy=63), B.E_SHAPE),
    (dict(ldadd=63), B.E_SHAPE), (dict(lddx=63), B.E_SHAPE), (dict(dx=P, lddx=65), B.E_SHAPE), (dict(dg=P + 2), B.E_ALIGN), (dict(add=P + 1), B.E_ALIGN),
    (dict(ws=P + 16), B.E_ALIGN), (dict(ws_bytes=256), B.E_WORKSPACE)])
def test_layernorm_backward(lib, kw, status):
    assert call(lib, "streambp_layernorm_backward", NORM_GRAD, kw) == status


EMBED = dict(table=P, ld=64, ids=P, n=3, vocab=100, d=64, dtype=1, scale=1.0, padding=-1, out=P, ldo=64, ws=P, ws_bytes=1 << 20, stream=None)
EMBED_GRAD = dict(dout=P, ldo=64, ids=P, n=3, vocab=100, d=64, dtype=1, scale=1.0, padding=-1, accumulate=0, dtable=P, ws=P, ws_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("kw,status", [
    (dict(table=None), B.E_NULL), (dict(ids=None), B.E_NULL), (dict(out=None), B.E_NULL), (dict(ws=None), B.E_NULL), (dict(dtype=5), B.E_DTYPE),
    (dict(n=0), B.E_SHAPE), (dict(n=2 ** 30), B.E_SHAPE), (dict(vocab=0), B.E_SHAPE), (dict(vocab=2 ** 31 - 1), B.E_SHAPE), (dict(d=0), B.E_SHAPE),
    (dict(scale=NAN), B.E_SHAPE), (dict(scale=INF), B.E_SHAPE), (dict(ld=63), B.E_SHAPE), (dict(ldo=63), B.E_SHAPE), (dict(table=P + 1), B.E_ALIGN),
    (dict(ids=P + 4), B.E_ALIGN), (dict(ws=P + 16), B.E_ALIGN), (dict(ws_bytes=16), B.E_WORKSPACE)])
def test_embedding_forward(lib, kw, status):
    assert call(lib, "streambp_embedding_forward", EMBED, kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dout=None), B.E_NULL), (dict(ids=None), B.E_NULL), (dict(dtable=None), B.E_NULL), (dict(ws=None), B.E_NULL), (dict(dtype=5), B.E_DTYPE),
    (dict(n=0), B.E_SHAPE), (dict(vocab=0), B.E_SHAPE), (dict(d=2 ** 20 + 1, ldo=2 ** 21), B.E_SHAPE), (dict(ldo=63), B.E_SHAPE), (dict(dout=P + 1), B.E_ALIGN),
    (dict(dtable=P + 4), B.E_ALIGN), (dict(ws=P + 16), B.E_ALIGN), (dict(ws_bytes=512), B.E_WORKSPACE), (dict(scale=NAN), B.E_SHAPE)])
def test_embedding_backward(lib, kw, status):
    assert call(lib, "streambp_embedding_backward", EMBED_GRAD, kw) == status


def test_sizes(lib):
    assert lib.streambp_layernorm_workspace_bytes(0, 8) == 0 and lib.streambp_layernorm_workspace_bytes(8, 0) == 0
    assert lib.streambp_embedding_backward_workspace_bytes(0, 8, 8) == 0 and lib.streambp_embedding_backward_workspace_bytes(8, 8, 2 ** 21) == 0
    assert lib.streambp_lmhead_distill_workspace_bytes(head(), 10, 4, 0) == 0 and lib.streambp_lmhead_logprobs_workspace_bytes(head(dtype=4), 10, 4) == 0
    assert lib.streambp_token_logprobs_workspace_bytes() >= 256 and lib.streambp_distill_topk_workspace_bytes() >= 256
