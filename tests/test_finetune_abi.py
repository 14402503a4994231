"""Host-side checks of the calls of petals_finetune.h, all of which fail before any device work.  No GPU."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2209_01188_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = [C.c_void_p(0x100000 * i) for i in range(1, 9)]         # aligned, never dereferenced
INVALID, CAPACITY, UNSUPPORTED = -1, -2, -3


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2209_01188_amd import build
    if not os.path.exists(b.LIB_PATH):
        build.build(force=False)


@pytest.fixture()
def client():
    cfg = b.ClientConfig(1000, 64, 1e-5, 8)
    h = C.c_void_p()
    p = b.ClientParams(*[0x10000] * 5)
    assert b.lib().petals_client_create(C.byref(cfg), C.byref(p), C.c_void_p(0x20000), C.byref(h)) == 0
    yield h
    assert b.lib().petals_client_destroy(h) == 0


def test_library_exports_every_symbol_of_the_header():
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "petals_finetune.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(petals_[a-z0-9_]+)\s*\(", header))
    assert declared == set(b.FINETUNE_EXPORTS) and len(declared) == 5
    for name in declared:
        assert hasattr(b.lib(), name), name


def test_logprobs_refusals(client):
    L, f = b.lib(), C.c_float
    logits, tok, lp, ent, top, tlp = FAKE[:6]

    def call(client=client, logits=logits, tok=tok, M=4, T=1.0, k=3, lp=lp, ent=ent, top=top, tlp=tlp):
        return L.petals_client_logprobs(client, logits, tok, M, f(T), k, lp, ent, top, tlp, None)
    assert call(client=None) == INVALID and call(logits=None) == INVALID
    assert call(M=0) == INVALID and call(M=-1) == INVALID and call(M=9) == CAPACITY
    assert call(tok=None) == INVALID and call(lp=None) == INVALID             # one without the other
    assert call(k=-1) == INVALID and call(k=65) == UNSUPPORTED
    assert call(k=0) == INVALID and call(k=0, top=None) == INVALID and call(top=None) == INVALID and call(tlp=None) == INVALID
    assert call(tok=None, lp=None, ent=None, k=0, top=None, tlp=None) == INVALID
    for T in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
        assert call(T=T) == INVALID and b"temperature" in L.petals_last_error()
    small, h = b.ClientConfig(5, 64, 1e-5, 8), C.c_void_p()
    p = b.ClientParams(*[0x10000] * 5)
    assert L.petals_client_create(C.byref(small), C.byref(p), C.c_void_p(0x20000), C.byref(h)) == 0
    assert call(client=h, k=6) == INVALID                                     # more alternatives than tokens
    assert L.petals_client_destroy(h) == 0


def test_distill_refusals(client):
    L, f = b.lib(), C.c_float
    logits, ids, vals, w, loss, grad = FAKE[:6]

    def call(client=client, logits=logits, M=4, ids=ids, vals=vals, K=3, T=1.0, loss=loss, grad=grad):
        return L.petals_client_distill(client, logits, M, ids, vals, K, f(T), w, loss, grad, None)
    assert call(client=None) == INVALID and call(logits=None) == INVALID and call(ids=None) == INVALID and call(vals=None) == INVALID
    assert call(M=0) == INVALID and call(M=9) == CAPACITY
    assert call(K=0) == INVALID and call(K=1025) == UNSUPPORTED
    assert call(loss=None, grad=None) == INVALID
    for T in (0.0, -2.0, float("nan"), float("inf"), 1e-45):
        assert call(T=T) == INVALID


def test_distill_refuses_outputs_over_inputs(client):
    L, f = b.lib(), C.c_float
    logits, ids, vals, w, loss, grad = FAKE[:6]
    for bad_loss, bad_grad in ((loss, vals), (loss, w), (loss, ids), (w, grad), (vals, grad), (ids, None), (logits, grad), (grad, grad)):
        assert L.petals_client_distill(client, logits, 4, ids, vals, 3, f(1.0), w, bad_loss, bad_grad, None) == INVALID


def test_embed_backward_refuses_outputs_over_inputs(client):
    ids, dy, tok, n = FAKE[:4]
    assert b.lib().petals_client_embed_backward(client, ids, dy, 4, tok, dy, n, None) == INVALID


def test_lm_head_backward_refusals(client):
    L = b.lib()
    store, x, g, out = FAKE[:4]

    def call(client=client, store=store, x=x, g=g, M=4, out=out):
        return L.petals_client_lm_head_backward(client, store, x, g, M, out, None)
    assert call(client=None) == INVALID and call(store=None) == INVALID and call(x=None) == INVALID
    assert call(g=None) == INVALID and call(out=None) == INVALID
    assert call(M=0) == INVALID and call(M=9) == CAPACITY
    assert call(store=C.c_void_p(0x100010)) == INVALID
    assert call(out=x) == INVALID and call(out=g) == INVALID
    n = C.c_size_t()
    cfg = b.ClientConfig(1000, 64, 1e-5, 8)
    assert L.petals_client_lm_head_backward_bytes(C.byref(cfg), 4, None) == INVALID
    assert L.petals_client_lm_head_backward_bytes(C.byref(cfg), 0, C.byref(n)) == INVALID
    assert L.petals_client_lm_head_backward_bytes(C.byref(cfg), 9, C.byref(n)) == CAPACITY
    assert L.petals_client_lm_head_backward_bytes(C.byref(b.ClientConfig(1000, 100, 1e-5, 8)), 4, C.byref(n)) == UNSUPPORTED
    # 2048 rows of a 7B1-shaped model: G as fp16 (1 GiB) and little else
    assert 2048 * 250880 * 2 <= b.petals_client_lm_head_backward_bytes(b.ClientConfig(250880, 4096, 1e-5, 2048), 2048) <= 2048 * 250880 * 2 * 1.5


def test_embed_backward_refusals(client):
    L = b.lib()
    ids, dy, tok, grads, n = FAKE[:5]

    def call(client=client, ids=ids, dy=dy, M=4, tok=tok, grads=grads, n=n):
        return L.petals_client_embed_backward(client, ids, dy, M, tok, grads, n, None)
    assert call(client=None) == INVALID and call(ids=None) == INVALID and call(dy=None) == INVALID
    assert call(tok=None) == INVALID and call(grads=None) == INVALID and call(n=None) == INVALID
    assert call(M=0) == INVALID and call(M=9) == CAPACITY and call(tok=ids) == INVALID


def test_the_binding_refuses_tensors_that_do_not_fit():
    """Types, shapes, devices and strides, on CPU tensors: nothing reaches the library."""
    c = object.__new__(b.Client)
    c.device, c.vocab, c.hidden, c.handle = torch.device("cpu"), 40, 64, None
    c.cfg = b.ClientConfig(40, 64, 1e-5, 8)
    f32, f16, i32 = torch.float32, torch.float16, torch.int32
    z = lambda dt, *s: torch.zeros(s, dtype=dt)                                # noqa: E731
    x = z(f32, 4, 40)
    bad = [lambda: c.logprobs(x[0]), lambda: c.logprobs(z(f16, 4, 40)), lambda: c.logprobs(z(f32, 4, 41)),
           lambda: c.logprobs(z(f32, 40, 4).T), lambda: c.logprobs(x, z(torch.int64, 4)), lambda: c.logprobs(x, z(i32, 3)),
           lambda: c.logprobs(x, top_k=41), lambda: c.logprobs(x, top_k=-1), lambda: c.logprobs([1.0]),
           lambda: c.distill(x, z(torch.int64, 4, 2), z(f32, 4, 2)), lambda: c.distill(x, z(i32, 4, 2), z(f32, 4, 3)),
           lambda: c.distill(x, z(i32, 3, 2), z(f32, 3, 2)), lambda: c.distill(x, z(i32, 4), z(f32, 4)),
           lambda: c.distill(x, z(i32, 4, 2), z(f32, 4, 2), loss_grad=z(f32, 4, 1)),
           lambda: c.distill(x, z(i32, 4, 2), z(f32, 4, 2), grad_out=z(f16, 4, 40)),
           lambda: c.lm_head_backward(z(f16, 4, 64), z(f16, 4, 40)), lambda: c.lm_head_backward(z(f32, 4, 64), x),
           lambda: c.lm_head_backward(z(f16, 3, 64), x), lambda: c.lm_head_backward(z(f16, 4, 64), x, store=z(torch.uint8, 8)),
           lambda: c.lm_head_backward(z(f16, 4, 64), x, out=z(f32, 4, 64)),
           lambda: c.embed_backward(z(torch.int64, 4), z(f16, 4, 64)), lambda: c.embed_backward(z(i32, 4), z(f16, 4, 32)),
           lambda: c.embed_backward(z(i32, 2, 2), z(f16, 4, 64)),
           lambda: c.embed_backward(z(i32, 4), z(f16, 4, 64), out=(z(i32, 4), z(f16, 4, 64), z(i32, 1)))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
