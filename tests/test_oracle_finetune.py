"""Pins for the oracle of the client's scoring and fine-tuning ends: torch's CPU autograd in fp64, central differences and
special cases.  No GPU."""
import numpy as np
import pytest
import torch

from oracle import finetune as of


def _t(a, grad=False):
    return torch.tensor(np.asarray(a, np.float64), dtype=torch.float64, requires_grad=grad)


@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
def test_logprobs_match_torch(T):
    r = np.random.default_rng(3)
    x = (r.standard_normal((5, 40)) * 4).astype(np.float32)
    tok = np.array([0, 39, 7, -1, 40])
    lp, ent, top, tlp = of.logprobs(x, tok, T, 6)
    want = torch.log_softmax(_t(x) / T, 1)
    assert np.allclose(lp[:3], want[torch.arange(3), torch.tensor(tok[:3])].numpy(), rtol=1e-13)
    assert (lp[3:] == 0).all()
    assert np.allclose(ent, torch.distributions.Categorical(logits=_t(x) / T).entropy().numpy(), rtol=1e-12)
    assert np.array_equal(top, torch.topk(_t(x), 6).indices.numpy())
    assert np.allclose(tlp, torch.topk(want, 6).values.numpy(), rtol=1e-13)


def test_rows_without_a_distribution_and_ruled_out_tokens():
    x = np.array([[-np.inf] * 4, [0.0, -np.inf, 0.0, -np.inf]], np.float32)
    lp, ent, top, tlp = of.logprobs(x, np.array([1, 1]), 1.0, 3)
    assert lp[0] == -np.inf and lp[1] == -np.inf and ent[0] == 0.0 and abs(ent[1] - np.log(2)) < 1e-15
    assert top.tolist() == [[0, 1, 2], [0, 2, 1]] and (tlp[0] == -np.inf).all()
    loss, grad = of.distill(x, np.array([[1], [1]]), np.zeros((2, 1), np.float32))
    assert (loss == np.inf).all() and (grad[0] == 0).all() and np.allclose(grad[1], [0.5, -1.0, 0.5, 0.0])
    loss, grad = of.distill(x, np.array([[-1], [4]]), np.zeros((2, 1), np.float32))       # no list
    assert (loss == 0).all() and (grad == 0).all()


@pytest.mark.parametrize("T,K", [(1.0, 1), (2.0, 7), (0.7, 30)])
def test_distillation_matches_autograd_and_differences(T, K):
    r = np.random.default_rng(K)
    x = r.standard_normal((4, 30)) * 2
    ids = np.stack([r.permutation(30)[:K] for _ in range(4)])
    vals = r.standard_normal((4, K))
    if K > 2:
        ids[1, 2] = ids[1, 0]                # the same token twice
        ids[2, 1] = -1                       # a shorter list
    w = r.random(4) + 0.5
    loss, grad = of.distill(x, ids, vals, T, w)
    z = _t(x, True)
    keep = _t(np.where(ids < 0, -np.inf, vals))
    logp = torch.log_softmax(keep / T, 1)
    logq = torch.log_softmax(z / T, 1).gather(1, torch.tensor(np.maximum(ids, 0)))
    want = T * T * torch.where(logp > -np.inf, logp.exp() * (torch.where(logp > -np.inf, logp, torch.zeros_like(logp)) - logq), torch.zeros_like(logq)).sum(1)
    (want * _t(w)).sum().backward()
    assert np.allclose(loss, want.detach().numpy(), rtol=1e-12)
    assert np.allclose(grad, z.grad.numpy(), rtol=1e-10, atol=1e-14)
    for t, v in ((0, int(ids[0, 0])), (1, 3), (3, 29)):
        h = 1e-5
        up, dn = x.copy(), x.copy()
        up[t, v] += h
        dn[t, v] -= h
        d = (of.distill(up, ids, vals, T)[0] - of.distill(dn, ids, vals, T)[0]).sum() * w[t] / (2 * h)
        assert abs(d - grad[t, v]) < 1e-7


def test_backward_of_both_ends_matches_autograd():
    r = np.random.default_rng(5)
    V, H, M = 11, 64, 6
    E, g, b = r.standard_normal((V, H)), 1 + 0.1 * r.standard_normal(H), 0.1 * r.standard_normal(H)
    x, G = r.standard_normal((M, H)), r.standard_normal((M, V))
    h = _t(x, True)
    (torch.nn.functional.layer_norm(h, (H,), _t(g), _t(b), 1e-5) @ _t(E).T * _t(G)).sum().backward()
    assert np.allclose(of.lm_head_backward(x, G, E, g), h.grad.numpy(), rtol=1e-9, atol=1e-12)
    ids = np.array([3, 0, 3, -2, 15, 3])                 # two of them clamped
    dy = r.standard_normal((M, H))
    W = _t(E, True)
    (torch.nn.functional.layer_norm(W[torch.tensor(np.clip(ids, 0, V - 1))], (H,), _t(g), _t(b), 1e-5) * _t(dy)).sum().backward()
    tokens, rows = of.embed_backward(ids, dy, E, g)
    assert tokens.tolist() == [0, 3, 10]
    assert np.allclose(rows, W.grad.numpy()[tokens], rtol=1e-9, atol=1e-12)
