"""GPU parity of the client's scoring and of its ends of a fine-tuning step (log probabilities, distillation loss, backward of LM
head and embedding lookup) against the definitions in fp64 (oracle/finetune.py), through the C ABI."""
import numpy as np
import pytest
import torch

from oracle import finetune as of
from paper_2209_01188_amd import binding
from tests.gpu_util import DEV, to_dev, to_np

pytestmark = pytest.mark.gpu
U32, U16 = 2.0 ** -24, 2.0 ** -11           # half a step of fp32 and fp16, relative


def _client(V, H, rows, seed=0, std=0.05):
    r = np.random.default_rng([seed, V, H])
    E = (r.standard_normal((V, H)) * std).astype(np.float16)
    vec = [(m + 0.1 * r.standard_normal(H)).astype(np.float16) for m in (1.0, 0.0, 1.0, 0.0)]
    return binding.Client(to_dev(E), *[to_dev(v) for v in vec], max_rows=rows), E, vec


def _logits(M, V, seed, spread=3.0):
    r = np.random.default_rng([seed, M, V])
    x = (r.standard_normal((M, V)) * spread).astype(np.float32)
    x[np.arange(M), r.integers(0, V, M)] += 8.0
    return r, x


def _shifted(a):
    """The same array on the GPU, beginning 4 bytes behind an aligned address."""
    flat = torch.empty(a.size + 1, dtype=torch.float32, device=DEV)
    v = flat[1:].view(a.shape)
    v.copy_(to_dev(a))
    return v


def _x_max(x, T):
    """Largest |t| log2(e) of a term that counts: beyond 150 a probability is 0 in fp32."""
    f = np.where(np.isfinite(x), x, np.nan)
    with np.errstate(all="ignore"):
        span = np.nan_to_num(np.nanmax(f, 1) - np.nanmin(f, 1))
    return np.minimum(span / T * 1.4427, 150.0)


def _rel(x, T):
    """Relative error of one exponential and thus of sums of them: three roundings of an exponent of up to x_max in base 2, each
    worth x_max * 2^-24 * ln 2, and the instruction's own 2^-23 (a whole step), twice."""
    return (3 * _x_max(x, T) + 4) * U32


def _check_logprobs(c, x, tokens, T, K, dev=None):
    lp, ent, top, tlp = c.logprobs(to_dev(x) if dev is None else dev, None if tokens is None else to_dev(tokens), T, K)
    with np.errstate(invalid="ignore"):
        rlp, rent, rtop, rtlp = of.logprobs(x, np.zeros(len(x), np.int64) if tokens is None else tokens, T, K)
    rel = _rel(x, T)

    def close(got, ref, tol, what):
        got = to_np(got).astype(np.float64)
        fine = np.isfinite(ref)
        assert np.array_equal(got[~fine], ref[~fine], equal_nan=True), what
        d = np.abs(got - np.where(fine, ref, 0.0))[fine]
        assert (d <= np.broadcast_to(tol, ref.shape)[fine]).all(), (what, d.max())
    if tokens is None:
        assert lp is None
    else:
        close(lp, rlp, U32 * np.abs(np.where(np.isfinite(rlp), rlp, 0)) + rel, "logprob")
    # log(1 + rest) and the sum of t e^t carry the terms' relative error; S itself is held in fp64
    close(ent, rent, 2 * (rel + 2 * U32) * np.abs(rent) + 1e-14, "entropy")
    if K:
        assert np.array_equal(to_np(top), rtop)
        close(tlp, rtlp, (U32 * np.abs(np.where(np.isfinite(rtlp), rtlp, 0)) + rel[:, None]), "top_logprob")
    else:
        assert top is None and tlp is None


@pytest.mark.parametrize("V,M,T,K", [(1, 1, 1.0, 1), (1, 3, 0.5, 0), (5, 2, 1.0, 5), (63, 4, 2.0, 20), (64, 1, 1.0, 64), (65, 3, 0.7, 64),
                                     (1023, 5, 1.0, 1), (1025, 2, 1.0, 3), (4099, 9, 0.8, 20), (16383, 2, 1.0, 64), (16385, 3, 4.0, 5),
                                     (50257, 12, 0.8, 20), (50257, 70, 1.0, 0), (20001, 300, 1.0, 33), (250880, 1, 1.0, 5),
                                     (250880, 3, 1.0, 64)])
def test_logprobs_match_the_definition(V, M, T, K):
    c, _, _ = _client(V, 64, M)
    r, x = _logits(M, V, 1)
    tokens = r.integers(0, V, M).astype(np.int32)
    tokens[::5] = x[::5].argmax(1)
    tokens[1::7] = -1
    tokens[2::7] = V
    _check_logprobs(c, x, tokens, T, K)
    _check_logprobs(c, x, None, T, K, dev=_shifted(x))
    c.close()


@pytest.mark.parametrize("V,M", [(7, 5), (3000, 5), (40000, 5), (250880, 5)])
def test_logprobs_of_ties_ruled_out_tokens_and_rows_without_a_distribution(V, M):
    c, _, _ = _client(V, 64, M)
    r, x = _logits(M, V, 2)
    K = min(V, 20)
    x[0] = 1.5                                             # all equal: the lowest tokens, in order
    x[1] = np.round(x[1])                                  # many equal ones
    x[2, V // 3:] = -np.inf                                # most tokens ruled out
    x[3] = -np.inf                                         # nothing left
    x[4, r.permutation(V)[:max(1, V - 3)]] = -np.inf       # three left, somewhere
    tokens = np.array([V - 1, 0, V - 1, 0, int(np.isfinite(x[4]).argmax())], np.int32)
    _check_logprobs(c, x, tokens, 1.0, K)
    # zeros of both signs are equal; the row falls steadily, then rises steadily
    x[0] = np.where(np.arange(V) % 2, -0.0, 0.0)
    x[1] = -np.arange(V) * 2.0 ** -12
    x[2] = np.arange(V) * 2.0 ** -12
    x[3, V // 2] = -3.0e38                                 # one token, however small
    _check_logprobs(c, x, tokens, 1.0, K)
    c.close()


def test_entropy_of_nearly_certain_rows_keeps_its_digits():
    V, M = 50257, 6
    c, _, _ = _client(V, 64, M)
    x = np.full((M, V), -60.0, np.float32)
    for t in range(M):
        x[t, 100 + t] = 6.0 * t - 30.0                     # entropies from log V down to 1e-13 and below
    _check_logprobs(c, x, np.arange(M, dtype=np.int32) + 100, 1.0, 2)
    c.close()


@pytest.mark.parametrize("what", [np.nan, np.inf])
def test_a_row_that_is_not_numbers_stays_by_itself(what):
    V, M = 5003, 3
    c, _, _ = _client(V, 64, M)
    _, x = _logits(M, V, 3)
    good = x.copy()
    x[1, 4000] = what
    tokens = np.array([5, 6, 7], np.int32)
    lp, ent, top, tlp = [to_np(a) for a in c.logprobs(to_dev(x), to_dev(tokens), 1.0, 10)]
    ref = [to_np(a) for a in c.logprobs(to_dev(good), to_dev(tokens), 1.0, 10)]
    for a, b in zip((lp, ent, top, tlp), ref):
        assert np.array_equal(a[[0, 2]], b[[0, 2]])
    assert np.isnan(lp[1]) and np.isnan(ent[1]) and np.isnan(tlp[1]).all() and ((top[1] >= 0) & (top[1] < V)).all()
    ids, vals = np.array([[5, 9]] * 3, np.int32), np.zeros((3, 2), np.float32)
    loss, grad = [to_np(a) for a in c.distill(to_dev(x), to_dev(ids), to_dev(vals))]
    rloss, rgrad = [to_np(a) for a in c.distill(to_dev(good), to_dev(ids), to_dev(vals))]
    assert np.isnan(loss[1]) and np.isnan(grad[1]).all()
    assert np.array_equal(loss[[0, 2]], rloss[[0, 2]]) and np.array_equal(grad[[0, 2]], rgrad[[0, 2]])
    c.close()


def _check_distill(c, x, ids, vals, T, w, dev=None, in_place=False):
    logits = to_dev(x) if dev is None else dev
    loss, grad = c.distill(logits, to_dev(ids), to_dev(vals), T, loss_grad=None if w is None else to_dev(w),
                           grad_out=logits if in_place else None)
    rloss, rgrad = of.distill(x, ids, vals, T, w)
    rel = _rel(x, T)
    fine = np.isfinite(rloss)
    got = to_np(loss).astype(np.float64)
    assert np.array_equal(got[~fine], rloss[~fine])
    tol = U32 * np.abs(rloss) + T * T * (rel + 1e-13)
    assert (np.abs(got - rloss)[fine] <= tol[fine]).all(), np.abs(got - rloss)[fine].max()
    # a column's q has the error of its own exponential and of the sum; the listed columns, whose q - p cancels, only the sum's
    q, _ = of.softmax_rows(x, T)
    scale = T * (np.ones(len(x)) if w is None else np.abs(w)).astype(np.float64)
    tol = (2 * rel + 2 * U32)[:, None] * scale[:, None] * q + U32 * np.abs(rgrad) + scale[:, None] * 2.0 ** -120
    d = np.abs(to_np(grad).astype(np.float64) - rgrad)
    assert (d <= tol).all(), (d - tol).max()
    return to_np(loss), to_np(grad)


@pytest.mark.parametrize("V,M,K,T", [(1, 2, 1, 1.0), (5, 3, 5, 2.0), (64, 2, 64, 1.0), (1000, 1, 1, 1.0), (1025, 3, 130, 0.5), (4099, 7, 17, 3.0),
                                     (16385, 2, 1024, 2.0), (50257, 20, 64, 2.0), (50257, 1, 1, 1.0), (50257, 300, 8, 1.0),
                                     (250880, 2, 128, 2.0), (250880, 1, 1, 1.0)])
def test_distillation_matches_the_definition(V, M, K, T):
    c, _, _ = _client(V, 64, M)
    r, x = _logits(M, V, 4)
    ids = np.stack([r.permutation(V)[:K] if K <= V else r.integers(0, V, K) for _ in range(M)]).astype(np.int32)
    vals = (r.standard_normal((M, K)) * 3).astype(np.float32)
    if K > 2:
        ids[0, K - 1] = ids[0, 0]                          # a token twice
        ids[-1, 1] = -1                                    # shorter lists
        ids[-1, 2] = V
        vals[0, 1] = -np.inf
    w = (r.random(M) + 0.5).astype(np.float32)
    loss, grad = _check_distill(c, x, ids, vals, T, w)
    dev = _shifted(x)
    loss2, grad2 = _check_distill(c, x, ids, vals, T, w, dev=dev, in_place=True)         # over the logits, 4-byte aligned
    assert np.array_equal(loss, loss2) and np.array_equal(grad, grad2)
    only, none = c.distill(to_dev(x), to_dev(ids), to_dev(vals), T, want_grad=False)
    assert none is None and np.array_equal(to_np(only), loss)
    _check_distill(c, x, ids, vals, T, None)
    c.close()


def test_distillation_of_rows_without_a_list_or_a_distribution_and_of_one_token_many_times():
    V, M, K = 3001, 7, 40
    c, _, _ = _client(V, 64, M)
    r, x = _logits(M, V, 5)
    ids = np.stack([r.permutation(V)[:K] for _ in range(M)]).astype(np.int32)
    vals = r.standard_normal((M, K)).astype(np.float32)
    ids[0] = -1                                            # not trained on
    vals[1] = -np.inf                                      # a list of nothing
    x[2] = -np.inf                                         # nothing to learn from
    x[3, ids[3, :5]] = -np.inf                             # the teacher wants what the student rules out
    x[4, V // 2:] = -np.inf
    ids[4] = np.arange(K)
    ids[5] = 77                                            # the same token K times
    ids[6, ::2] = ids[6, 1]
    w = np.array([1, 1, 1, 1, 0, -2.5, 1024.0], np.float32)
    _check_distill(c, x, ids, vals, 2.0, w)
    x[2, 7] = ids[0, 0] = 0
    _check_distill(c, x, ids, vals, 1.0, w)
    c.close()


def test_gradient_of_the_loss_against_differences_of_the_loss():
    """The kernel's own loss, in steps of a size at which the difference of two fp32 losses has 4 digits."""
    V, K, T, h = 300, 6, 2.0, 0.125
    c, _, _ = _client(V, 64, 2 * V)
    r, x = _logits(1, V, 6)
    ids, vals = r.permutation(V)[:K].astype(np.int32)[None], r.standard_normal((1, K)).astype(np.float32)
    _, grad = c.distill(to_dev(x), to_dev(ids), to_dev(vals), T)
    steps = np.concatenate([x + h * np.eye(V, dtype=np.float32), x - h * np.eye(V, dtype=np.float32)])
    loss, _ = c.distill(to_dev(steps), to_dev(np.repeat(ids, 2 * V, 0)), to_dev(np.repeat(vals, 2 * V, 0)), T, want_grad=False)
    loss = to_np(loss).astype(np.float64)
    diff = (loss[:V] - loss[V:]) / (2 * h)
    # truncation: h^2 / 6 times the third derivative, at most T^2 / T^3 * q < 1/2; rounding: two losses of up to 50 at 2^-24, and their rel
    tol = h * h / 6 * 0.5 + (2 * 50 * U32 + 2 * T * T * _rel(x, T).max()) / (2 * h)
    assert np.abs(diff - to_np(grad)[0]).max() <= tol
    c.close()


def _norm_error(err, x, gain, eps=1e-5):
    """What errors of at most err in dy can become behind the LayerNorm's derivative."""
    x = x.astype(np.float64)
    xc = x - x.mean(1, keepdims=True)
    inv = 1 / np.sqrt((xc ** 2).mean(1, keepdims=True) + eps)
    xh, e = xc * inv, err * np.abs(gain.astype(np.float64))
    return inv * (e + e.mean(1, keepdims=True) + np.abs(xh) * (e * np.abs(xh)).mean(1, keepdims=True))


def _check_head(c, E, gain, x, G, dev=None):
    got = to_np(c.lm_head_backward(to_dev(x), to_dev(G) if dev is None else dev)).astype(np.float64)
    ref = of.lm_head_backward(x, G, E, gain)
    M, V = G.shape
    mass = np.abs(G).astype(np.float64) @ np.abs(E).astype(np.float64)
    # G as one fp16 value (2^-11) or two (2^-22); values below 2^-29 of a section's largest are off by at most 2^-40 of that;
    # sums of V products in fp32, 32 at a time, and of the parts
    steps = (U16 if M > 64 else U16 ** 2) + (V / 32 + 40) * U32
    err = steps * mass + np.abs(G).max(1, keepdims=True) * 2.0 ** -40 * np.abs(E).astype(np.float64).sum(0)
    tol = _norm_error(err, x, gain) + 2 * U16 * np.abs(ref) + 2.0 ** -25 + 1e-6 * np.abs(ref).max(1, keepdims=True)
    # beyond 65520 an fp16 value is an infinity (whatever comes within the tolerance of that border may be one or not)
    over, may = np.abs(ref) - tol >= 65520.0, np.abs(ref) + tol >= 65520.0
    assert np.array_equal(got[over], np.sign(ref[over]) * np.inf)
    d = np.abs(got - ref)[~may]
    assert (d <= tol[~may]).all(), (d / tol[~may]).max()
    # and as a whole: independent roundings of G and of the result, each at most half a step
    fine = ~may.any(1)
    norm = np.linalg.norm(ref[fine])
    if norm > 2.0 ** -10 * np.sqrt(ref[fine].size):       # (in fp16's normal range)
        assert np.linalg.norm((got - ref)[fine]) <= 1.5 * U16 * norm
    return got


def _softmax_grad(r, M, V):
    _, x = _logits(M, V, int(r.integers(1 << 30)))
    q, _ = of.softmax_rows(x)
    q[np.arange(M), r.integers(0, V, M)] -= 1.0
    return q.astype(np.float32)


# V: below one k-tile, ends inside k-tiles and sections; one and several sections to a workgroup; H: below, across and beside
# the blocks' 256 columns; M: one row, all block sizes, full and ragged, both forms of the product
@pytest.mark.parametrize("V,H,M", [(1, 64, 1), (31, 64, 3), (33, 128, 16), (1000, 192, 17), (4095, 320, 33), (4097, 1024, 48), (5003, 1088, 64),
                                   (9001, 512, 65), (8192, 2560, 100), (12289, 256, 257), (5003, 4096, 300), (777, 14336, 5), (777, 16384, 70),
                                   (50257, 1024, 16), (30011, 2560, 351), (2000, 9024, 130),
                                   (21001, 14336, 3), (20011, 8192, 64), (21001, 8192, 300), (9999, 4096, 192), (3333, 1024, 600),
                                   (128, 64, 2500)])
def test_lm_head_backward_matches_the_definition(V, H, M):
    c, E, vec = _client(V, H, M, seed=7)
    r = np.random.default_rng([8, V, H])
    x = (r.standard_normal((M, H)) * 2).astype(np.float16)
    x[:, 3] = 40.0                                         # an outlier feature
    G = _softmax_grad(r, M, V)
    G[M // 2] = 0.0                                        # a position that is not trained on
    a = _check_head(c, E, vec[2], x, G)
    assert (a[M // 2] == 0).all()
    b = _check_head(c, E, vec[2], x, G, dev=_shifted(G))
    assert np.array_equal(a, b)
    c.close()


@pytest.mark.parametrize("M", [5, 80])
def test_lm_head_backward_of_gradients_of_any_size(M):
    """Sections of very different size in one row, rows of very different size in one call; zeros and denormals."""
    V, H = 12500, 8192                                     # (a workgroup's share of the vocabulary spans sections)
    c, E, vec = _client(V, H, M, seed=9)
    r = np.random.default_rng(10)
    x = r.standard_normal((M, H)).astype(np.float16)
    G = r.standard_normal((M, V)).astype(np.float32)
    G[0, :4096] *= 1e-20
    G[0, 9000:] *= 1e15
    G[1, 4096:8192] = 0.0
    G[2, 4096:] *= 1e-12
    G[3] = 1e-42
    G[4] *= 1e-6
    got = _check_head(c, E, vec[2], x, G)
    assert (got[3] == 0).all()
    c.close()


# runs of all lengths around the pieces of 32; one token everywhere, all different, ids that are clamped
@pytest.mark.parametrize("V,H,M,kind", [(10, 64, 1, "any"), (10, 64, 63, "same"), (10, 64, 64, "same"), (300, 128, 500, "any"), (50, 1024, 1000, "any"),
                                        (2000, 2560, 65, "different"), (7, 4096, 260, "any"), (16, 4096, 128, "prompt"), (5000, 192, 4096, "zipf"),
                                        (40, 8192, 130, "any"), (9, 14336, 97, "any"), (30, 16384, 40, "any"), (5000, 64, 3000, "same"),
                                        (4000, 64, 2100, "lengths")])
def test_embed_backward_matches_the_definition(V, H, M, kind):
    c, E, vec = _client(V, H, M, seed=11)
    r = np.random.default_rng([12, V, H, M])
    ids = {"any": lambda: r.integers(-2, V + 2, M), "same": lambda: np.full(M, V // 2), "different": lambda: r.permutation(V)[:M],
           "prompt": lambda: np.tile(np.arange(16), 8), "zipf": lambda: (r.random(M) ** 6 * V).astype(np.int64),
           "lengths": lambda: r.permutation(np.repeat(r.permutation(V)[:70], np.arange(70)))[:M]}[kind]().astype(np.int32)
    M = len(ids)
    dy = r.standard_normal((M, H)).astype(np.float16)
    out = (torch.full((M,), -7, dtype=torch.int32, device=DEV), torch.full((M, H), 77.0, device=DEV),
           torch.zeros(1, dtype=torch.int32, device=DEV))
    tokens, grads, count = [to_np(a) for a in c.embed_backward(to_dev(ids), to_dev(dy), out=out)]
    rtok, ref = of.embed_backward(ids, dy, E, vec[0])
    n = len(rtok)
    assert count[0] == n and np.array_equal(tokens[:n], rtok)
    assert (tokens[n:] == -7).all() and (grads[n:] == 77.0).all()          # left as they were
    clamped = np.clip(ids, 0, V - 1)
    place = np.searchsorted(rtok, clamped)
    mass, most = np.zeros((n, H)), np.bincount(place).max()
    np.add.at(mass, place, np.abs(dy.astype(np.float64)))
    # fp32 sums of up to `most` values, the gain's product, the rounding of the result (statistics and row sums in fp64)
    tol = _norm_error((most + 1) * U32 * mass, E[rtok], vec[0]) + U32 * np.abs(ref) + 1e-12 * np.abs(ref).max()
    d = np.abs(grads[:n] - ref)
    assert (d <= tol).all(), (d / tol).max()
    again = c.embed_backward(to_dev(ids), to_dev(dy))
    assert np.array_equal(to_np(again[1])[:n], grads[:n]) and to_np(again[2])[0] == n
    c.close()


def test_a_fine_tuning_step_runs_through_all_of_them():
    """embed -> span -> LM head -> loss -> LM head backward -> span backward -> embed backward, as prompt tuning would: the
    prompt vectors' gradient against that of the oracle's chain."""
    import oracle
    from oracle import backward as ob
    from paper_2209_01188_amd import synth
    from tests.gpu_util import build_pair
    from tests.test_gpu_backward import grad_close
    cfg = synth.scaled(synth.CONFIGS["C2"], n_blocks=2)
    H, B, T, V, P = cfg.hidden, 2, 6, 1500, 3
    osp, gsp, params = build_pair(cfg, n_blocks=2, max_rows=B * T)
    head, E, vec = _client(V, H, B * T, seed=13, std=0.02)
    prompts, PE, pvec = _client(P, H, B * T, seed=14, std=1.0)
    r = np.random.default_rng(15)
    ids = np.concatenate([np.concatenate([np.arange(P), r.integers(0, P, T - P)]) for _ in range(B)]).astype(np.int32)
    labels = r.integers(0, V, (B * T, 1)).astype(np.int32)
    labels[::4] = -1                                       # positions that are not trained on
    zeros = np.zeros((B * T, 1), np.float32)
    weight = np.full(B * T, 64.0, np.float32)              # a loss scale: the gradients stay in fp16's range
    # the GPU's chain
    x = prompts.embed(to_dev(ids))
    y, _ = gsp.backward(x.view(B, T, H), torch.zeros((B, T, H), dtype=torch.float16, device=DEV))
    y = y.view(B * T, H)
    _, logits = head.lm_head(y, want_logits=True)
    lp, _, _, _ = head.logprobs(logits, to_dev(labels[:, 0]))
    loss, dl = head.distill(logits, to_dev(labels), to_dev(zeros), loss_grad=to_dev(weight), grad_out=logits)
    dy = head.lm_head_backward(y, dl)
    _, dx = gsp.backward(x.view(B, T, H), dy.view(B, T, H), want_output=False)
    tokens, grads, count = prompts.embed_backward(to_dev(ids), dx.view(B * T, H))
    # the oracle's
    rx = oracle.embed(ids, PE, pvec[0], pvec[1])
    assert np.array_equal(to_np(x).view(np.uint16), rx.view(np.uint16))
    _, rlog = oracle.lm_head(to_np(y), E, vec[2], vec[3], want_logits=True)
    rloss, rdl = of.distill(rlog.astype(np.float32), labels, zeros, 1.0, weight)
    assert np.allclose(to_np(loss), rloss, rtol=1e-5, atol=1e-5) and np.allclose(-to_np(lp), rloss, rtol=1e-5, atol=1e-5)
    rdy = of.lm_head_backward(to_np(y), rdl, E, vec[2]).astype(np.float16)
    ry, rdx = ob.span_backward(osp, params, rx.reshape(B, T, H), rdy.reshape(B, T, H))
    assert np.array_equal(to_np(y).view(np.uint16), np.asarray(ry, np.float16).reshape(B * T, H).view(np.uint16))
    rtok, rgrads = of.embed_backward(ids, np.asarray(rdx, np.float16).reshape(B * T, H), PE, pvec[0])
    n = int(to_np(count)[0])
    assert np.array_equal(to_np(tokens)[:n], rtok) and np.abs(rgrads).max() > 1e-4
    grad_close(to_np(dy), rdy)
    grad_close(to_np(grads)[:n], rgrads, "prompt vectors")
    head.close(); prompts.close(); gsp.close(); osp.destroy()


def test_calls_captured_into_a_graph_replay_to_the_same_bits():
    V, H, M = 5003, 256, 70
    c, E, vec = _client(V, H, M, seed=16)
    r = np.random.default_rng(17)
    state = dict(x=to_dev(r.standard_normal((M, H)).astype(np.float16)), logits=to_dev(_logits(M, V, 18)[1]),
                 tokens=to_dev(r.integers(-1, V, M).astype(np.int32)), ids=to_dev(r.integers(-1, V, (M, 9)).astype(np.int32)),
                 vals=to_dev(r.standard_normal((M, 9)).astype(np.float32)))
    store = torch.empty(binding.petals_client_lm_head_backward_bytes(c.cfg, M), dtype=torch.uint8, device=DEV)

    def step():
        lp = c.logprobs(state["logits"], state["tokens"], 0.9, 7)
        loss, dl = c.distill(state["logits"], state["ids"], state["vals"], 2.0)
        dx = c.lm_head_backward(state["x"], dl, store=store)
        rows = c.embed_backward(state["tokens"], dx)
        return [*lp, loss, dl, dx, rows[0], rows[1], rows[2]]
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = step()
    for i in range(4):
        state["logits"].copy_(to_dev(_logits(M, V, 20 + i)[1]))
        state["tokens"].copy_(to_dev(r.integers(-1, V, M).astype(np.int32)))
        eager = [a.clone() for a in step()]
        n = int(eager[-1][0])
        torch.cuda.synchronize()
        for a in captured:
            a.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        for k, (a, b) in enumerate(zip(captured, eager)):
            a, b = (a[:n], b[:n]) if k in (7, 8) else (a, b)
            assert torch.equal(a, b), (i, k)
    c.close()


def test_calls_on_another_stream():
    V, H, M = 3000, 128, 20
    c, E, vec = _client(V, H, M, seed=19)
    r, x = _logits(M, V, 21)
    tokens = r.integers(0, V, M).astype(np.int32)
    s = torch.cuda.Stream()
    dx, dtok = to_dev(x), to_dev(tokens)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        lp = c.logprobs(dx, dtok)[0]
        loss, grad = c.distill(dx, dtok[:, None].contiguous(), torch.zeros((M, 1), device=DEV))
    s.synchronize()
    assert np.allclose(to_np(lp), of.logprobs(x, tokens)[0], rtol=1e-5, atol=1e-5)
    assert np.allclose(to_np(loss), -to_np(lp), rtol=1e-6, atol=1e-6)
    c.close()


def test_offsets_beyond_32_bits():
    """More than 2^32 logits: the rows at the end come out as the same rows do in a call of their own."""
    V, H, M, K = 250880, 64, 17200, 3                      # 4.3e9 logits, 17 GB; and more rows than one launch takes
    c, E, vec = _client(V, H, M, seed=21)
    r = np.random.default_rng(22)
    base = to_dev((r.standard_normal((1 << 20) + 7)).astype(np.float32) * 3)
    x = torch.empty((M, V), device=DEV)
    flat, n = x.view(-1), base.numel()                     # (a period prime to V: no two rows alike)
    whole = flat.numel() // n * n
    flat[:whole].view(-1, n).copy_(base)
    flat[whole:] = base[:flat.numel() - whole]
    rows = [0, 1, 16383, 16384, 17119, 17198, 17199]       # 2^32 logits end in row 17119
    own = x[rows].contiguous()
    tokens = r.integers(0, V, M).astype(np.int32)
    lp, ent, top, tlp = c.logprobs(x, to_dev(tokens), 1.0, 5)
    rlp, rent, rtop, rtlp = of.logprobs(to_np(own), tokens[rows], 1.0, 5)
    rel = _rel(to_np(own), 1.0)
    assert np.array_equal(to_np(top)[rows], rtop)
    assert (np.abs(to_np(lp)[rows] - rlp) <= U32 * np.abs(rlp) + rel).all()
    assert (np.abs(to_np(ent)[rows] - rent) <= 2 * (rel + 2 * U32) * rent).all()

    ids = r.integers(0, V, (M, K)).astype(np.int32)
    vals = r.standard_normal((M, K)).astype(np.float32)
    loss, grad = c.distill(x, to_dev(ids), to_dev(vals), grad_out=x)          # in place
    want_loss, want = c.distill(own, to_dev(ids[rows]), to_dev(vals[rows]))
    mine = grad[rows].contiguous()
    # (a row is cut into other parts in a call of few rows: the same sums in fp64, of exponentials about other maxima)
    assert (np.abs(to_np(loss)[rows] - to_np(want_loss)) <= (2 * rel + 2 * U32) * np.abs(to_np(want_loss)) + 2 * rel).all()
    assert (np.abs(to_np(mine) - to_np(want)) <= 2 * (rel[:, None] + U32) * np.abs(to_np(want)) + 2.0 ** -126).all()

    hid = r.standard_normal((M, H)).astype(np.float16)
    out = to_np(c.lm_head_backward(to_dev(hid), grad))
    G = to_np(mine)
    ref = of.lm_head_backward(hid[rows], G, E, vec[2])
    mass = np.abs(G).astype(np.float64) @ np.abs(E).astype(np.float64)
    err = (U16 + (V / 32 + 40) * U32) * mass + np.abs(G).max(1, keepdims=True) * 2.0 ** -40 * np.abs(E).astype(np.float64).sum(0)
    tol = _norm_error(err, hid[rows], vec[2]) + 2 * U16 * np.abs(ref) + 2.0 ** -25 + 1e-6 * np.abs(ref).max(1, keepdims=True)
    assert (np.abs(out[rows].astype(np.float64) - ref) <= tol).all()
    c.close()


def test_the_most_rows_of_the_backward_calls():
    """2^20 rows: 65536 token tiles of the head, tokens with long and short lists."""
    V, H, M = 40, 64, 1 << 20
    c, E, vec = _client(V, H, M, seed=23)
    r = np.random.default_rng(24)
    G = r.standard_normal((M, V)).astype(np.float32)
    hid = r.standard_normal((M, H)).astype(np.float16)
    out = to_np(c.lm_head_backward(to_dev(hid), to_dev(G))).astype(np.float64)
    ref = of.lm_head_backward(hid, G, E, vec[2])
    mass = np.abs(G).astype(np.float64) @ np.abs(E).astype(np.float64)
    tol = _norm_error((U16 + 42 * U32) * mass + 2.0 ** -36, hid, vec[2]) + 2 * U16 * np.abs(ref) + 2.0 ** -25
    assert (np.abs(out - ref) <= tol).all()

    ids = np.minimum((r.random(M) ** 4 * V).astype(np.int32), V - 3)          # the last token: once; the one before: never
    ids[12345] = V - 1
    dy = r.integers(-8, 9, (M, H)).astype(np.float16)                         # sums below 2^24 are exact in fp32
    tokens, grads, count = [to_np(a) for a in c.embed_backward(to_dev(ids), to_dev(dy))]
    rtok, ref = of.embed_backward(ids, dy, E, vec[0])
    n = len(rtok)
    assert count[0] == n and np.array_equal(tokens[:n], rtok)
    mass = np.abs(np.stack([np.bincount(ids, dy[:, j].astype(np.float64), V) for j in range(H)], 1))[rtok]
    tol = _norm_error(2 * U32 * mass, E[rtok], vec[0]) + U32 * np.abs(ref) + 1e-12 * np.abs(ref).max()
    assert (np.abs(grads[:n] - ref) <= tol).all()
    c.close()


# the border of the calls that go in one launch (128 positions, 2^19 values), a position's first and last appearance across waves
@pytest.mark.parametrize("H,M", [(64, 127), (64, 128), (64, 129), (1088, 128), (2048, 100), (2112, 128), (4096, 128), (4160, 126), (8192, 64), (8256, 63),
                                 (16384, 32), (16384, 33), (14336, 36), (14336, 37)])
@pytest.mark.parametrize("kind", ["one", "turn", "reverse", "pairs", "outside"])
def test_embed_backward_around_the_smallest_calls(H, M, kind):
    V = 300
    c, E, vec = _client(V, H, M, seed=25)
    r = np.random.default_rng([26, H, M])
    ids = {"one": np.full(M, 7), "turn": np.arange(M) % 16, "reverse": np.arange(M)[::-1], "pairs": np.arange(M) // 2 * 3 % 64,
           "outside": r.integers(-3, 3, M) * 200}[kind].astype(np.int32)
    dy = r.standard_normal((M, H)).astype(np.float16)
    out = (torch.full((M,), -7, dtype=torch.int32, device=DEV), torch.full((M, H), 77.0, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV))
    tokens, grads, count = [to_np(a) for a in c.embed_backward(to_dev(ids), to_dev(dy), out=out)]
    rtok, ref = of.embed_backward(ids, dy, E, vec[0])
    n = len(rtok)
    assert count[0] == n and np.array_equal(tokens[:n], rtok)
    assert (tokens[n:] == -7).all() and (grads[n:] == 77.0).all()
    place = np.searchsorted(rtok, np.clip(ids, 0, V - 1))
    mass = np.zeros((n, H))
    np.add.at(mass, place, np.abs(dy.astype(np.float64)))
    tol = _norm_error((np.bincount(place).max() + 1) * U32 * mass, E[rtok], vec[0]) + U32 * np.abs(ref) + 1e-12 * np.abs(ref).max()
    assert (np.abs(grads[:n] - ref) <= tol).all()
    c.close()


# lists of up to 64 keys: rising logits (every key enters), falling ones, many equal, infinities below, at every size of a join
@pytest.mark.parametrize("V,M", [(64, 3), (100, 2), (4096, 2), (4097, 2), (20000, 3), (70000, 1100), (250880, 2)])
@pytest.mark.parametrize("K", [1, 2, 17, 63, 64])
def test_the_best_of_rows_in_any_order(V, M, K):
    c, _, _ = _client(V, 64, M, seed=27)
    r = np.random.default_rng([28, V, M])
    x = r.standard_normal((M, V)).astype(np.float32)
    x[0] = np.arange(V, dtype=np.float32) / V                     # the best come last
    x[1] = -np.arange(V, dtype=np.float32) / V
    if M > 2:
        x[2] = r.integers(0, 3, V)
    x[-1, r.permutation(V)[:V - V // 3 - 30]] = -np.inf
    some = [0, 1, min(2, M - 1), M // 2, M - 1]
    top = to_np(c.logprobs(to_dev(x), None, 1.0, K)[2])[some]
    assert np.array_equal(top, np.argsort(-x[some].astype(np.float64), axis=1, kind="stable")[:, :K])
    c.close()


# blocks of 128, 160, 192 and 256 tokens, with one or several to a call, full and ragged
@pytest.mark.parametrize("V,H,M", [(6007, 2112, 127), (6007, 2112, 129), (6007, 2112, 385), (30011, 2560, 129), (30011, 2560, 160), (20011, 4096, 257),
                                   (8009, 14336, 161), (8009, 14336, 192), (777, 8192, 2000), (777, 16384, 1000), (777, 16384, 1024)])
def test_lm_head_backward_at_the_blocks_of_tokens(V, H, M):
    c, E, vec = _client(V, H, M, seed=29)
    r = np.random.default_rng([30, M])
    x = r.standard_normal((M, H)).astype(np.float16)
    _check_head(c, E, vec[2], x, _softmax_grad(r, M, V))
    c.close()


# rows that one workgroup takes as a whole: the number of rows from which on it does, both widths of workgroup, vocabularies beside them
@pytest.mark.parametrize("V,M,K,T", [(1, 192, 1, 1.0), (7, 200, 7, 2.0), (100, 139, 100, 1.0), (300, 140, 1024, 2.0), (1000, 193, 130, 0.5),
                                     (8193, 256, 1024, 1.0), (65536, 192, 64, 2.0), (65537, 141, 64, 2.0), (100003, 194, 1, 1.0),
                                     (20011, 139, 1024, 1.0)])
def test_distillation_by_whole_rows(V, M, K, T):
    c, _, _ = _client(V, 64, M)
    r, x = _logits(M, V, 31)
    ids = r.integers(-1, V, (M, K)).astype(np.int32)
    vals = (r.standard_normal((M, K)) * 3).astype(np.float32)
    ids[1], vals[2], x[3] = -1, -np.inf, -np.inf           # no list, a list of nothing, no distribution
    if V > 1:
        ids[3, 0] = 0
        x[4, V // 2:] = -np.inf
        ids[4] = 0
    w = (r.random(M) + 0.5).astype(np.float32)
    loss, grad = _check_distill(c, x, ids, vals, T, w)
    loss2, grad2 = _check_distill(c, x, ids, vals, T, w, dev=_shifted(x), in_place=True)
    assert np.array_equal(loss, loss2) and np.array_equal(grad, grad2)
    only, none = c.distill(to_dev(x), to_dev(ids), to_dev(vals), T, w if w is None else to_dev(w), want_grad=False)
    assert none is None and np.array_equal(to_np(only), loss)
    c.close()


@pytest.mark.parametrize("M", [3, 40, 150, 300, 1000])
def test_a_first_call_inside_a_capture(M):
    """No call before it that could have prepared something; eager work between the replays."""
    V, H = 2003, 4160
    c, E, vec = _client(V, H, M, seed=32)
    r, x = _logits(M, V, 33)
    logits, hid = to_dev(x), to_dev(r.standard_normal((M, H)).astype(np.float16))
    ids, vals = to_dev(r.integers(0, V, (M, 4)).astype(np.int32)), to_dev(r.standard_normal((M, 4)).astype(np.float32))
    tokens = to_dev(r.integers(0, V, M).astype(np.int32))
    store = torch.empty(binding.petals_client_lm_head_backward_bytes(c.cfg, M), dtype=torch.uint8, device=DEV)

    def step():
        out = list(c.logprobs(logits, tokens, 1.0, 50)) + list(c.distill(logits, ids, vals, 2.0))
        out.append(c.lm_head_backward(hid, out[-1], store=store))
        return out + list(c.embed_backward(tokens, out[-1]))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = step()
    for i in range(3):
        for a in captured:
            a.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        eager = step()
        n = int(eager[-1][0])
        for k, (a, b) in enumerate(zip(captured, eager)):
            a, b = (a[:n], b[:n]) if k in (7, 8) else (a, b)
            assert torch.equal(a, b), (i, k)
        logits.mul_(0.9)
        tokens.copy_(tokens.flip(0))
    c.close()


def test_two_clients_on_two_streams_at_once():
    V, H, M = 20011, 1024, 150
    calls = []
    for seed in (34, 35):
        c, E, vec = _client(V, H, M, seed=seed)
        r, x = _logits(M, V, seed)
        state = (to_dev(x), to_dev(r.integers(0, V, M).astype(np.int32)), to_dev(r.standard_normal((M, 1)).astype(np.float32)),
                 to_dev(r.standard_normal((M, H)).astype(np.float16)), to_dev(r.integers(0, 90, M).astype(np.int32)))

        def step(c=c, s=state):
            lp = c.logprobs(s[0], s[1], 1.0, 20)
            loss, dl = c.distill(s[0], s[1][:, None], s[2])
            dx = c.lm_head_backward(s[3], dl)
            return [*lp, loss, dl, dx, *c.embed_backward(s[4], dx)]
        calls.append((c, step, torch.cuda.Stream()))
    alone = [step() for _, step, _ in calls]
    torch.cuda.synchronize()
    for _ in range(5):
        both = []
        for _, step, s in calls:
            with torch.cuda.stream(s):
                both.append(step())
        torch.cuda.synchronize()
        for a, b in zip(alone, both):
            n = int(a[-1][0])
            for k, (u, v) in enumerate(zip(a, b)):
                u, v = (u[:n], v[:n]) if k in (7, 8) else (u, v)
                assert torch.equal(u, v), k
    for c, _, _ in calls:
        c.close()


@pytest.mark.parametrize("V,M", [(300, 6), (50257, 6), (20011, 200)])
@pytest.mark.parametrize("T", [1.0, 3.0])
def test_masks_of_the_lowest_value(V, M, T):
    """Tokens ruled out with the type's lowest number instead of an infinity, in logits and in teachers' lists."""
    lowest = float(np.finfo(np.float32).min)
    c, _, _ = _client(V, 64, M)
    r, x = _logits(M, V, 36)
    x[0] = lowest                                          # every one: all equal
    x[1, 1:] = lowest                                      # all but the first
    x[2, :V - 1] = lowest                                  # all but the last
    x[3, r.random(V) < 0.9] = lowest
    x[4, :V // 2] = lowest
    tokens = np.full(M, V - 1, np.int32)
    tokens[1], tokens[3] = 0, int(x[3].argmax())
    _check_logprobs(c, x, tokens, T, 5)
    ids = np.stack([r.permutation(np.flatnonzero(x[t] > lowest) if t else V)[:1].repeat(4) for t in range(M)]).astype(np.int32)
    ids[5:] = r.integers(0, V, (M - 5, 4))
    vals = r.standard_normal((M, 4)).astype(np.float32)
    vals[:, 1] = lowest
    vals[3] = lowest                                       # (a list of equal logits)
    _check_distill(c, x, ids, vals, T, None)
    c.close()
