"""The float64 checker of the drafter's calls, pinned by closed forms, brute force, autograd and differences (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import drafter_oracle as orc


def rows(seed, T, V, sigma=2.0):
    return np.random.default_rng(seed).normal(0, sigma, size=(T, V))


def lists(seed, T, V, K, tail=True):
    rng = np.random.default_rng([seed, 1])
    index = np.stack([rng.permutation(V)[:K] for _ in range(T)])
    p = rng.dirichlet(np.ones(K + 1), size=T)[:, :K]
    return index, np.log(p)


def test_top_by_sorting_pairs():
    z = np.round(rows(0, 6, 40), 1)            # ties
    z[2, 5:] = -np.inf                          # fewer unmasked logits than K
    z[3] = -np.inf
    z[4, 3] = -3e38
    index, lp, lse = orc.top(z, 40, 8)
    for t in range(6):
        want = [j for _, j in sorted((-v, j) for j, v in enumerate(z[t]) if v > -1e30)][:8]
        assert index[t].tolist() == want + [-1] * (8 - len(want))
        assert np.isneginf(lp[t, len(want):]).all()
    assert np.isneginf(lse[3]) and not np.isneginf(lse[4])
    assert np.allclose(np.exp(orc.top(z[:1], 40, 40)[1]).sum(), 1.0)


@pytest.mark.parametrize("tail", [0, 1])
def test_distill_is_the_autograd_of_its_definition(tail):
    T, V, K = 5, 23, 6
    z, (index, lp) = rows(1, T, V), lists(1, T, V, K)
    w = np.array([0.5, 0.0, 1.0, 2.0, -0.25])
    got = orc.distill(z, V, index, lp, w, tail, 3.0)
    x = torch.tensor(z, requires_grad=True)
    q = torch.softmax(x, 1)
    p, i = torch.exp(torch.tensor(lp)), torch.tensor(index)
    qi = q.gather(1, i)
    if tail:
        pr = 1 - p.sum(1)
        qr = q.sum(1) - qi.sum(1)
        L = (p * (p.log() - qi.log())).sum(1) + pr * (pr.log() - qr.log())
    else:
        p = p / p.sum(1, keepdim=True)
        L = (p * (p.log() - qi.log())).sum(1)
    loss = (torch.tensor(w) * L).sum()
    loss.backward()
    assert np.allclose(got["row_loss"][w != 0], L.detach().numpy()[w != 0], rtol=1e-12)
    assert np.isclose(got["loss"], loss.item(), rtol=1e-12)
    assert np.allclose(got["dlogits"], 3.0 * x.grad.numpy(), rtol=1e-9, atol=1e-12)
    assert np.abs(got["dlogits"].sum(1)).max() < 1e-12      # a shift of a row's logits changes nothing


@pytest.mark.parametrize("tail", [0, 1])
def test_distill_gradient_by_differences(tail):
    V, K, h = 11, 4, 1e-5
    z, (index, lp) = rows(2, 1, V), lists(2, 1, V, K)
    d = orc.distill(z, V, index, lp, [1.0], tail, 1.0)["dlogits"][0]
    for j in range(V):
        up, dn = z.copy(), z.copy()
        up[0, j] += h
        dn[0, j] -= h
        f = [orc.distill(x, V, index, lp, [1.0], tail, 1.0)["loss"] for x in (up, dn)]
        assert abs((f[0] - f[1]) / (2 * h) - d[j]) < 1e-8


def test_distill_of_itself_vanishes_and_edges():
    z = rows(3, 1, 30)
    index, lp, _ = orc.top(z, 30, 9)
    out = orc.distill(z, 30, index, lp, [1.0], 1, 1.0)
    assert abs(out["row_loss"][0]) < 1e-12 and np.abs(out["dlogits"]).max() < 1e-12
    out = orc.distill(z, 30, index, lp, [1.0], 0, 1.0)      # renormalised: minus the log of the list's mass
    assert np.isclose(out["row_loss"][0], -np.log(np.exp(lp).sum()))
    absent = np.full_like(index, -1)
    assert orc.distill(z, 30, absent, lp, [1.0], 1, 1.0)["loss"] == 0.0
    twice = index.copy()
    twice[0, 1] = twice[0, 0]
    assert orc.distill(z, 30, twice, lp, [1.0], 1, 1.0)["bad"][0]
    z[0, index[0, 0]] = -np.inf                              # teacher probability on a masked logit
    out = orc.distill(z, 30, index, lp, [1.0], 1, 1.0)
    assert np.isposinf(out["row_loss"][0]) and np.isfinite(out["dlogits"]).all()


@pytest.mark.parametrize("probs", [True, False])
def test_verification_draws_from_the_policy(probs):
    """Over many random numbers the first token out is distributed as the policy's first row, whatever the drafter."""
    V, N = 4, 40000
    rng = np.random.default_rng(5)
    zt, zd = rng.normal(size=(1, 2, V)), rng.normal(size=(1, 1, V))
    p = np.exp(orc.log_softmax(zt[0, 0]))
    q = np.exp(orc.log_softmax(zd[0, 0])) if probs else None
    drafted = rng.choice(V, size=N, p=q) if probs else np.full(N, 2)
    u, e = rng.random(N), rng.exponential(size=(N, V))
    first = np.zeros(V)
    for k in range(N // 8):
        out = orc.verify(zt, zd if probs else None, V, [[drafted[k]]], None, [[u[k]]], [e[k]])
        first[out["tokens"][0, 0]] += 1
    n = N // 8
    assert (np.abs(first / n - p) < 4.5 * np.sqrt(p * (1 - p) / n)).all()


def test_verification_edges():
    V = 6
    z = rows(7, 3, V)[None]
    e = np.random.default_rng(8).exponential(size=(1, V))
    same = orc.verify(z, z[:, :2], V, [[1, 4]], None, [[0.999, 0.999]], e)     # p = q: always accepted
    assert same["accepted"][0] == 2 and same["tokens"][0, :2].tolist() == [1, 4]
    none = orc.verify(z, z[:, :2], V, [[1, 4]], [0], [[0.0, 0.0]], e)
    assert none["accepted"][0] == 0 and none["tokens"][0, 1:].tolist() == [-1, -1]
    assert none["tokens"][0, 0] == np.argmax(np.exp(orc.log_softmax(z[0, 0])) / e[0])
    idle = orc.verify(z, z[:, :2], V, [[1, 4]], [-1], [[0.0, 0.0]], e)
    assert (idle["tokens"] == -1).all()
    cut = orc.verify(z, z[:, :2], V, [[1, 9]], None, [[0.0, 0.0]], e)
    assert cut["accepted"][0] == 1 and cut["tokens"][0, 2] == -1
    copied = orc.verify(z, None, V, [[1, 4]], None, [[1.0 - 1e-9, 0.0]], e)
    assert copied["accepted"][0] == 0 and copied["tokens"][0, 0] != 1
    z[0, 0] = -np.inf
    empty = orc.verify(z, None, V, [[1, 4]], None, [[0.0, 0.0]], e)
    assert empty["accepted"][0] == 0 and (empty["tokens"] == -1).all()


def test_embedding_gradient_is_the_adjoint():
    rng = np.random.default_rng(9)
    V, H, T = 7, 5, 20
    ids = rng.integers(-1, V + 1, size=T)
    table, dout = rng.normal(size=(V, H)), rng.normal(size=(T, H))
    out = orc.embedding(table, ids, 1.5)
    d, mag = orc.embedding_grad(dout, ids, V, 1.5)
    assert np.isclose((out * dout).sum(), (table * d).sum())
    assert (mag >= np.abs(d) - 1e-12).all() and not out[(ids < 0) | (ids >= V)].any()
