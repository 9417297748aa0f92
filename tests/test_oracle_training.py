"""The plain forms of the losses and the update (oracle/training.py): gradients against differences, and
the update and the losses against torch's own where torch has them."""
import numpy as np
import pytest
import torch

from oracle import training as T


def _difference(f, z, h=1e-6):
    g = np.zeros_like(z)
    for i in np.ndindex(*z.shape):
        up, down = z.copy(), z.copy()
        up[i] += h
        down[i] -= h
        g[i] = (f(up) - f(down)) / (2 * h)
    return g


@pytest.mark.parametrize("kl", [0.0, 0.3])
def test_policy_gradient_is_the_difference_of_the_loss(kl):
    rng = np.random.default_rng(3)
    n, C = 7, 5
    z = rng.normal(size=(n, C))
    a = rng.integers(0, C, n)
    a[2] = -1
    adv, w = rng.normal(size=n), rng.random(n)
    w[4] = 0.0
    logp = np.array([T.row_distribution(z[r])[0][max(0, a[r])] for r in range(n)])
    old = logp + rng.normal(size=n) * 0.5           # ratios on both sides of both borders
    kw = dict(ref_logp=logp + rng.normal(size=n) if kl else None, weight=w, clip_low=0.2, clip_high=0.3, kl_coef=kl)
    got = T.policy_loss(z, a, old, adv, **kw)
    want = _difference(lambda y: T.policy_loss(y, a, old, adv, **kw)["loss"].sum(), z)
    assert np.max(np.abs(got["grad"] - want)) < 1e-7 * max(1.0, np.max(np.abs(want))) * 10
    assert not got["grad"][[2, 4]].any() and np.any(got["slope"] == 0.0)


def test_preference_gradient_is_the_difference_of_the_loss():
    rng = np.random.default_rng(4)
    ptr = np.array([1, 3, 3, 4, 8])                 # an empty sequence, rows in front of and behind the sequences
    n, C = 9, 4
    z = rng.normal(size=(n, C))
    a = rng.integers(0, C, n)
    a[5] = C
    kw = dict(ref_logp=rng.normal(size=4), weight=np.array([0.4, 1.3]), beta=0.7, smoothing=0.1)
    got = T.preference_loss(z, a, ptr, **kw)
    want = _difference(lambda y: T.preference_loss(y, a, ptr, **kw)["loss"].sum(), z)
    assert np.max(np.abs(got["grad"] - want)) < 1e-8
    assert not got["grad"][[0, 5, 8]].any() and got["grad"][[1, 2, 4]].any()


def test_update_against_torch():
    rng = np.random.default_rng(5)
    p0 = [rng.normal(size=n) for n in (7, 3)]
    ps = [torch.nn.Parameter(torch.tensor(p)) for p in p0]
    opt = torch.optim.AdamW(ps, lr=3e-3, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    p, m, v = [x.copy() for x in p0], [np.zeros_like(x) for x in p0], [np.zeros_like(x) for x in p0]
    for step in range(1, 5):
        g = [rng.normal(size=x.size) for x in p0]
        for q, x in zip(ps, g):
            q.grad = torch.tensor(x)
        norm = float(torch.nn.utils.clip_grad_norm_(ps, 1.0))
        opt.step()
        mine = T.grad_norm(g)
        assert abs(mine - norm) < 1e-12 * norm
        for k in range(2):
            p[k], m[k], v[k] = T.adamw(p[k], g[k], m[k], v[k], lr=3e-3, beta1=0.8, beta2=0.95, eps=1e-6, weight_decay=0.1,
                                       step=step, factor=T.clip_factor(mine, 1.0))
    for q, x in zip(ps, p):     # (torch divides by the norm plus 1e-6)
        assert np.max(np.abs(q.detach().numpy() - x)) < 1e-7


def test_losses_against_torch():
    rng = np.random.default_rng(6)
    z = rng.normal(size=(6, 5))
    a = rng.integers(0, 5, 6)
    logp = torch.log_softmax(torch.tensor(z), 1)[torch.arange(6), torch.tensor(a)].numpy()
    got = T.policy_loss(z, a, logp, np.ones(6))
    assert np.allclose(got["loss"], -1 / 6) and np.allclose(got["logp"], logp)
    got = T.preference_loss(z, a, np.arange(7), beta=2.0)
    want = -torch.nn.functional.logsigmoid(2.0 * torch.tensor(logp[0::2] - logp[1::2])).numpy() / 3
    assert np.allclose(got["loss"], want)
