"""A training step of a GraphSAGE model whose targets have a head each for their type, with all operators that it takes: sampling, loading, the
model forward, targets sorted by type, the heads' products, a policy loss, its gradient through the heads and the model, orthogonalised
momentum for the matrices and AdamW for the biases.  Every operator is held to its float64 form on what it was given (its own file has
the tolerances), the whole step eager against captured and replayed, bit for bit."""
import numpy as np
import pytest
import torch

import row_loss_check as K
from oracle import grouped as O
from oracle import training as T

pytestmark = pytest.mark.gpu
F32 = torch.float32
U = K.U
TYPES, CLASSES = 5, 11


class Model:
    def __init__(self, w, ctx):
        from paper_2303_13775_amd import AdamwTensors, MuonTensors, SageParams
        gen = torch.Generator(device="cuda").manual_seed(3)
        r = lambda *s: torch.randn(s, device="cuda", generator=gen) * 0.1
        d = list(w.dims)
        self.ctx, self.dims, self.n = ctx, d, w.batch
        self.w_self, self.w_neigh = [[r(a, b) for a, b in zip(d, d[1:])] for _ in range(2)]
        self.bias = [r(b) for b in d[1:]]
        self.head, self.head_bias = r(TYPES, d[-1], CLASSES), r(TYPES, CLASSES)
        self.params = SageParams(d, self.w_self, self.w_neigh, self.bias)
        z = lambda ts: [torch.zeros_like(t) for t in ts]
        self.gw_self, self.gw_neigh, self.gbias = z(self.w_self), z(self.w_neigh), z(self.bias)
        self.g_head, self.g_head_bias = torch.zeros_like(self.head), torch.zeros_like(self.head_bias)
        matrices, grads = [*self.w_self, *self.w_neigh, self.head], [*self.gw_self, *self.gw_neigh, self.g_head]
        self.momenta = z(matrices)
        self.muon = MuonTensors(matrices, grads, self.momenta)
        vectors, vgrads = [*self.bias, self.head_bias], [*self.gbias, self.g_head_bias]
        self.m, self.v = z(vectors), z(vectors)
        self.adamw = AdamwTensors(vectors, vgrads, self.m, self.v)
        self.state = [*matrices, *self.momenta, *vectors, *self.m, *self.v]
        i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
        self.type, self.ptr, self.rows = i32(self.n), i32(TYPES + 1), i32(self.n)
        self.hidden, self.g_hidden = (torch.zeros((self.n, d[-1]), device="cuda") for _ in range(2))
        self.logits, self.g_logits = (torch.zeros((self.n, CLASSES), device="cuda") for _ in range(2))
        self.actions = torch.zeros(self.n, dtype=torch.int64, device="cuda")
        self.old, self.adv, self.loss = (torch.zeros(self.n, device="cuda") for _ in range(3))
        self.work = ctx.gsplit_grouped_linear_work(self.hidden, self.head)
        self.step_no, self.lr = torch.ones(1, dtype=torch.int64, device="cuda"), torch.full((1,), 0.02, device="cuda")

    def forward(self, feat):
        c = self.ctx
        c.gsplit_sage_fwd(self.params, feat, self.hidden)
        c.gsplit_group_rows(self.type, self.ptr, self.rows)
        self.logits.zero_()
        c.gsplit_grouped_linear_fwd(self.hidden, self.ptr, self.rows, self.head, self.head_bias, self.logits)

    def backward(self):
        c = self.ctx
        c.gsplit_policy_loss(self.logits, self.actions, self.old, self.adv, self.g_logits, row_loss=self.loss)
        self.g_hidden.zero_()           # (targets of no type have no gradient)
        c.gsplit_grouped_linear_bwd(self.hidden, self.ptr, self.rows, self.head, self.g_logits, self.g_hidden, self.g_head, self.g_head_bias, self.work)
        c.gsplit_sage_bwd(self.params, self.g_hidden, self.gw_self, self.gw_neigh, self.gbias)

    def update(self):
        self.ctx.gsplit_muon_step(self.muon, weight_decay=0.01, lr_dev=self.lr)
        self.ctx.gsplit_adamw_step(self.adamw, step_dev=self.step_no, lr_dev=self.lr)

    def step(self, feat):
        self.forward(feat)
        self.backward()
        self.update()


def _setup(seed=0):
    import workloads
    from paper_2303_13775_amd import Context
    w = workloads.tiny(device="cuda")
    ctx = Context(w.indptr, w.indices, w.pmap, w.n_splits, w.fanouts, w.batch)
    ctx.gsplit_sample_split(w.targets(seed).cuda(), 9, seed)
    n_local = ctx.gsplit_batch_sizes()[0]
    feat = torch.zeros((sum(n_local[0]), w.feat.shape[1]), device="cuda")
    ctx.gsplit_gather_features(w.feat, feat)
    m = Model(w, ctx)
    rng = np.random.default_rng(seed)
    m.type.copy_(torch.from_numpy(rng.integers(-1, TYPES, m.n).astype(np.int32)))
    m.actions.copy_(torch.from_numpy(rng.integers(0, CLASSES, m.n)))
    m.actions[m.type < 0] = -1
    m.old.copy_(torch.from_numpy(-np.log(CLASSES) + 0.3 * rng.standard_normal(m.n)))
    m.adv.copy_(torch.from_numpy(rng.standard_normal(m.n)))
    return w, ctx, m, feat


def _np(t):
    return t.double().cpu().numpy()


def test_every_operator_of_the_step():
    w, ctx, m, feat = _setup()
    m.forward(feat)
    p, r = O.group_rows(m.type.cpu().numpy(), TYPES)
    assert (m.ptr.cpu().numpy() == p).all() and (m.rows.cpu().numpy()[:len(r)] == r).all()
    y, size, used = O.linear(_np(m.hidden), p, r, _np(m.head), _np(m.head_bias))
    tol = lambda s, n: 4 * (np.sqrt(n / 16 + 64) + 2) * U * s
    K.check("logits", m.logits, np.where(used[:, None], y, 0.0), tol(size, m.dims[-1]))
    m.backward()
    want = T.policy_loss(_np(m.logits), m.actions.cpu().numpy(), _np(m.old), _np(m.adv))
    K.check("loss", m.loss, want["loss"], 200 * U * np.abs(want["loss"]) + 1e-7)
    (dx, dxs), (dw, dws), (db, dbs) = O.linear_grad(_np(m.hidden), p, r, _np(m.head), _np(m.g_logits))
    K.check("dx", m.g_hidden, dx, tol(dxs, CLASSES))
    K.check("dw", m.g_head, dw, tol(dws, int(np.diff(p).max())))
    K.check("db", m.g_head_bias, db, tol(dbs, int(np.diff(p).max())))
    # a head's weight moved: the loss follows its gradient.  The second difference of a step h is h^2 times the curvature, which cancels
    # between the two sides; what is left is the third, h^2 / 6 of it, and the rounding of the losses over 2 h
    h = 2.0 ** -7
    for at in ((1, 3, 2), (4, 0, 10)):
        sides = []
        for by in (h, -h):
            head = _np(m.head)
            head[at] += by
            z = np.where(used[:, None], O.linear(_np(m.hidden), p, r, head, _np(m.head_bias))[0], 0.0)
            sides.append(T.policy_loss(z, m.actions.cpu().numpy(), _np(m.old), _np(m.adv))["loss"].sum())
        assert abs((sides[0] - sides[1]) / (2 * h) - float(m.g_head[at])) < 1e-3 * float(m.g_head.abs().max()), at
    before = [t.clone() for t in m.state]
    m.update()
    n = len(m.momenta)
    for i, (old, new, mom, g) in enumerate(zip(before[:n], m.state[:n], m.momenta, [*m.gw_self, *m.gw_neigh, m.g_head])):
        old, new, mom, g = (_np(t).reshape(-1, *t.shape[-2:]) for t in (old, new, mom, g))
        scale = np.sqrt(max(1.0, old.shape[2] / old.shape[1]))
        for a, b, c, d in zip(old, new, mom, g):
            want, m1, o = T.muon(a, d, 0 * d, lr=float(np.float32(0.02)), momentum=0.95, nesterov=True, weight_decay=0.01, scale=scale, steps=5,
                                 coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7)
            assert np.abs(c - m1).max() <= 4 * U * np.abs(m1).max()
            # (its own file has the elements' tolerance: the steps raise a rounding of 2^-24 by 3.45^5 = 490 at most)
            assert np.abs(b - want).max() <= 0.02 * scale * 490 * 8 * U + 3 * U * np.abs(want).max(), i
    ctx.close()


def test_the_step_captured():
    w, ctx, m, feat = _setup()
    w2, ctx2, e, feat2 = _setup()
    assert torch.equal(feat, feat2)
    m.step(feat), e.step(feat2)         # (buffers that a first call allocates)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        m.step(feat)
    for k in range(2, 6):
        for x in (m, e):
            x.step_no.fill_(k)
            x.lr.fill_(0.02 / k)
            x.type.copy_(torch.roll(x.type, 7))
            x.actions.copy_(torch.where(x.type < 0, -1, torch.roll(x.actions, 3).clamp(min=0)))
        e.step(feat2)
        graph.replay()
        if k % 2:
            torch.cuda.synchronize()
        assert torch.equal(m.logits, e.logits) and torch.equal(m.loss, e.loss), k
        assert all(torch.equal(a, b) for a, b in zip(m.state, e.state)), k
    assert all(bool(t.isfinite().all()) for t in m.state)
    ctx.close()
    ctx2.close()
