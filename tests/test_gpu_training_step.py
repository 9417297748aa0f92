"""Whole training steps: sampling, loading, GraphSAGE, a loss over actions or over pairs, the backward pass, the clipped update, several
times over.  Every stage is held to its float64 form on what the stage before it left on the device."""
import numpy as np
import pytest
import torch

import workloads
from oracle import reference as R, training as T
from test_gpu_parity import TOL_F32

pytestmark = pytest.mark.gpu

STEP = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.01)


class _Trainer:
    def __init__(self, loss):
        from paper_2303_13775_amd import AdamwTensors, Context, SageParams
        self.w = w = workloads.custom(3000, 40000, dims=[32, 48, 8], fanouts=[6, 4], batch=200, n_splits=4, name="training")
        self.loss = loss
        dev = self.dev = torch.device("cuda:0")
        self.ctx = Context(w.indptr.to(dev), w.indices.to(dev), w.pmap.to(dev), w.n_splits, w.fanouts, w.batch)
        self.feat = w.feat.to(dev)
        self.weights = [[t.to(dev).clone() for t in lst] for lst in (w.w_self, w.w_neigh, w.bias)]
        self.params = SageParams(w.dims, *self.weights)
        self.grads = [[torch.zeros_like(t) for t in lst] for lst in self.weights]
        flat = [t for lst in self.weights for t in lst]
        self.m, self.v = ([torch.zeros_like(t) for t in flat] for _ in range(2))
        self.flat, self.gflat = flat, [t for lst in self.grads for t in lst]
        self.table = AdamwTensors(flat, self.gflat, self.m, self.v)
        self.x0 = torch.zeros((self.ctx.gsplit_max_rows(0), w.dims[0]), device=dev)
        n = w.batch
        self.logits, self.glog = (torch.zeros((n, w.dims[-1]), device=dev) for _ in range(2))
        self.norm = torch.zeros(1, device=dev)
        self.targets = torch.zeros(n, dtype=torch.int32, device=dev)
        self.seed_iter = torch.zeros(2, dtype=torch.int64, device=dev)
        self.step_dev = torch.zeros(1, dtype=torch.int64, device=dev)
        rng = np.random.default_rng(5)
        self.actions = torch.from_numpy(rng.integers(0, w.dims[-1], n)).to(dev)
        self.old = torch.from_numpy((-2 - rng.random(n)).astype(np.float32)).to(dev)
        self.adv = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).to(dev)
        self.ptr = torch.arange(0, n + 1, 5, device=dev)           # 20 pairs of sequences of five targets
        self.work = torch.zeros((n, 4), device=dev)

    def step(self, captured=False):
        c = self.ctx
        if captured:
            c.gsplit_sample_split_dev(self.targets, self.seed_iter)
        else:
            c.gsplit_sample_split(self.targets, 77, int(self.seed_iter[1]))
        c.gsplit_gather_features(self.feat, self.x0)
        c.gsplit_sage_fwd(self.params, self.x0, self.logits)
        if self.loss == "policy":
            c.gsplit_policy_loss(self.logits, self.actions, self.old, self.adv, self.glog, ref_logp=self.old, kl_coef=0.1)
        else:
            c.gsplit_preference_loss(self.logits, self.actions, self.ptr, self.glog, self.work, beta=0.5)
        c.gsplit_sage_bwd(self.params, self.glog, *self.grads)
        c.gsplit_adamw_step(self.table, step_dev=self.step_dev, max_norm=0.05, norm=self.norm, **STEP)

    def at(self, k):
        self.targets.copy_(self.w.targets(k).to(self.dev))
        self.seed_iter.copy_(torch.tensor([77, k]))
        self.step_dev.fill_(k + 1)


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_every_stage_of_three_steps(loss):
    t = _Trainer(loss)
    w = t.w
    for k in range(3):
        t.at(k)
        before = [[x.double().cpu().numpy() for x in lst] for lst in (t.flat, t.m, t.v)]
        op = R.SageParams(*[[x.double().cpu().numpy() for x in lst] for lst in t.weights])
        t.step()
        torch.cuda.synchronize()
        ob = R.sp_sample(w.indptr.numpy(), w.indices.numpy(), w.pmap.numpy(), w.n_splits, w.fanouts, t.targets.cpu().numpy(), 77, k)
        of = R.sp_forward(ob, R.gather_rows(w.feat.numpy(), ob.local_cat(0)), op)
        z = t.logits.double().cpu().numpy()
        assert R.max_rel_err(z, of.logits) < TOL_F32
        a = t.actions.cpu().numpy()
        if loss == "policy":
            old = t.old.double().cpu().numpy()
            want = T.policy_loss(z, a, old, t.adv.double().cpu().numpy(), ref_logp=old, kl_coef=0.1)["grad"]
        else:
            want = T.preference_loss(z, a, t.ptr.cpu().numpy(), beta=0.5)["grad"]
        g = t.glog.double().cpu().numpy()
        assert R.max_rel_err(g, want) < 1e-5
        act = [None] + [t.ctx.fetch_sage_activations(l, w.dims[l]).cpu().numpy() for l in range(1, w.n_layers)]
        masks, report = R.conditioned_relu_masks(ob, of, act, 1e-5)
        assert all(r[2] == 0 for r in report), report
        back = R.sp_backward(ob, of, op, g, relu_mask=masks)
        for got, ref in zip(t.grads, (back.gw_self, back.gw_neigh, back.gbias)):
            for x, y in zip(got, ref):
                assert R.max_rel_err(x.cpu().numpy(), y) < TOL_F32
        grads = [x.double().cpu().numpy() for x in t.gflat]
        norm = T.grad_norm(grads)
        assert abs(float(t.norm) - norm) < 1e-6 * norm and norm > 0.05        # clipped
        for i in range(len(t.flat)):
            p, m, v = T.adamw(before[0][i], grads[i], before[1][i], before[2][i], step=k + 1, factor=T.clip_factor(norm, 0.05), **STEP)
            # (the moments start at 0: a step of lr for every element that is not far below eps)
            assert np.max(np.abs(t.flat[i].double().cpu().numpy() - p)) < 2 ** -22 * np.max(np.abs(p)) + 1e-5 * STEP["lr"]
            assert R.max_rel_err(t.m[i].cpu().numpy(), m) < 1e-5 and R.max_rel_err(t.v[i].cpu().numpy(), v) < 1e-5
    t.ctx.close()


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_captured_steps_train_as_eager_ones_do(loss):
    t, e = _Trainer(loss), _Trainer(loss)
    t.at(0)
    t.step()                                # sizes the context's buffers
    torch.cuda.synchronize()
    for x, y in zip(t.flat + t.m + t.v, e.flat + e.m + e.v):
        x.copy_(y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        t.step(captured=True)
    for k in range(4):
        t.at(k)
        e.at(k)
        e.step()
        if k % 2:
            torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(t.logits, e.logits) and torch.equal(t.glog, e.glog), k
        # gradients of the layers below come in the order of the reverse index, which may differ in the last bits
        for x, y in zip(t.gflat, e.gflat):
            assert R.max_rel_err(x.cpu().numpy(), y.double().cpu().numpy()) < TOL_F32
        for x, y in zip(e.flat + e.m + e.v, t.flat + t.m + t.v):    # and the next step starts from the same weights
            assert float((x - y).abs().max()) < 1e-3 * STEP["lr"] + 1e-6 * float(y.abs().max())
            x.copy_(y)
    t.ctx.close()
    e.ctx.close()


def test_bench_trains_with_the_update():
    """The update's figures in a run of the benchmark's steps: the weights move and stay finite, and the norm's kernels are among them."""
    import bench
    w = workloads.tiny(device="cuda:0")
    start = [t.clone() for t in w.w_self]
    bench.Runner.with_update = True
    try:
        r = bench.Runner(w, torch.device("cuda:0"))
        r.ctx.gsplit_timing_enable(True)
        for i in range(3):
            r.step(w.targets(i), i)
        torch.cuda.synchronize()
        labels = r.ctx.gsplit_timing_read()
        assert "adamw" in labels and w.updates == 3
        for a, b in zip(w.w_self, start):
            assert torch.isfinite(a).all() and not torch.equal(a, b)
            assert float((a - b).abs().max()) < 4 * 1e-3       # three steps of at most about lr each
        r.ctx.close()
    finally:
        bench.Runner.with_update = False


def _bench_model(r):
    """The tensors that a benchmark Runner trains, one list."""
    return [t for lst in (r.gat_w if r.model == "gat" else (r.w.w_self, r.w.w_neigh, r.w.bias)) for t in lst]


@pytest.mark.parametrize("model", ["sage", "gat"])
def test_bench_slots_train_one_model(model):
    """The benchmark's schedules let several slots run the steps in turn: every step is the update of the weights that the step before
    left, with the gradients of its own batch, and all slots go on from it."""
    import bench
    w = workloads.tiny(device="cuda:0")
    bench.Runner.with_update = True
    try:
        slots = [bench.Runner(w, torch.device("cuda:0"), model, 4) for _ in range(3)]
        state = [_bench_model(slots[0])] + w.moments
        for i in range(6):
            before = [[t.double().cpu().numpy() for t in ts] for ts in state]
            r = slots[i % 3]
            r.step(w.targets(i), i)
            torch.cuda.synchronize()
            grads = [t.double().cpu().numpy() for lst in r.grads for t in lst]
            f = T.clip_factor(T.grad_norm(grads), 1.0)
            for k, g in enumerate(grads):
                want = T.adamw(before[0][k], g, before[1][k], before[2][k], lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01,
                               step=i + 1, factor=f)
                for ts, x in zip(state, want):
                    # (parameters: a step of about lr off by some roundings; moments: three roundings)
                    tol = 1e-5 * 1e-3 + 2 ** -22 * np.max(np.abs(x)) if ts is state[0] else 1e-5 * np.max(np.abs(x))
                    assert np.max(np.abs(ts[k].double().cpu().numpy() - x)) <= tol, (i, k)
        assert w.updates == 6
        for r in slots:         # and one batch has one answer, whichever slot computes it
            r.ctx.gsplit_sample_split(w.targets(9), r.seed, 9)
            r.load()
            r.forward()
        torch.cuda.synchronize()
        assert all(torch.equal(r.logits, slots[0].logits) for r in slots)
        for r in slots:
            r.ctx.close()
    finally:
        bench.Runner.with_update = False


@pytest.mark.parametrize("model, separate", [("sage", False), ("sage", True), ("gat", False)])
def test_bench_times_the_update_by_itself(monkeypatch, model, separate):
    """Every stage of a step has its events, the update's behind those of the backward pass."""
    import bench
    monkeypatch.setattr(bench.Runner, "with_update", True)
    monkeypatch.setattr(bench.Runner, "separate_calls", separate)
    w = workloads.tiny(device="cuda:0")
    r = bench.Runner(w, torch.device("cuda:0"), model, 4)
    names = bench.stage_names(model)
    assert names[-1] == "update"
    r.step(w.targets(0), 0)
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(len(names) + 1)]
    r.step(w.targets(1), 1, ev)
    torch.cuda.synchronize()
    assert all(ev[k].elapsed_time(ev[k + 1]) > 0 for k in range(len(names))) and w.updates == 2
    r.ctx.close()


@pytest.mark.parametrize("n_splits", [1, 4])
def test_preference_of_chosen_targets(n_splits):
    """Pairs of sequences of chosen target vertices.  The forward pass leaves its rows grouped by split: a caller brings them into the
    order of the sequences, and the gradient back; the weights' gradients are those of the loss of these vertices."""
    from paper_2303_13775_amd import Context, SageParams
    w = workloads.custom(3000, 40000, dims=[32, 48, 8], fanouts=[6, 4], batch=200, n_splits=n_splits, name="pairs")
    dev = torch.device("cuda:0")
    ctx = Context(w.indptr.to(dev), w.indices.to(dev), w.pmap.to(dev), w.n_splits, w.fanouts, w.batch)
    params = SageParams(w.dims, *[[t.to(dev) for t in lst] for lst in (w.w_self, w.w_neigh, w.bias)])
    tg = w.targets(0)
    x0 = torch.zeros((ctx.gsplit_max_rows(0), w.dims[0]), device=dev)
    ctx.gsplit_sample_split(tg.to(dev), 11, 0)
    ctx.gsplit_gather_features(w.feat.to(dev), x0)
    logits = torch.zeros((w.batch, w.dims[-1]), device=dev)
    ctx.gsplit_sage_fwd(params, x0, logits)
    # sequences of targets in an order of their own, ten targets in none
    rng = np.random.default_rng(3)
    used = rng.permutation(w.batch)[:190]
    lengths = [7, 12, 1, 30, 0, 25, 40, 75]
    assert sum(lengths) == len(used)
    ptr = np.concatenate([[0], np.cumsum(lengths)])
    action = rng.integers(0, w.dims[-1], w.batch)       # of every target
    # where each target's row is
    cat = torch.cat(ctx.fetch_batch()["local_front"][w.n_layers]).cpu().numpy()
    row_of = {int(v): r for r, v in enumerate(cat)}
    rows = np.array([row_of[int(tg[k])] for k in used])
    if n_splits > 1:
        assert (np.diff(rows) != 1).any()
    rows_dev = torch.from_numpy(rows).to(dev)
    z = logits[rows_dev].contiguous()
    g, work, loss = torch.zeros_like(z), torch.zeros((len(used), 4), device=dev), torch.zeros(4, device=dev)
    ctx.gsplit_preference_loss(z, torch.from_numpy(action[used]).to(dev), torch.from_numpy(ptr).to(dev), g, work, beta=0.5, pair_loss=loss)
    glog = torch.zeros_like(logits).index_copy_(0, rows_dev, g)
    grads = [[torch.zeros_like(t) for t in lst] for lst in params.tensors]
    ctx.gsplit_sage_bwd(params, glog, *grads)
    torch.cuda.synchronize()
    op = R.SageParams(*[[t.numpy() for t in lst] for lst in (w.w_self, w.w_neigh, w.bias)])
    ob = R.sp_sample(w.indptr.numpy(), w.indices.numpy(), w.pmap.numpy(), w.n_splits, w.fanouts, tg.numpy(), 11, 0)
    of = R.sp_forward(ob, R.gather_rows(w.feat.numpy(), ob.local_cat(0)), op)
    # the oracle's rows by its own map from targets to rows
    back = np.empty(w.batch, np.int64)
    back[np.asarray(ob.target_perm)] = np.arange(w.batch)
    z64 = logits.double().cpu().numpy()
    assert R.max_rel_err(z64, of.logits) < TOL_F32
    want = T.preference_loss(z64[back[used]], action[used], ptr, beta=0.5)
    assert np.abs(loss.cpu().numpy() - want["loss"]).max() < 1e-5 * np.abs(want["loss"]).max()
    full = np.zeros((w.batch, w.dims[-1]))
    full[back[used]] = want["grad"]
    assert R.max_rel_err(glog.cpu().numpy(), full) < 1e-5
    act = [None] + [ctx.fetch_sage_activations(l, w.dims[l]).cpu().numpy() for l in range(1, w.n_layers)]
    masks, report = R.conditioned_relu_masks(ob, of, act, 1e-5)
    assert all(r[2] == 0 for r in report), report
    # the weights' gradients of the gradient that the device formed
    bw = R.sp_backward(ob, of, op, glog.double().cpu().numpy(), relu_mask=masks)
    for got, ref in zip(grads, (bw.gw_self, bw.gw_neigh, bw.gbias)):
        for x, y in zip(got, ref):
            assert R.max_rel_err(x.cpu().numpy(), y) < TOL_F32
    ctx.close()
