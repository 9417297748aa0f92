"""The norm, clipping and the AdamW step on dense tensors of millions of elements, in the forms that smaller ones do not take: the norm
added up over several launches and read from one slot, its largest chunks, and the update that moves past the caches, with both types of
parameters and gradients, at odd sizes and addresses.  The float64 forms are computed on the device, tensor by tensor, with the
tolerances of test_gpu_update.py."""
import numpy as np
import pytest
import torch

import row_loss_check as K
from test_gpu_update import _cut, _room, _types

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = K.U


@pytest.fixture(scope="module")
def ctx():
    c = K.context()
    yield c
    c.close()


def _odd_sizes(tensors, total, seed):
    """Odd and even sizes of that many elements together, from a handful to a tenth of all."""
    rng = np.random.default_rng(seed)
    x = np.exp(rng.uniform(0, 8, tensors))
    return [int(n) for n in np.maximum(1, x / x.sum() * total)]


# (16 << 20 and one more: both sides of the update's bar)
LARGE_SETS = [_odd_sizes(300, 20_000_000, 1), _odd_sizes(40, 6_000_000, 2), _odd_sizes(400, 9_000_000, 3), [3_000_001, 0, 1_500_003], [16 << 20], [(16 << 20) + 1],
              [12_000_005, 3, 0, 7_000_003], [1_500_007, 9]]


def _tensors(gen, sizes, dtypes, scale, gap, fill=7.0):
    """Tensors of these sizes and types, of each type `gap` values apart in one buffer: (tensors, buffers)."""
    flats, out = {}, [None] * len(sizes)
    for dt in sorted(set(dtypes), key=str):
        which = [i for i, d in enumerate(dtypes) if d == dt]
        flat = torch.full((_room([sizes[i] for i in which], gap),), fill, dtype=dt, device="cuda")
        for i, v in zip(which, _cut(flat, [sizes[i] for i in which], gap)):
            v.copy_(torch.randn(sizes[i], device="cuda", generator=gen) * scale)
            out[i] = v
        flats[dt] = flat
    return out, flats


def _gaps_kept(flats, sizes, dtypes, gap, fill=7.0):
    for dt, flat in flats.items():
        kept = torch.ones_like(flat, dtype=torch.bool)
        for v in _cut(kept, [s for s, d in zip(sizes, dtypes) if d == dt], gap):
            v.fill_(False)
        if not bool((flat[kept] == fill).all()):
            return False
    return True


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _near(name, got, want, tol):
    """|got - want| within tol plus the rounding to got's type, element by element."""
    over = (got.double() - want).abs() - (tol + (K.EPS[got.dtype] + U) * want.abs() + K.TINY)
    assert got.numel() == 0 or float(over.max()) <= 0, (name, float(over.max()), int((over > 0).sum()))


def _norm(grads):
    return float(torch.stack([g.double().square().sum() for g in grads]).sum().sqrt())


@pytest.mark.parametrize("which", range(len(LARGE_SETS)))
@pytest.mark.parametrize("kind, gap", [("f32", 0), ("bf16", 0), ("mixed", 1), ("mixed", 3)])
def test_norm_and_clipping(ctx, which, kind, gap):
    from paper_2303_13775_amd import GradTensors
    sizes = LARGE_SETS[which]
    dtypes = _types(kind, len(sizes))
    grads, flats = _tensors(_gen(which), sizes, dtypes, 0.5, gap)
    outs, oflats = _tensors(_gen(100), sizes, dtypes, 0.5, gap)
    kept = {dt: f.clone() for dt, f in flats.items()}
    want = _norm(grads)
    norm = torch.full((1,), 9.0, device="cuda")
    ctx.gsplit_grad_norm(GradTensors(grads), norm)
    assert abs(float(norm) - want) <= 1.5 * U * want
    for bound in (0.37 * want, 3.0 * want):
        norm.fill_(9.0)
        ctx.gsplit_clip_grads(GradTensors(grads, outs), bound, norm)
        assert abs(float(norm) - want) <= 1.5 * U * want
        f = bound / want if want > bound else 1.0
        for g, o in zip(grads, outs):
            x = f * g.double()
            _near("clipped", o, x, 4 * U * x.abs())
        assert all(torch.equal(flats[dt], kept[dt]) for dt in flats) and _gaps_kept(oflats, sizes, dtypes, gap)
        if f == 1.0:
            assert all(torch.equal(a, b) for a, b in zip(grads, outs))
    ctx.gsplit_clip_grads(GradTensors(grads, outs), 0.37 * want)
    ctx.gsplit_clip_grads(GradTensors(grads), 0.37 * want)        # in place
    assert all(torch.equal(a, b) for a, b in zip(grads, outs)) and _gaps_kept(flats, sizes, dtypes, gap)


@pytest.mark.parametrize("which", range(len(LARGE_SETS)))
@pytest.mark.parametrize("pk, gk, gap", [("f32", "f32", 0), ("bf16", "bf16", 0), ("mixed", "f32", 1), ("f32", "bf16", 3), ("mixed", "mixed", 5)])
@pytest.mark.parametrize("max_norm", [0.0, 2.5])
def test_adamw(ctx, which, pk, gk, gap, max_norm):
    from paper_2303_13775_amd import AdamwTensors
    sizes = LARGE_SETS[which]
    n = len(sizes)
    ptypes, gtypes, floats = _types(pk, n), _types(gk, n), [F32] * n
    lr, b1, b2, eps, wd, step = 1e-2, 0.9, 0.99, 1e-8, 0.05, 3
    params, pf = _tensors(_gen(1), sizes, ptypes, 0.3, gap)
    grads, gf = _tensors(_gen(2), sizes, gtypes, 0.1, gap)
    m, mf = _tensors(_gen(3), sizes, floats, 0.05, gap)
    v, vf = _tensors(_gen(4), sizes, floats, 0.05, gap)
    for t in v:
        t.square_()
    full, ff = _tensors(_gen(5), sizes, floats, 0.3, gap)
    masters = [w if p.dtype == BF16 else None for p, w in zip(params, full)]
    updated = [p if w is None else w for p, w in zip(params, masters)]
    old = [[t.clone() for t in ts] for ts in (updated, grads, m, v)]
    norm = torch.full((1,), 9.0, device="cuda")
    ctx.gsplit_adamw_step(AdamwTensors(params, grads, m, v, masters), lr=lr, beta1=b1, beta2=b2, eps=eps, weight_decay=wd, step=step, max_norm=max_norm,
                          norm=norm)
    want_norm = _norm(old[1])
    f = 1.0
    if max_norm:
        assert abs(float(norm) - want_norm) <= 1.5 * U * want_norm and want_norm > max_norm
        f = max_norm / want_norm
    else:
        assert float(norm) == 9.0
    for i in range(n):
        p0, g0, m0, v0 = (ts[i].double() for ts in old)
        g = f * g0
        m1, v1 = b1 * m0 + (1 - b1) * g, b2 * v0 + (1 - b2) * g * g
        mt = (b1 * m0).abs() + ((1 - b1) * g).abs()
        root = (v1 / (1 - b2 ** step)).sqrt() + eps
        rate = lr / (1 - b1 ** step)
        _near("m", m[i], m1, 5 * U * mt)
        _near("v", v[i], v1, 7 * U * v1)
        _near("p", updated[i], (1 - lr * wd) * p0 - rate * m1 / root, rate / root * (6 * U * mt + 14 * U * m1.abs()) + 2 * U * p0.abs())
        assert torch.equal(grads[i], old[1][i])
        if masters[i] is not None:
            assert torch.equal(params[i], masters[i].bfloat16())
    for flats, types in ((pf, ptypes), (gf, gtypes), (mf, floats), (vf, floats), (ff, floats)):
        assert _gaps_kept(flats, sizes, types, gap)


def test_adamw_of_a_device_step(ctx):
    """Step and learning rate in device memory, in the large form: the bits of the same numbers from the host."""
    from paper_2303_13775_amd import AdamwTensors
    sizes = LARGE_SETS[6]
    got = []
    for dev in (False, True):
        ts = [_tensors(_gen(k), sizes, [F32] * 4, s, 1)[0] for k, s in ((1, 0.3), (2, 0.1), (3, 0.05), (4, 0.05))]
        for t in ts[3]:
            t.square_().add_(0.01)          # (a change of at most 0.01 an element)
        lr = float(np.float32(0.01))
        kw = dict(step_dev=torch.tensor([7], device="cuda"), lr_dev=torch.tensor([lr], device="cuda")) if dev else dict(step=7, lr=lr)
        ctx.gsplit_adamw_step(AdamwTensors(*ts), max_norm=2.5, **kw)
        got.append(ts)
    # the host's and the device's power may round each of the step's two numbers apart: 2 u and u of the change, and one sum and product
    for a, b in zip(got[0][0], got[1][0]):
        assert a.numel() == 0 or float((a - b).abs().max()) <= 2 * U * float(a.abs().max()) + 8 * U * 0.01
    for k in (2, 3):
        assert all(torch.equal(a, b) for a, b in zip(got[0][k], got[1][k]))
