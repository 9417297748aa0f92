"""The losses over rows of logits (gsplit_policy_loss, gsplit_preference_loss) against their plain float64 forms: every width
class of a row on both sides of its borders, odd sizes, strides and addresses, rows and classes that are left out, and the ways a
caller may run them."""
import numpy as np
import pytest
import torch

import row_loss_check as K
from oracle import training as T

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = K.context()
    yield c
    c.close()


def _dev(x, dtype=None):
    return torch.as_tensor(x).to("cuda") if dtype is None else torch.as_tensor(x).to(dtype).to("cuda")


def _logits(rng, n, C, dtype, scale=3.0):
    return torch.from_numpy((rng.standard_normal((n, C)) * scale).astype(np.float32)).to(dtype)


def _chosen_logp(z64, a):
    out = np.zeros(len(a))
    for r, k in enumerate(a):
        if 0 <= k < z64.shape[1]:
            d = T.row_distribution(z64[r])
            out[r] = 0.0 if d is None else d[0][k]
    return np.nan_to_num(out, nan=-1.0, neginf=-5.0, posinf=0.0)


def _policy(ctx, z, a, *, seed=0, dtype=F32, pad=0, gpad=0, offset=0, kl=0.05, weights=True, masked=0.0, low=0.2, high=0.3, grad="out",
            spread=0.5):
    """One call on logits z (CPU, dtype) and its checks; returns the outputs."""
    n, C = z.shape
    rng = np.random.default_rng(seed + 1)
    z64 = z.double().numpy()
    logp = _chosen_logp(z64, a)
    old = K.away_from_borders(logp, (logp + rng.standard_normal(n) * spread).astype(np.float32), low, high)
    ref = (logp + rng.standard_normal(n) * 0.4).astype(np.float32) if kl is not None else None
    adv = rng.standard_normal(n).astype(np.float32)
    w = (rng.random(n) + 0.1).astype(np.float32) if weights else None
    if weights and masked:
        w[rng.random(n) < masked] = 0.0
    want = T.policy_loss(z64, a, old, adv, ref_logp=ref, weight=w, clip_low=low, clip_high=float(np.float32(high)), kl_coef=float(np.float32(kl or 0.0)))
    whole, zd = K.rows_buffer(z, dtype, pad, offset)
    gwhole, gd = (whole, zd) if grad == "in place" else K.rows_buffer(torch.zeros(n, C), dtype, gpad, offset) if grad else (None, None)
    outs = {k: torch.full((n,), 5.0, device="cuda") for k in ("loss", "logp", "kl")}
    before = whole.clone()
    ctx.gsplit_policy_loss(zd, _dev(np.asarray(a, np.int64)), _dev(old), _dev(adv), gd, ref_logp=None if ref is None else _dev(ref),
                           row_weight=None if w is None else _dev(w), clip_low=low, clip_high=high, kl_coef=kl or 0.0,
                           row_loss=outs["loss"], row_logp=outs["logp"], row_kl=outs["kl"])
    torch.cuda.synchronize()
    slope = np.nan_to_num(want["slope"])
    dlp, dgrad = K.terms(z64, slope)
    ww = np.full(n, 1.0 / n) if w is None else w.astype(np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        lp = want["logp"]
        steep = np.abs(adv) * np.exp(lp - old)                         # |d (policy term) / d log p| at most, and its derivative
        ed = np.exp(ref - lp) if ref is not None else np.zeros(n)
        b = kl or 0.0
        dslope = np.abs(ww) * (steep + b * ed) * dlp + 3 * K.U * np.abs(ww) * (steep + b * (ed + 1))
        dloss = np.abs(ww) * (steep + b * np.abs(ed - 1)) * dlp + 3 * K.U * np.abs(ww) * (steep + np.abs(adv) * (1 + high))
        dlp, dslope, dloss, dkl = (np.nan_to_num(t, nan=0.0, posinf=0.0) for t in (dlp, dslope, dloss, np.abs(ed - 1) * dlp))
    K.check("logp", outs["logp"], want["logp"], dlp)
    K.check("loss", outs["loss"], want["loss"], dloss)
    K.check("kl", outs["kl"], want["kl"], dkl)
    if gd is not None:
        K.check("grad", gd, want["grad"], np.nan_to_num(dgrad) + dslope[:, None], dtype)
        assert K.untouched(gwhole, gd)
    if grad != "in place":
        assert torch.equal(before.view(torch.uint8), whole.view(torch.uint8)), "the logits changed"
    return outs, gd


def _actions(rng, n, C):
    return rng.integers(0, C, n)


# widths on both sides of the borders between the kernels' forms, odd ones among them
WIDTHS = [1, 2, 3, 7, 16, 31, 47, 64, 65, 127, 128, 172, 255, 256, 257, 511, 513, 1000, 1023, 1024, 1025, 2047, 2049, 4095, 4097, 8193]


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_policy_widths(ctx, C, dtype):
    rng = np.random.default_rng(C)
    n = 37 if C > 300 else 333
    _policy(ctx, _logits(rng, n, C, dtype), _actions(rng, n, C), dtype=dtype, masked=0.2)


@pytest.mark.parametrize("C", [16383, 16385, 32768, 32769, 50001, 65536, 65537, 131071, 131072, 140001, 262145])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 5])
def test_policy_wide_rows(ctx, C, dtype, n):
    rng = np.random.default_rng(C + n)
    _policy(ctx, _logits(rng, n, C, dtype), _actions(rng, n, C), dtype=dtype, pad=(C + n) % 3)


# (rows, classes) of the forms that need many rows, or that the widths above leave out
POLICY_FORMS = [(260, 60001), (257, 65543), (130, 70001), (128, 131079), (130, 140001)]


@pytest.mark.parametrize("n, C", [(300, 16385), (270, 33001), (600, 9000)] + POLICY_FORMS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_policy_many_wide_rows(ctx, n, C, dtype):
    rng = np.random.default_rng(C)
    _policy(ctx, _logits(rng, n, C, dtype), _actions(rng, n, C), dtype=dtype, masked=0.3)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 255, 256, 257, 2049, 9001])
def test_policy_row_counts(ctx, n):
    rng = np.random.default_rng(n)
    _policy(ctx, _logits(rng, n, 47, F32), _actions(rng, n, 47), masked=0.1 if n > 60 else 0.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [5, 47, 172, 600, 5000, 40003])
@pytest.mark.parametrize("pad, gpad, offset", [(1, 0, 0), (0, 3, 1), (8, 8, 5), (5, 1, 2)])
def test_policy_strides_and_addresses(ctx, dtype, C, pad, gpad, offset):
    rng = np.random.default_rng(C + pad)
    n = 21 if C > 1000 else 90
    _policy(ctx, _logits(rng, n, C, dtype), _actions(rng, n, C), dtype=dtype, pad=pad, gpad=gpad, offset=offset)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, C, pad", [(100, 47, 0), (100, 172, 3), (50, 1500, 0), (3, 70001, 0), (300, 20000, 1), (2, 300000, 0)])
def test_policy_gradient_in_place(ctx, dtype, n, C, pad):
    rng = np.random.default_rng(C)
    _policy(ctx, _logits(rng, n, C, dtype), _actions(rng, n, C), dtype=dtype, pad=pad, grad="in place")


@pytest.mark.parametrize("n, C", [(100, 47), (40, 3001), (3, 90001)])
def test_policy_forward_alone_and_defaults(ctx, n, C):
    rng = np.random.default_rng(n)
    _policy(ctx, _logits(rng, n, C, F32), _actions(rng, n, C), grad=None)
    _policy(ctx, _logits(rng, n, C, F32), _actions(rng, n, C), weights=False, kl=None)
    _policy(ctx, _logits(rng, n, C, F32), _actions(rng, n, C), kl=0.0)          # the KL term reported, not in the loss


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, C", [(60, 9), (60, 47), (60, 200), (60, 1111), (60, 5003), (12, 40000), (9, 90001)])
def test_policy_left_out_rows_and_classes(ctx, dtype, n, C):
    rng = np.random.default_rng(C)
    z = _logits(rng, n, C, dtype)
    a = _actions(rng, n, C)
    low = torch.finfo(dtype).min
    z[0] = -np.inf                      # no class is possible
    z[1, torch.arange(C) != a[1]] = -np.inf         # one class is
    z[2] = low                          # all alike, at the type's lowest value
    z[3, ::2] = low
    a[4], a[5], a[6] = -1, C, 2 ** 40
    z[7, 1:] = -np.inf
    a[7] = 0
    z[8, a[8]] = 60000.0                # one class has it all
    if n > 9:
        z[9, 0] = np.inf                # NaN results of this row alone
        z[10, 0] = np.nan
        z[11, :] = -np.inf
        z[11, C - 1] = np.nan
        a[11] = 0
    _policy(ctx, z, a, dtype=dtype)
    # the same in rows of weight 0: nothing of them shows
    w0, g0 = torch.zeros(n, device="cuda"), torch.full((n, C), 3.0, dtype=dtype, device="cuda")
    outs = [torch.full((n,), 5.0, device="cuda") for _ in range(3)]
    one = torch.ones(n, device="cuda")
    ctx.gsplit_policy_loss(z.cuda(), _dev(a.astype(np.int64)), one, one, g0, row_weight=w0, row_loss=outs[0], row_logp=outs[1], row_kl=outs[2])
    assert not g0.any() and not any(t.any() for t in outs)


@pytest.mark.parametrize("n, C", [(6, 47), (6, 3000), (6, 40000), (6, 90001)])
def test_policy_impossible_action(ctx, n, C):
    """An action whose logit is -inf: log p = -inf, ratio 0, the loss and gradient that the formula gives; also without an advantage."""
    rng = np.random.default_rng(C)
    z = _logits(rng, n, C, F32)
    a = _actions(rng, n, C)
    for r in (1, 2, 3):
        z[r, a[r]] = -np.inf
    old, adv = np.full(n, -3.0, np.float32), np.array([1, 1, -1, 0, 0, -1], np.float32)
    old[4] = -200.0             # a ratio of e^190 and no advantage
    want = T.policy_loss(z.double().numpy(), a, old, adv)
    g, loss, logp, kl = torch.zeros(n, C, device="cuda"), *(torch.zeros(n, device="cuda") for _ in range(3))
    ctx.gsplit_policy_loss(z.cuda(), _dev(a), _dev(old), _dev(adv), g, row_loss=loss, row_logp=logp, ref_logp=_dev(old), row_kl=kl)
    assert bool((logp[1:4] == -np.inf).all()) and bool((kl[1:4] == np.inf).all()) and bool(torch.isfinite(kl[[0, 5]]).all())
    assert np.allclose(loss.cpu().numpy(), want["loss"], rtol=1e-4)
    assert (g.any(1).cpu().numpy() == (want["slope"] != 0)).all() and not want["slope"][1:5].any()


@pytest.mark.parametrize("n, C", [(12, 47), (12, 3000), (12, 40000), (12, 90001)])
def test_policy_row_without_a_number(ctx, n, C):
    """A NaN among what a row brings (advantage, old log p, weight) shows in its loss and in its whole gradient, on either side of the
    clip and inside it; the other rows do not see it."""
    rng = np.random.default_rng(C + 1)
    z, a = _logits(rng, n, C, F32), _actions(rng, n, C)
    logp = _chosen_logp(z.double().numpy(), a)
    off = np.tile(np.array([1.0, -1.0, 0.01]), n // 3)              # ratios of e, 1 / e and within the clip
    old, adv, w = (logp - off).astype(np.float32), rng.standard_normal(n).astype(np.float32), np.ones(n, np.float32)
    adv[0:3], old[3:5], w[6:9] = np.nan, np.nan, np.nan
    want = T.policy_loss(z.double().numpy(), a, old, adv, weight=w)
    bad = np.isnan(want["loss"])
    assert list(np.flatnonzero(bad)) == [0, 1, 2, 3, 4, 6, 7, 8]
    g, loss = torch.zeros(n, C, device="cuda"), torch.zeros(n, device="cuda")
    ctx.gsplit_policy_loss(z.cuda(), _dev(a), _dev(old), _dev(adv), g, row_weight=_dev(w), row_loss=loss)
    assert (torch.isnan(loss).cpu().numpy() == bad).all()
    nan = torch.isnan(g)
    assert (nan.all(1).cpu().numpy() == bad).all() and (nan.any(1).cpu().numpy() == bad).all()


def test_policy_far_ratios(ctx):
    """Ratios from e^-30 to e^30, on either side of an advantage."""
    rng = np.random.default_rng(8)
    _policy(ctx, _logits(rng, 500, 47, F32), _actions(rng, 500, 47), spread=10.0, kl=None)


def test_policy_far_reference(ctx):
    """References far from the policy, down to probability 0: the KL term's slope is kl_coef (1 - exp(delta)), which stays a number."""
    rng = np.random.default_rng(17)
    far = np.array([-np.inf, torch.finfo(F32).min, -1e8, -1e6, -1e4, -300, -90, -30, -20, -17, -5, -1.01, 1.01, 3, 9, 30], np.float32)
    n, C, b = len(far), 47, 0.5
    z, a = _logits(rng, n, C, F32), _actions(rng, n, C)
    z64 = z.double().numpy()
    lp = _chosen_logp(z64, a)
    old, ref, adv = lp.astype(np.float32), np.where(far < -200, far, lp + far).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    w = np.ones(n, np.float32)
    want = T.policy_loss(z64, a, old, adv, ref_logp=ref, weight=w, kl_coef=b)
    g, loss, kl = torch.zeros(n, C, device="cuda"), *(torch.zeros(n, device="cuda") for _ in range(2))
    ctx.gsplit_policy_loss(z.cuda(), _dev(a), _dev(old), _dev(adv), g, ref_logp=_dev(ref), row_weight=_dev(w), kl_coef=b, row_loss=loss, row_kl=kl)
    dlp, dgrad = K.terms(z64, want["slope"])
    ed = np.exp(ref.astype(np.float64) - lp)
    # delta rounds by u |delta|, its exponential by that and 2 u: u (|delta| + 2) e^delta; a KL term near |delta| by u |delta| and its last
    # steps, u (|kl| + 1) each; the loss and the slope by three roundings of their terms
    delta = np.where(np.isfinite(ref), np.abs(ref.astype(np.float64) - lp), 0.0)
    rel = np.where(ed > 0, K.U * (delta + 2) * ed, 0.0)
    dkl = np.abs(ed - 1) * dlp + rel + K.U * (delta + 3)
    K.check("kl", kl, want["kl"], dkl)
    K.check("loss", loss, want["loss"], np.abs(adv) * dlp + b * dkl + 3 * K.U * (np.abs(adv) + np.nan_to_num(b * want["kl"], posinf=0.0)))
    dslope = (np.abs(adv) + b * ed) * dlp + b * rel + 3 * K.U * (np.abs(adv) + b * (ed + 1))
    assert np.isfinite(want["slope"]).all() and (np.abs(want["slope"]) > 1e-3).all()
    K.check("grad", g, want["grad"], dgrad + dslope[:, None])


def test_policy_gradient_against_differences(ctx):
    """The gradient against differences of the device's own loss: a step h changes the loss of a row by slope h (1 - p) + O(h^2)."""
    rng = np.random.default_rng(2)
    n, C = 64, 47
    z = _logits(rng, n, C, F32, 1.0)
    a = _actions(rng, n, C)
    logp = _chosen_logp(z.double().numpy(), a)
    old = K.away_from_borders(logp, (logp + rng.standard_normal(n) * 0.3).astype(np.float32), 0.2, 0.2, by=0.02)
    ref, adv = (logp + 0.2).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    args = [_dev(a), _dev(old), _dev(adv)]

    def loss(y, g=None):
        out = torch.zeros(n, device="cuda")
        ctx.gsplit_policy_loss(y, *args, g, ref_logp=_dev(ref), kl_coef=0.1, row_weight=torch.ones(n, device="cuda"), row_loss=out)
        return out.double()

    g = torch.zeros(n, C, device="cuda")
    loss(z.cuda(), g)
    h = 2.0 ** -7
    for c in (0, 13, 46):
        up, down = z.cuda(), z.cuda()
        up[:, c] += h
        down[:, c] -= h
        step = (up[:, c] - down[:, c]).double()
        diff = (loss(up) - loss(down)) / step
        # third derivative h^2 / 6 of terms up to |A| rho + 0.1 e^delta <= 6, times up to 8; losses up to 6 off by 100 u each
        tol = h * h / 6 * 48 + 2 * 6 * 100 * K.U / (2 * h)
        assert float((diff - g[:, c].double()).abs().max()) < tol


# -- preference ---------------------------------------------------------------------------------

def _preference(ctx, z, a, ptr, *, seed=0, dtype=F32, pad=0, gpad=0, offset=0, beta=0.1, e=0.1, ref=True, weights=True, grad="out"):
    n, C = z.shape
    pairs = len(ptr) // 2
    rng = np.random.default_rng(seed + 1)
    z64 = z.double().numpy()
    logp = _chosen_logp(z64, a)
    sums = np.array([logp[ptr[q]:ptr[q + 1]].sum() for q in range(2 * pairs)])
    R = (sums + rng.standard_normal(2 * pairs) * 4).astype(np.float32) if ref else None
    w = (rng.random(pairs) + 0.1).astype(np.float32) if weights else None
    if weights and pairs > 3:
        w[1] = 0.0
    f32 = lambda x: float(np.float32(x))
    want = T.preference_loss(z64, a, ptr, ref_logp=R, weight=w, beta=f32(beta), smoothing=f32(e))
    whole, zd = K.rows_buffer(z, dtype, pad, offset)
    gwhole, gd = (whole, zd) if grad == "in place" else K.rows_buffer(torch.full((n, C), 7.0), dtype, gpad, offset) if grad else (None, None)
    before = whole.clone()
    o = {k: torch.full((m,), 5.0, device="cuda") for k, m in (("loss", pairs), ("margin", pairs), ("logp", n))}
    work = torch.full((max(n, 1), 4), float("nan"), device="cuda")[:n]
    ctx.gsplit_preference_loss(zd, _dev(np.asarray(a, np.int64)), _dev(np.asarray(ptr, np.int64)), gd, work, ref_logp=None if R is None else _dev(R),
                               pair_weight=None if w is None else _dev(w), beta=beta, label_smoothing=e, pair_loss=o["loss"],
                               pair_margin=o["margin"], row_logp=o["logp"])
    torch.cuda.synchronize()
    lo, hi = int(ptr[0]), int(ptr[-1])
    slope = np.nan_to_num(want["slope"])
    dlp, dgrad = K.terms(z64, slope) if n else (np.zeros(0), np.zeros((0, C)))
    dlp = np.nan_to_num(dlp)
    dsum = np.array([dlp[ptr[q]:ptr[q + 1]].sum() for q in range(2 * pairs)])
    dh = abs(beta) * (dsum[0::2] + dsum[1::2])
    ww = np.full(pairs, 1.0 / max(1, pairs)) if w is None else w.astype(np.float64)
    K.check("margin", o["margin"], want["margin"], dh)
    K.check("loss", o["loss"], want["loss"], ww * dh)
    K.check("logp", o["logp"][lo:hi], want["logp"][lo:hi], dlp[lo:hi])
    assert bool((o["logp"][:lo] == 5.0).all()) and bool((o["logp"][hi:] == 5.0).all())
    if gd is not None:
        dslope = np.zeros(n)
        for p in range(pairs):          # |d slope / d margin| <= beta w / 4
            dslope[ptr[2 * p]:ptr[2 * p + 2]] = abs(beta) * ww[p] * dh[p] / 4 + 3 * K.U * abs(beta) * ww[p]
        K.check("grad", gd[lo:hi], want["grad"][lo:hi], (np.nan_to_num(dgrad) + dslope[:, None])[lo:hi], dtype)
        assert K.untouched(gwhole, gd)
        rest = torch.cat([gd[:lo].reshape(-1), gd[hi:].reshape(-1)])
        kept = torch.cat([zd[:lo].reshape(-1), zd[hi:].reshape(-1)]) if grad == "in place" else torch.full_like(rest, 7.0)
        assert torch.equal(rest, kept), "rows of no sequence were written"
    if grad != "in place":
        assert torch.equal(before.view(torch.uint8), whole.view(torch.uint8)), "the logits changed"
    return o, gd


def _ptr(lengths, first=0):
    return np.concatenate([[first], first + np.cumsum(lengths)]).astype(np.int64)


@pytest.mark.parametrize("C", [1, 2, 3, 16, 47, 64, 65, 172, 256, 257, 513, 1024, 1025, 2049, 4097, 8193, 20001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_preference_widths(ctx, C, dtype):
    rng = np.random.default_rng(C)
    lengths = rng.integers(0, 6, 12)
    n = int(lengths.sum()) + 9
    a = _actions(rng, n, C)
    a[rng.random(n) < 0.2] = -1
    _preference(ctx, _logits(rng, n, C, dtype), a, _ptr(lengths, 4), dtype=dtype)


@pytest.mark.parametrize("lengths", [[1, 1], [0, 0], [0, 3], [7, 0], [1] * 600, [300, 5, 2, 700], [64, 65, 63, 1], [0] * 8,
                                     [1000, 1000], [33] * 200])
@pytest.mark.parametrize("C", [10, 300])
def test_preference_lengths(ctx, lengths, C):
    rng = np.random.default_rng(len(lengths))
    n = int(np.sum(lengths))
    _preference(ctx, _logits(rng, n, C, F32), _actions(rng, n, C), _ptr(lengths))


# lengths and classes of every way a pair is taken: a workgroup of 64, 256 or 1024 threads or three launches, teams of 16, 64 and 256
# lanes, and rows in parts
PREFERENCE_FORMS = [([1, 1] * 20, 47), ([3, 5] * 30, 47), ([40, 30] * 5, 172), ([700, 400], 172), ([1, 0] * 10, 1000), ([2, 1] * 9, 3000),
                    ([7, 6] * 3, 600), ([100, 150], 900), ([1, 1], 5000), ([150, 160], 5001), ([20, 10], 20000)]


@pytest.mark.parametrize("lengths, C", PREFERENCE_FORMS)
def test_preference_forms(ctx, lengths, C):
    rng = np.random.default_rng(C)
    n = int(np.sum(lengths)) + 2
    a = _actions(rng, n, C)
    a[rng.random(n) < 0.2] = -1
    for dtype in (F32, BF16):
        _preference(ctx, _logits(rng, n, C, dtype), a, _ptr(lengths, 1), dtype=dtype)
        _preference(ctx, _logits(rng, n, C, dtype), a, _ptr(lengths, 1), dtype=dtype, pad=3, gpad=3, grad="in place")


@pytest.mark.parametrize("lengths, C", [([5, 1, 0, 0, 1, 0, 0, 1], 8191), ([0, 2, 1, 1, 0, 4, 0, 0], 4097), ([1] * 990 + [20, 14] + [0] * 32, 9001)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_preference_wide_rows_by_a_workgroup_a_pair(ctx, lengths, C, dtype):
    """As many rows as sequences, but not one each: a workgroup takes several wide rows one after the other."""
    import row_rules as R
    n = int(np.sum(lengths))
    assert n == len(lengths) and R.lib().part(C) == 256 == R.lib().whole(n, n // 2, C, R.N_CU)
    rng = np.random.default_rng(C)
    a = _actions(rng, n, C)
    a[rng.random(n) < 0.2] = -1
    _preference(ctx, _logits(rng, n, C, dtype), a, _ptr(lengths), dtype=dtype)
    _preference(ctx, _logits(rng, n, C, dtype), a, _ptr(lengths), dtype=dtype, pad=3, gpad=3, grad="in place")


@pytest.mark.parametrize("lengths, C", [([1, 1], 65537), ([2, 1], 131072), ([1, 0], 140001), ([3, 4, 1, 0], 50001), ([150, 160], 9001)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_preference_wide_rows(ctx, lengths, C, dtype):
    rng = np.random.default_rng(C)
    n = int(np.sum(lengths)) + 2
    _preference(ctx, _logits(rng, n, C, dtype), _actions(rng, n, C), _ptr(lengths, 1), dtype=dtype, pad=1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad, gpad, offset, grad", [(1, 0, 0, "out"), (0, 3, 1, "out"), (8, 8, 5, "out"), (3, 3, 1, "in place"), (0, 0, 0, None)])
@pytest.mark.parametrize("C", [47, 172, 700, 5003])
def test_preference_strides_and_forms(ctx, dtype, pad, gpad, offset, grad, C):
    rng = np.random.default_rng(C)
    lengths = [5, 3, 0, 2, 8, 8]
    n = int(np.sum(lengths)) + 5
    z, a = _logits(rng, n, C, dtype), _actions(rng, n, C)
    _preference(ctx, z, a, _ptr(lengths, 3), dtype=dtype, pad=pad, gpad=gpad, offset=offset, grad=grad)
    _preference(ctx, z, a, _ptr(lengths, 3), dtype=dtype, pad=pad, gpad=gpad, offset=offset, grad=grad, ref=False, weights=False, e=0.0, beta=2.0)


@pytest.mark.parametrize("C", [9, 47, 300, 3001, 20000])
def test_preference_left_out_rows_and_classes(ctx, C):
    rng = np.random.default_rng(C)
    lengths = [6, 6, 3, 3, 2, 2, 1, 1]
    n = int(np.sum(lengths))
    z, a = _logits(rng, n, C, F32), _actions(rng, n, C)
    z[0] = -np.inf
    z[1, torch.arange(C) != a[1]] = -np.inf
    z[2] = torch.finfo(F32).min
    a[3], a[4] = -1, C
    z[8, ::2] = -np.inf
    a[8] = 1
    z[18, 0] = np.nan               # a NaN goes as far as its pair
    a[18] = 1
    _preference(ctx, z, a, _ptr(lengths))


@pytest.mark.parametrize("C", [9, 47, 3001, 20000])
@pytest.mark.parametrize("e", [0.0, 0.25, 1.0])
def test_preference_impossible_answers(ctx, C, e):
    """Answers of probability 0 (an action whose logit is -inf): the rejected one's makes the margin inf, the chosen one's -inf; a term of
    the loss whose factor is 0 is 0 whatever the margin."""
    rng = np.random.default_rng(C)
    z, a = _logits(rng, 12, C, F32), _actions(rng, 12, C)
    z[3, a[3]] = -np.inf            # pair 0: the rejected answer
    z[4, a[4]] = -np.inf            # pair 1: the chosen one
    g = _preference(ctx, z, a, _ptr([2, 2, 2, 2, 2, 2]), e=e)[1]
    assert bool(g[:4].any()) == (e > 0) and bool(g[4:8].any()) == (e < 1) and bool(torch.isfinite(g).all())


def test_preference_offsets_that_make_no_sense_stay_inside(ctx):
    """Descending offsets and such outside the buffers: wrong values, but nothing outside the rows is written."""
    rng = np.random.default_rng(1)
    n, C = 20, 33
    for ptr in ([-5, 10, 50], [15, 3, 8], [2 ** 40, 3, -2 ** 40], [0, 2 ** 62, 20], [18, 2, 19, 1, 20]):
        whole, z = K.rows_buffer(_logits(rng, n, C, F32), F32, 2, 1)
        gw, g = K.rows_buffer(torch.zeros(n, C), F32, 2, 1)
        pairs = len(ptr) // 2
        work = torch.full((n + 2, 4), 9.0, device="cuda")
        outs = [torch.full((pairs + 2,), 9.0, device="cuda") for _ in range(2)]
        ctx.gsplit_preference_loss(z, _dev(_actions(rng, n, C)), _dev(np.array(ptr, np.int64)), g, work[1:n + 1],
                                   pair_loss=outs[0][1:pairs + 1], pair_margin=outs[1][1:pairs + 1])
        torch.cuda.synchronize()
        assert K.untouched(gw, g) and K.untouched(whole, z)
        assert bool((work[0] == 9).all() and (work[n + 1] == 9).all())
        assert all(bool(t[0] == 9) and bool(t[-1] == 9) for t in outs)


# (rows, classes) of the launches over all rows, with teams of 16, 64 and 256 lanes, and of the rows in parts
OFFSET_FORMS = [(1100, 172, 16, False), (300, 900, 64, False), (300, 9001, 256, False), (20, 20000, 256, True), (250, 9001, 256, True)]


@pytest.mark.parametrize("n, C, lanes, parts", OFFSET_FORMS)
@pytest.mark.parametrize("grad", ["out", "in place"])
def test_preference_offsets_that_make_no_sense_in_several_launches(ctx, n, C, lanes, parts, grad):
    """The same offsets where the rows' statistics, the pairs and the gradient are launches of their own: nothing around the rows of any
    buffer is written, nothing but rows between the first and the last offset gets a gradient, and the context stays usable."""
    import row_rules as R
    rng = np.random.default_rng(n + C)
    for ptr in ([-5, n // 2, n + 30], [n - 5, 3, 8], [2 ** 40, 3, -2 ** 40], [0, 2 ** 62, n], [0, -2 ** 62, n], [7, n - 3, 2, n - 1, n // 2]):
        pairs = len(ptr) // 2
        assert R.lib().part(C) == lanes and not R.lib().whole(n, pairs, C, R.N_CU)
        assert bool(lanes == 256 and R.lib().preference_parts(n, C, R.N_CU)) == parts
        z0 = _logits(rng, n, C, F32)
        whole, z = K.rows_buffer(z0, F32, 2, 1)
        gw, g = (whole, z) if grad == "in place" else K.rows_buffer(torch.full((n, C), 7.0), F32, 2, 1)
        a = _actions(rng, n, C)
        a[rng.random(n) < 0.2] = -1
        work = torch.full((n + 2, 4), 9.0, device="cuda")
        logp = torch.full((n + 2,), 9.0, device="cuda")
        outs = [torch.full((pairs + 2,), 9.0, device="cuda") for _ in range(2)]
        ctx.gsplit_preference_loss(z, _dev(a), _dev(np.array(ptr, np.int64)), g, work[1:n + 1], row_logp=logp[1:n + 1],
                                   pair_loss=outs[0][1:pairs + 1], pair_margin=outs[1][1:pairs + 1])
        torch.cuda.synchronize()
        assert K.untouched(gw, g) and K.untouched(whole, z)
        assert bool((work[0] == 9).all() and (work[n + 1] == 9).all())
        assert all(bool(t[0] == 9) and bool(t[-1] == 9) for t in outs + [logp])
        lo, hi = (min(max(ptr[k], 0), n) for k in (0, -1))
        kept = z0.cuda() if grad == "in place" else torch.full((n, C), 7.0, device="cuda")
        hi = max(lo, hi)
        assert torch.equal(g[:lo], kept[:lo]) and torch.equal(g[hi:], kept[hi:])
    _preference(ctx, _logits(rng, n, C, F32), _actions(rng, n, C), _ptr([n // 2, n - n // 2]))


def test_preference_gradient_against_differences(ctx):
    rng = np.random.default_rng(6)
    lengths, C = [3, 2, 1, 4], 11
    n = int(np.sum(lengths))
    z, a, ptr = _logits(rng, n, C, F32, 1.0), _dev(_actions(rng, n, C)), _dev(_ptr(lengths))
    work = torch.zeros(n, 4, device="cuda")

    def loss(y, g=None):
        out = torch.zeros(2, device="cuda")
        ctx.gsplit_preference_loss(y, a, ptr, g, work, beta=0.5, label_smoothing=0.1, pair_loss=out)
        return out.double().sum()

    g = torch.zeros(n, C, device="cuda")
    loss(z.cuda(), g)
    h = 2.0 ** -7
    for r in range(n):
        c = int(a[r])
        up, down = z.cuda(), z.cuda()
        up[r, c] += h
        down[r, c] -= h
        diff = float((loss(up) - loss(down)) / (up[r, c] - down[r, c]).double())
        # third derivatives of at most 1 by a logit; losses up to 4, off by 100 u
        assert abs(diff - float(g[r, c])) < h * h / 6 * 2 + 2 * 4 * 100 * K.U / (2 * h)


# -- the ways a caller runs them ------------------------------------------------------------------

def _calls(ctx, n, C, dtype, seed):
    """A function that runs both losses on inputs it may be given anew, and the outputs it writes."""
    rng = np.random.default_rng(seed)
    z = _dev(_logits(rng, n, C, dtype))
    a = _dev(_actions(rng, n, C))
    old, adv = _dev(rng.standard_normal(n).astype(np.float32) - 4), _dev(rng.standard_normal(n).astype(np.float32))
    ptr = _dev(_ptr([n // 4, n // 4, n // 4, n - 3 * (n // 4)]))
    outs = [torch.zeros(n, C, dtype=dtype, device="cuda") for _ in range(2)] + [torch.zeros(n, device="cuda") for _ in range(2)] + [
        torch.zeros(2, device="cuda")]
    work = torch.zeros(n, 4, device="cuda")

    def run(c=ctx):
        c.gsplit_policy_loss(z, a, old, adv, outs[0], ref_logp=old, kl_coef=0.1, row_loss=outs[2])
        c.gsplit_preference_loss(z, a, ptr, outs[1], work, row_logp=outs[3], pair_loss=outs[4])

    return run, outs, z


SHAPES = [(64, 47, F32), (700, 172, BF16), (100, 2000, F32), (4, 66000, F32), (2, 140001, BF16), (300, 17001, BF16)]


@pytest.mark.parametrize("n, C, dtype", SHAPES)
def test_same_bits_every_time_and_on_another_stream(ctx, n, C, dtype):
    run, outs, z = _calls(ctx, n, C, dtype, 3)
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    for t in outs:
        t.fill_(9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("n, C, dtype", SHAPES)
def test_captured_and_replayed(ctx, n, C, dtype):
    """Replays with new logits, eager calls of the same context and synchronisations between them."""
    run, outs, z = _calls(ctx, n, C, dtype, 4)
    other, _, _ = _calls(ctx, 50, 70001, F32, 5)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    rng = np.random.default_rng(9)
    for k in range(4):
        z.copy_(_logits(rng, n, C, dtype))
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for t in outs:
            t.fill_(9)
        if k % 2:
            other()
        g.replay()
        if k > 1:
            torch.cuda.synchronize()
        other()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), k


def test_two_contexts_on_two_streams(ctx):
    """Calls that overlap in time, each with the scratch of its own context."""
    c2 = K.context()
    jobs = [_calls(c, 3, 90001, F32, 11 + k) for k, c in enumerate((ctx, c2))]
    want = []
    for (run, outs, _), c in zip(jobs, (ctx, c2)):
        run(c)
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs])
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(10):
        for (run, outs, _), c, s in zip(jobs, (ctx, c2), streams):
            with torch.cuda.stream(s):
                run(c)
    torch.cuda.synchronize()
    for (run, outs, _), w in zip(jobs, want):
        assert all(torch.equal(a, b) for a, b in zip(outs, w))
    c2.close()


def test_no_rows_and_refusals(ctx):
    from paper_2303_13775_amd import GsplitError
    z0, a0, f0 = torch.zeros(0, 5, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, device="cuda")
    ctx.gsplit_policy_loss(z0, a0, f0, f0, z0)
    loss = torch.full((1,), 9.0, device="cuda")
    ctx.gsplit_preference_loss(z0, a0, torch.zeros(3, dtype=torch.int64, device="cuda"), z0, torch.zeros(0, 4, device="cuda"), pair_loss=loss)
    assert abs(float(loss) - np.log(2)) < 1e-6          # two empty sequences: margin 0
    ctx.gsplit_preference_loss(z0, a0, torch.zeros(1, dtype=torch.int64, device="cuda"), z0, torch.zeros(0, 4, device="cuda"))
    z, a, f = torch.zeros(2, 5, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(2, device="cuda")
    for kw in (dict(kl_coef=0.1), dict(clip_low=1.5), dict(clip_high=-0.1), dict(kl_coef=float("nan"), ref_logp=f)):
        with pytest.raises(GsplitError) as e:
            ctx.gsplit_policy_loss(z, a, f, f, z, **kw)
        assert e.value.code == -1 and "gsplit_policy_loss" in str(e.value)
    ptr = torch.tensor([0, 1, 2], device="cuda")
    for kw in (dict(beta=float("inf")), dict(label_smoothing=2.0)):
        with pytest.raises(GsplitError) as e:
            ctx.gsplit_preference_loss(z, a, ptr, z, torch.zeros(2, 4, device="cuda"), **kw)
        assert e.value.code == -1 and "gsplit_preference_loss" in str(e.value)
    for bad in (lambda: ctx.gsplit_policy_loss(z.half(), a, f, f, None), lambda: ctx.gsplit_policy_loss(z, a.int(), f, f, None),
                lambda: ctx.gsplit_policy_loss(z, a, f[:1], f, None), lambda: ctx.gsplit_policy_loss(z, a, f, f, z.bfloat16()),
                lambda: ctx.gsplit_policy_loss(z.t(), a, f, f, None), lambda: ctx.gsplit_preference_loss(z, a, ptr[:2], None, z)):
        with pytest.raises(AssertionError):
            bad()
    ctx.gsplit_policy_loss(z, a, f, f, z.clone())       # the context stays usable
    torch.cuda.synchronize()


def test_rows_behind_32_bits_of_elements(ctx):
    """Logits of more than 2^31 elements, whose last rows lie more than 4 GiB into the buffers: the bits of a call on those rows alone."""
    n, C = 32800, 65537
    z = torch.empty(n, C, dtype=BF16, device="cuda")
    for i in range(0, n, 4100):
        z[i:i + 4100].normal_(generator=torch.Generator(device="cuda").manual_seed(i))
    g = torch.empty_like(z)
    a = (torch.arange(n, device="cuda") * 7919) % C
    old, adv = torch.full((n,), -11.0, device="cuda"), torch.ones(n, device="cuda")
    w, logp = torch.full((n,), 0.25, device="cuda"), torch.zeros(n, device="cuda")
    ctx.gsplit_policy_loss(z, a, old, adv, g, row_weight=w, row_logp=logp, clip_high=50.0)
    ptr, work, plogp = torch.tensor([0, n - 300, n], device="cuda"), torch.zeros(n, 4, device="cuda"), torch.zeros(n, device="cuda")
    for lo in (0, n - 300):         # (as many rows as take the same form)
        few = slice(lo, lo + 300)
        g1, logp1 = torch.zeros(300, C, dtype=BF16, device="cuda"), torch.zeros(300, device="cuda")
        ctx.gsplit_policy_loss(z[few].clone(), a[few].clone(), old[few].clone(), adv[few].clone(), g1, row_weight=w[few].clone(), row_logp=logp1, clip_high=50.0)
        assert torch.equal(g[few], g1) and torch.equal(logp[few], logp1) and bool(g1.any(1).all())
    g.fill_(3.0)
    ctx.gsplit_preference_loss(z, a, ptr, g, work, beta=1e-4, row_logp=plogp)
    assert float((plogp - logp).abs().max()) < 1e-5
    for r in (0, n - 301, n - 300, n - 1):
        slope = float(work[r, 2])               # (where the call leaves it)
        assert (slope < 0) == (r < n - 300)
        p = torch.softmax(z[r].double(), 0)
        p[a[r]] -= 1.0
        assert slope and float((g[r].double() + slope * p).abs().max()) <= 2.0 ** -8 * abs(slope) + 1e-12, r


def test_capture_with_timing_on(ctx):
    """Calls under capture take no timing, whatever is enabled; eager ones around them do."""
    run, outs, _ = _calls(ctx, 64, 47, F32, 2)
    ctx.gsplit_timing_enable(True)
    ctx.gsplit_timing_read()
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for t in outs:
        t.fill_(9)
    g.replay()
    run()
    torch.cuda.synchronize()
    got = ctx.gsplit_timing_read()
    ctx.gsplit_timing_enable(False)
    assert got["policy_loss"][0] == 2 and all(torch.equal(a, b) for a, b in zip(outs, want))


def test_timing_labels(ctx):
    run, _, _ = _calls(ctx, 64, 47, F32, 1)
    ctx.gsplit_timing_enable(True)
    run()
    got = ctx.gsplit_timing_read()
    ctx.gsplit_timing_enable(False)
    assert "policy_loss" in got and any(k.startswith("preference") for k in got)
