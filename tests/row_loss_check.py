"""Inputs of the losses over rows of logits, and how far their results may be from float64 (not a test module itself).

With u = 2^-24 (half a step of a float) and x = z_c - max z: the difference rounds by u |x|, its product with log2(e) and that
constant by 2 u |x|, the exponential by 2 u of its own and 2 u more for the steps around it: rel_exp(x) <= u (3 |x| + 4).  A sum
of exponentials is off by the mean of that, weighted with the probabilities, and by u for each addition a value goes through:
at most max(C / 256, 64) in its thread and 16 in joining the threads.  That is the error of log p before its own rounding (the
rest of a row is double); a slope and a loss follow with their derivatives by log p, and each value is then rounded once more to
its type."""
import numpy as np
import torch

U = 2.0 ** -24
EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}        # half a step, relative
TINY = 1e-36


def context():
    """A context for calls that need no batch: its graph is one vertex."""
    from paper_2303_13775_amd import Context
    assert torch.cuda.is_available(), "these tests need the MI355X"
    dev = torch.device("cuda:0")
    return Context(torch.zeros(2, dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev),
                   torch.zeros(1, dtype=torch.uint8, device=dev), 1, [1], 1)


def rows_buffer(values, dtype, pad=0, offset=0, fill=7.0):
    """(whole buffer, view [rows, C]) on the GPU, rows `pad` values further apart than C, `offset` values into the buffer."""
    n, C = values.shape
    whole = torch.full((offset + n * (C + pad) + 3,), fill, dtype=dtype, device="cuda")
    view = torch.as_strided(whole, (n, C), (C + pad, 1), offset)
    view.copy_(values.to(dtype))
    return whole, view


def untouched(whole, view, fill=7.0):
    """Whether everything around the view holds what it was filled with."""
    mask = torch.ones_like(whole, dtype=torch.bool)
    torch.as_strided(mask, view.shape, view.stride(), view.storage_offset()).fill_(False)
    return bool((whole[mask] == fill).all())


def terms(z, slope):
    """(error of log p, error of a gradient of this slope apart from its last rounding) of every row, from its float64 logits."""
    C = z.shape[1]
    with np.errstate(invalid="ignore", over="ignore"):
        x = z - np.max(z, axis=1, keepdims=True)
        e = np.exp(x)
        p = e / e.sum(1, keepdims=True)
        rel = U * (3 * np.where(np.isfinite(x), np.abs(x), 0.0) + 4)
        dlp = (p * rel).sum(1) + U * (max(C / 256, 64) + 16)
        dgrad = np.abs(slope)[:, None] * p * (rel + dlp[:, None] + 4 * U)
    return dlp, dgrad


def check(name, got, want, tol, dtype=torch.float32):
    """|got - want| within tol plus the rounding to its type; NaN where the other is NaN."""
    got = got.detach().double().cpu().numpy()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    assert (np.isnan(got) == np.isnan(want)).all(), (name, "NaN", np.argwhere(np.isnan(got) != np.isnan(want))[:4])
    fine = ~np.isnan(want)
    same = got == want
    with np.errstate(invalid="ignore"):
        over = np.abs(got - want) - (tol + (EPS[dtype] + U) * np.abs(want) + TINY)
    bad = fine & ~same & ~(over <= 0)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])


def away_from_borders(logp, old, clip_low, clip_high, by=1e-3):
    """old, changed where the ratio is within `by` of a border of the clip (which side it lies on is not decided by floats)."""
    ratio = np.exp(logp - old)
    near = (np.abs(ratio - (1 - clip_low)) < by) | (np.abs(ratio - (1 + clip_high)) < by)
    return np.where(near, logp - 0.01, old).astype(np.float32)
