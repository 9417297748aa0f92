"""Performance cases of the operators at the two ends of a training step: losses with their gradients
before the backward pass, and behind it the norm over all gradients, clipping and the update.

A case is one call.  Class counts, batches and layer widths come from the repository's own workloads
(`workloads/synth.py`: 47 and 172 classes, batches of 1024 to 8192, widths 64 to 256) where it is one of
theirs; the wider ones are generic.  Keys of a case:

  op         policy      clipped policy loss with a KL term, and its gradient by the logits
             preference  loss of paired log ratios over ragged sequences of rows, and its gradient
             clip        global norm over many gradient tensors, and the clipped gradients
             adamw       the same norm with the clipped AdamW update of the parameters
  rows, classes, pad      logits [rows x classes], rows `classes + pad` values apart
  dtype      "f32" or "bf16" logits and their gradient; clip, adamw: "f32", "bf16" or "mixed" (half the
             elements each; a bf16 parameter has a float copy that is updated, moments are float)
  kl         weight of the KL term (0: none, and no reference)
  masked     share of the rows that take no part: weight 0 (policy), no action (preference)
  pairs, longest, spare   preference: pairs of sequences of 1 .. `longest` rows (some of none), and the
             rows of the buffers behind the last sequence
  dims       clip, adamw: the gradients of a GraphSAGE model of these widths
  tensors, elements       or that many tensors of all sizes with that many elements together
  clipped    the norm exceeds the bound
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

CLIP_LOW, CLIP_HIGH = 0.2, 0.25
BETA, SMOOTHING = 0.1, 0.05
LR, BETA1, BETA2, EPS, DECAY, STEP = 1e-3, 0.9, 0.999, 1e-8, 0.01, 1000
MAX_NORM = 1.0
MOST_LOGITS = 8192 * 65536          # of a drawn case, as of the largest listed one
MOST_ELEMENTS = 400_000_000

_POLICY = {"op": "policy", "rows": 1024, "classes": 47, "pad": 0, "dtype": "f32", "kl": 0.04, "masked": 0.1}
_PREFERENCE = {"op": "preference", "pairs": 512, "longest": 1, "spare": 0, "classes": 47, "pad": 0, "dtype": "f32",
               "masked": 0.0}
_TENSORS = {"dims": "", "tensors": 0, "elements": 0, "dtype": "f32", "clipped": True}


def listed():
    return [
        # a batch of the benchmark workload: latency is all of it
        dict(_POLICY, name="policy_1024x47"),
        # one row with many classes, as a loop that samples one action at a time has it: the row is the only parallel axis
        dict(_POLICY, name="policy_1x65537_bf16", rows=1, classes=65537, dtype="bf16", masked=0.0),
        # the largest batch of the sweep workload, no reference model
        dict(_POLICY, name="policy_8192x172", rows=8192, classes=172, kl=0.0),
        # rows of odd length in a padded buffer, bf16
        dict(_POLICY, name="policy_4095x50001_bf16", rows=4095, classes=50001, pad=15, dtype="bf16"),
        # the largest
        dict(_POLICY, name="policy_8192x65536", rows=8192, classes=65536),
        # ranking pairs of target vertices
        dict(_PREFERENCE, name="preference_512x47"),
        # paths through the graph, 1 to 32 vertices each, and room behind them
        dict(_PREFERENCE, name="preference_256_of_32x172", pairs=256, longest=32, spare=100, classes=172),
        # long ragged sequences with many classes, the rows of the prompts left out
        dict(_PREFERENCE, name="preference_16_of_512x32768_bf16", pairs=16, longest=512, classes=32768, dtype="bf16",
             masked=0.3),
        # gradients of the tiny workload's model
        dict(_TENSORS, name="clip_sage_tiny", op="clip", dims="64,64,16"),
        # many tensors of two types and all sizes
        dict(_TENSORS, name="clip_387_mixed", op="clip", tensors=387, elements=400_000_000, dtype="mixed"),
        # the update of the benchmark workload's model
        dict(_TENSORS, name="adamw_sage_medium", op="adamw", dims="100,256,256,47"),
        # a large model's update, bf16 parameters with a float copy among them
        dict(_TENSORS, name="adamw_150_mixed", op="adamw", tensors=150, elements=250_000_000, dtype="mixed"),
    ]


def draw(rng: random.Random):
    """One more case of the ranges the listed ones span."""
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["policy", "policy", "preference", "clip", "adamw"])
    if op == "policy":
        c = dict(_POLICY, rows=log_uniform(1, 32768), classes=log_uniform(2, 131072), pad=rng.choice([0, 0, 0, 1, 8, 33]),
                 dtype=rng.choice(["f32", "bf16"]), kl=rng.choice([0.0, 0.01, 0.04, 0.1]), masked=rng.choice([0.0, 0.1, 0.5]))
        c["rows"] = max(1, min(c["rows"], MOST_LOGITS // c["classes"]))
        if c["rows"] < 64:      # a few rows all of which are left out would be no work
            c["masked"] = 0.0
    elif op == "preference":
        c = dict(_PREFERENCE, pairs=log_uniform(1, 2048), longest=log_uniform(1, 1024), spare=rng.choice([0, 0, 1, 50]),
                 classes=log_uniform(2, 65536), pad=rng.choice([0, 0, 1, 8]), dtype=rng.choice(["f32", "bf16"]),
                 masked=rng.choice([0.0, 0.3]))
        c["longest"] = max(1, min(c["longest"], 32768 // c["pairs"]))
        c["classes"] = max(2, min(c["classes"], MOST_LOGITS // 2 // (c["pairs"] * c["longest"])))
    else:
        c = dict(_TENSORS, op=op, dtype=rng.choice(["f32", "f32", "bf16", "mixed"]), clipped=rng.random() < 0.7)
        if rng.random() < 0.4:
            hidden = rng.randint(30, 512)
            c["dims"] = ",".join(str(x) for x in [rng.randint(30, 256)] + [hidden] * rng.randint(0, 3) + [rng.randint(5, 180)])
        else:
            c["elements"] = log_uniform(2000, MOST_ELEMENTS if op == "clip" else MOST_ELEMENTS // 2)
            c["tensors"] = min(log_uniform(1, 500), c["elements"] // 8)
    return c


# -- what a case consists of -------------------------------------------------------------------

def _lengths(c):
    """Rows of the sequences 2 p (chosen) and 2 p + 1 (rejected) of every pair p."""
    rng = random.Random(f"{c['pairs']} {c['longest']}")
    if c["longest"] == 1:
        return [1] * (2 * c["pairs"])
    return [0 if rng.random() < 0.02 else rng.randint(1, c["longest"]) for _ in range(2 * c["pairs"])]


def _tensor_sizes(c):
    if c["dims"]:
        d = [int(x) for x in c["dims"].split(",")]
        pairs = list(zip(d, d[1:]))
        return [a * b for a, b in pairs] * 2 + [b for _, b in pairs]
    rng = random.Random(f"{c['tensors']} {c['elements']}")
    parts = [math.exp(rng.uniform(0.0, 6.0)) for _ in range(c["tensors"])]
    sizes = [max(1, int(c["elements"] * p / sum(parts))) for p in parts]
    sizes[0] += max(0, c["elements"] - sum(sizes))
    return sizes


def _halves(c):
    """The tensors' sizes of either type: (float, bfloat16)."""
    sizes = _tensor_sizes(c)
    return (sizes, []) if c["dtype"] == "f32" else ([], sizes) if c["dtype"] == "bf16" else (sizes[0::2], sizes[1::2])


def work(c):
    if c["op"] in ("policy", "preference"):
        rows = c["rows"] if c["op"] == "policy" else sum(_lengths(c))
        size = 4 if c["dtype"] == "f32" else 2
        read = rows * (1.0 - c["masked"])
        per_row = 8 + 4 * 7 if c["op"] == "policy" else 8 + 4
        return {"bytes": (read + rows) * c["classes"] * size + rows * per_row, "flops": 6 * read * c["classes"]}
    n32, n16 = (sum(s) for s in _halves(c))
    if c["op"] == "clip":
        return {"bytes": 8 * n32 + 4 * n16, "flops": 3 * (n32 + n16)}
    # parameter (float; or the float copy, read and written, and the bfloat16 one, written), two moments, gradient
    return {"bytes": (4 * 6 + 4) * n32 + (4 * 6 + 2 + 2) * n16, "flops": 15 * (n32 + n16)}


_kept = {}


def _context():
    """The program's context.  These calls need no batch of it, so its graph is a single vertex."""
    if "ctx" not in _kept:
        from paper_2303_13775_amd import Context
        dev = torch.device("cuda")
        _kept["ctx"] = Context(torch.zeros(2, dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev),
                               torch.zeros(1, dtype=torch.uint8, device=dev), 1, [1], 1)
    return _kept["ctx"]


def _row_terms(logits, actions):
    """Per row: maximum, exponentials above it (float), their sum, and the action's log-probability in 64 bits."""
    z = logits.float()
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1)
    at = actions.clamp(0, z.shape[1] - 1)[:, None]
    logp = (z.gather(1, at).double() - top.double())[:, 0] - torch.log(total.double())
    return e, total, logp


def _logits(c, rows, gen, dev):
    """Logits of a trained model: spread wide enough that the classes of a row differ by some powers of ten."""
    wide = c["classes"] + c["pad"]
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    z = torch.randn((rows, wide), device=dev, generator=gen).mul_(2.0).to(dt)
    grad = torch.zeros((rows, wide), dtype=dt, device=dev)
    return z[:, :c["classes"]], grad[:, :c["classes"]]


def _actions(logits, gen):
    """Actions as a policy picks them: the likeliest of a few drawn at random."""
    rows, classes = logits.shape
    few = torch.randint(0, classes, (rows, 8), device=logits.device, generator=gen)
    return few.gather(1, logits.gather(1, few).float().argmax(1, keepdim=True))[:, 0].contiguous()


def prepare(c, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed * 1000003 + 17)
    s = SimpleNamespace(c=c)

    def normal(n, scale=1.0):
        return torch.randn(n, device=dev, generator=gen).mul_(scale)

    if c["op"] == "policy":
        rows = c["rows"]
        s.logits, s.grad = _logits(c, rows, gen, dev)
        s.actions = _actions(s.logits, gen)
        logp = _row_terms(s.logits, s.actions)[2]
        # the policy has moved since the actions were drawn.  A ratio within 1e-3 of the clip's borders is
        # moved off: 32 bits do not say on which side it lies
        moved = normal(rows, 0.2).double()
        ratio = torch.exp(moved)
        near = ((ratio - (1 - CLIP_LOW)).abs() < 1e-3) | ((ratio - (1 + CLIP_HIGH)).abs() < 1e-3)
        s.old_logp = (logp - torch.where(near, 0.01, moved)).float()
        s.ref_logp = (logp + normal(rows, 0.3).double()).float() if c["kl"] else None
        s.advantage = normal(rows)
        used = torch.rand(rows, device=dev, generator=gen) >= c["masked"]
        s.weight = used.float() / used.sum().clamp(min=1)
        s.row_loss, s.row_logp, s.row_kl = (torch.zeros(rows, device=dev) for _ in range(3))
    elif c["op"] == "preference":
        lengths = torch.tensor(_lengths(c))
        s.seq_ptr = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)]).to(dev)
        n = int(lengths.sum())
        rows = n + c["spare"]
        s.logits, s.grad = _logits(c, rows, gen, dev)
        s.actions = _actions(s.logits, gen)
        s.actions[torch.rand(rows, device=dev, generator=gen) < c["masked"]] = -1
        logp = torch.where(s.actions >= 0, _row_terms(s.logits, s.actions)[2], 0.0)
        summed = torch.cat([logp.new_zeros(1), logp.cumsum(0)])[s.seq_ptr]
        s.ref_logp = ((summed[1:] - summed[:-1]) + normal(2 * c["pairs"], 3.0).double()).float()
        s.weight = torch.full((c["pairs"],), 1.0 / c["pairs"], device=dev)
        s.pair_loss, s.pair_margin = (torch.zeros(c["pairs"], device=dev) for _ in range(2))
        s.row_logp = torch.zeros(rows, device=dev)
        s.row_work = torch.zeros((rows, 4), device=dev)
    else:
        s.sizes = _halves(c)
        n = [sum(x) for x in s.sizes]
        types = (torch.float32, torch.bfloat16)
        spread = (3.7 if c["clipped"] else 0.25) * MAX_NORM / math.sqrt(sum(n))
        s.grads = [normal(k, spread).to(t) for k, t in zip(n, types)]
        s.norm = torch.zeros(1, device=dev)
        if c["op"] == "clip":
            s.outs = [torch.zeros_like(g) for g in s.grads]
        else:
            s.params = [normal(k, 0.05) for k in n]         # float: the parameters, and the copies of the bfloat16 ones
            s.half = s.params[1].bfloat16()
            s.m = [normal(k, 0.3 * spread) for k in n]
            s.v = [normal(k, spread).square_() for k in n]
    if own:
        s.ctx = _context()
        if c["op"] in ("clip", "adamw"):
            from paper_2303_13775_amd import AdamwTensors, GradTensors

            def tensors(two):
                return [t for flat, sizes in zip(two, s.sizes) if sizes for t in torch.split(flat, sizes)]

            if c["op"] == "clip":
                s.table = GradTensors(tensors(s.grads), tensors(s.outs))
            else:
                n32 = len(s.sizes[0])
                copies = tensors(s.params)
                params = copies[:n32] + (list(torch.split(s.half, s.sizes[1])) if s.sizes[1] else [])
                s.table = AdamwTensors(params, tensors(s.grads), tensors(s.m), tensors(s.v),
                                       [None] * n32 + copies[n32:])
    return s


# -- the plain forms ---------------------------------------------------------------------------

def _gradient(like, e, total, coef, actions):
    """coef (1[c = action] - p) for every row; rows whose coefficient is 0 take no part."""
    coef = coef.float()
    grad = e * (-coef / total)[:, None]
    grad.scatter_add_(1, actions.clamp(0, grad.shape[1] - 1)[:, None], coef[:, None])
    return grad.to(like.dtype)


def _policy_terms(s, logp):
    """(loss, KL term, d loss / d log-probability) per row, in the type of logp."""
    c = s.c
    w, adv = s.weight.to(logp.dtype), s.advantage.to(logp.dtype)
    ratio = torch.exp(logp - s.old_logp.to(logp.dtype))
    free = -adv * ratio
    held = -adv * ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH)
    loss = torch.maximum(free, held)
    slope = torch.where(free >= held, free, 0.0)
    kl = torch.zeros_like(logp)
    if c["kl"]:
        d = s.ref_logp.to(logp.dtype) - logp
        kl = torch.expm1(d) - d
        loss = loss + c["kl"] * kl
        slope = slope - c["kl"] * torch.expm1(d)
    used = w != 0
    return w * loss, torch.where(used, kl, 0.0), w * slope, used


def _plain_policy(s):
    e, total, logp = _row_terms(s.logits, s.actions)
    loss, kl, coef, used = _policy_terms(s, logp)
    grad = _gradient(s.logits, e, total, coef, s.actions)
    return {"grad": grad, "loss": loss.float(), "logp": torch.where(used, logp, 0.0).float(), "kl": kl.float()}


def _pair_terms(s, logp):
    """(loss, margin, d loss / d log-probability of every row) in the type of logp."""
    summed = torch.cat([logp.new_zeros(1), logp.cumsum(0)])[s.seq_ptr]
    gap = (summed[1:] - summed[:-1]) - s.ref_logp.to(logp.dtype)
    margin = BETA * (gap[0::2] - gap[1::2])
    w = s.weight.to(logp.dtype)
    soft = torch.clamp(-margin.abs(), max=0.0).exp().log1p()
    loss = w * ((1 - SMOOTHING) * (soft + torch.clamp(-margin, min=0.0)) + SMOOTHING * (soft + torch.clamp(margin, min=0.0)))
    slope = BETA * w * (SMOOTHING - 1.0 / (1.0 + torch.exp(margin)))
    row = torch.arange(logp.shape[0], device=logp.device)
    seq = torch.searchsorted(s.seq_ptr, row, right=True) - 1
    inside = (seq >= 0) & (seq < s.ref_logp.shape[0])
    sign = 1.0 - 2.0 * (seq % 2).to(logp.dtype)
    coef = torch.where(inside & (s.actions >= 0), sign * slope[(seq // 2).clamp(0, slope.shape[0] - 1)], 0.0)
    return loss, margin, coef, inside


def _plain_preference(s):
    e, total, logp = _row_terms(s.logits, s.actions)
    logp = torch.where(s.actions >= 0, logp, 0.0)
    loss, margin, coef, inside = _pair_terms(s, logp)
    return {"grad": _gradient(s.logits, e, total, coef, s.actions), "loss": loss.float(), "margin": margin.float(),
            "logp": torch.where(inside, logp, 0.0).float()}


def _norm_and_factor(s):
    a, b = (torch.sum(g.float() * g.float(), dtype=torch.float64) for g in s.grads)
    norm = torch.sqrt(a + b).float()
    return norm[None], torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)


def _plain_clip(s):
    norm, factor = _norm_and_factor(s)
    return {"norm": norm, "out32": s.grads[0] * factor, "out16": (s.grads[1].float() * factor).bfloat16()}


def _plain_adamw_part(p, m, v, g, factor):
    g = g.float() * factor
    m.mul_(BETA1).add_(g * (1 - BETA1))
    v.mul_(BETA2).add_(g * g * (1 - BETA2))
    root = torch.sqrt(v * (1 / (1 - BETA2 ** STEP))).add_(EPS)
    p.mul_(1 - LR * DECAY).sub_(m * (LR / (1 - BETA1 ** STEP)) / root)


def _adamw_outputs(s):
    return {"norm": s.norm, "half": s.half, **{f"{n}{k}": t for n in ("params", "m", "v") for k, t in enumerate(getattr(s, n))}}


def _plain_adamw(s):
    s.norm, factor = _norm_and_factor(s)
    _plain_adamw_part(s.params[0], s.m[0], s.v[0], s.grads[0], factor)
    _plain_adamw_part(s.params[1], s.m[1], s.v[1], s.grads[1], factor)
    s.half.copy_(s.params[1])
    return _adamw_outputs(s)


_PLAIN = {"policy": _plain_policy, "preference": _plain_preference, "clip": _plain_clip, "adamw": _plain_adamw}


def run(s):
    op = s.c["op"]
    if not own:
        return _PLAIN[op](s)
    if op == "policy":
        s.ctx.gsplit_policy_loss(s.logits, s.actions, s.old_logp, s.advantage, s.grad, ref_logp=s.ref_logp, row_weight=s.weight,
                                 clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=s.c["kl"], row_loss=s.row_loss,
                                 row_logp=s.row_logp, row_kl=s.row_kl)
        return {"grad": s.grad, "loss": s.row_loss, "logp": s.row_logp, "kl": s.row_kl}
    if op == "preference":
        s.ctx.gsplit_preference_loss(s.logits, s.actions, s.seq_ptr, s.grad, ref_logp=s.ref_logp, pair_weight=s.weight,
                                     beta=BETA, label_smoothing=SMOOTHING, pair_loss=s.pair_loss, pair_margin=s.pair_margin,
                                     row_logp=s.row_logp, row_work=s.row_work)
        return {"grad": s.grad, "loss": s.pair_loss, "margin": s.pair_margin, "logp": s.row_logp}
    if op == "clip":
        s.ctx.gsplit_clip_grads(s.table, MAX_NORM, s.norm)
        return {"norm": s.norm, "out32": s.outs[0], "out16": s.outs[1]}
    s.ctx.gsplit_adamw_step(s.table, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY, step=STEP,
                            max_norm=MAX_NORM, norm=s.norm)
    return _adamw_outputs(s)


# -- the definition in 64 bits, row block by row block -------------------------------------------

def _exact_rows(logits, actions, then):
    """log-probabilities of all rows, and then(log-probabilities) (1[c = action] - p) in blocks of rows."""
    rows, classes = logits.shape
    step = max(1, (1 << 27) // classes)
    at = actions.clamp(0, classes - 1)
    logp = torch.cat([torch.log_softmax(logits[i:i + step].double(), 1).gather(1, at[i:i + step, None])[:, 0]
                      for i in range(0, rows, step)])
    extra, coef = then(logp)
    grad = torch.empty((rows, classes), dtype=torch.float64, device=logits.device)
    for i in range(0, rows, step):
        p = torch.softmax(logits[i:i + step].double(), 1).neg_()
        p[torch.arange(p.shape[0], device=p.device), at[i:i + step]] += 1.0
        grad[i:i + step] = p * coef[i:i + step, None]
    return dict(extra, grad=grad)


def _exact_policy(s):
    def then(logp):
        adv, w, old = s.advantage.double(), s.weight.double(), s.old_logp.double()
        ratio = (logp - old).exp()
        # an advantage above 0 gains nothing from a ratio over 1 + high, one below 0 nothing from one under 1 - low
        held = torch.where(adv >= 0, ratio > 1 + CLIP_HIGH, ratio < 1 - CLIP_LOW)
        kept = torch.where(adv >= 0, ratio.clamp(max=1 + CLIP_HIGH), ratio.clamp(min=1 - CLIP_LOW))
        kl = torch.zeros_like(logp)
        slope = torch.where(held, 0.0, -adv * ratio)
        if s.c["kl"]:
            towards = (s.ref_logp.double() - logp).exp()
            kl = towards - 1 - (s.ref_logp.double() - logp)
            slope = slope + s.c["kl"] * (1 - towards)
        out = w == 0
        return {"loss": w * (-adv * kept + s.c["kl"] * kl), "logp": logp.masked_fill(out, 0.0),
                "kl": kl.masked_fill(out, 0.0)}, w * slope
    return _exact_rows(s.logits, s.actions, then)


def _exact_preference(s):
    def then(logp):
        logp = logp.masked_fill(s.actions < 0, 0.0)
        ptr = s.seq_ptr.tolist()
        sums = torch.stack([logp[a:b].sum() for a, b in zip(ptr, ptr[1:])])
        margin = BETA * ((sums[0::2] - sums[1::2]) - (s.ref_logp[0::2].double() - s.ref_logp[1::2].double()))
        chosen, rejected = torch.sigmoid(margin), torch.sigmoid(-margin)
        w = s.weight.double()
        loss = -w * ((1 - SMOOTHING) * torch.nn.functional.logsigmoid(margin)
                     + SMOOTHING * torch.nn.functional.logsigmoid(-margin))
        slope = BETA * w * (SMOOTHING * chosen - (1 - SMOOTHING) * rejected)
        per_seq = torch.stack([slope, -slope], 1).reshape(-1)
        lengths = s.seq_ptr[1:] - s.seq_ptr[:-1]
        coef = torch.zeros_like(logp)
        coef[ptr[0]:ptr[-1]] = torch.repeat_interleave(per_seq, lengths)
        coef[s.actions < 0] = 0.0
        logp = logp.clone()
        logp[ptr[-1]:] = 0.0
        return {"loss": loss, "margin": margin, "logp": logp}, coef
    return _exact_rows(s.logits, s.actions, then)


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "policy":
        return _exact_policy(s)
    if c["op"] == "preference":
        return _exact_preference(s)
    grads = [g.double() for g in s.grads]
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g) for g in grads]))
    scaled = [g * min(1.0, MAX_NORM / float(norm)) for g in grads]
    if c["op"] == "clip":
        return {"norm": norm[None], "out32": scaled[0], "out16": scaled[1]}
    out = {"norm": norm[None]}
    for k, g in enumerate(scaled):
        m = BETA1 * s.m[k].double() + (1 - BETA1) * g
        v = BETA2 * s.v[k].double() + (1 - BETA2) * g * g
        change = (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
        p = s.params[k].double()
        out[f"params{k}"], out[f"m{k}"], out[f"v{k}"] = p - LR * (change + DECAY * p), m, v
    return dict(out, half=out["params1"])
