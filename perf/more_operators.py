"""Performance cases of the operators for models whose weights come in stacks, a matrix for every type of vertex,
task or expert: the rows sorted by group, the grouped products forward and backward, and the update of matrices
by orthogonalised momentum, with the orthogonalisation by itself.

A case is one call.  Batches, widths and class counts come from the repository's own workloads
(`workloads/synth.py`: batches of 1024 to 8192, widths 64 to 256, 47 and 172 classes) where it is one of theirs;
the wider ones are generic.  Keys of a case:

  op         group     rows sorted by their group: offsets of the groups and the rows in their order
             forward   y[r] = x[r] W[g] + b[g] for the rows r of every group g
             backward  the gradients of x, W and b of the same product
             orth      matrices orthogonalised by Newton-Schulz steps
             muon      momentum, its orthogonalisation, and the update of parameters with weight decay
  rows, groups            rows and the groups they are dealt to
  skew                    group g gets a share of (g + 1)^-skew of the rows, in an order of its own
  left_out                share of the rows that belong to no group
  sorted                  the rows lie sorted by group already: no list of rows
  n_in, n_out, pad        widths of the product; rows of x and y are `pad` values apart
  dtype                   "f32" or "bf16": x, W, y and their gradients (bias and gradients of W and b are
                          float); orth: the matrices; muon: "f32", "bf16" or "mixed" (every other tensor;
                          a bf16 parameter has a float copy that is updated, its gradient is bf16)
  shapes                  orth, muon: "COUNTxROWSxCOLS,..." stacks of matrices
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

STEPS, A, B, C, EPS = 5, 3.4445, -4.7750, 2.0315, 1e-7
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01
MOST_PRODUCT = 65536 * 2048 * 2048      # multiply-adds of a drawn product, as of the largest listed one
MOST_NEWTON = 1.2e12                    # the same of a drawn update's steps

_GROUPED = {"rows": 1024, "groups": 4, "skew": 0.5, "left_out": 0.0, "sorted": False, "n_in": 256, "n_out": 47, "pad": 0,
            "dtype": "f32"}
_MATRICES = {"shapes": "", "dtype": "f32"}


def listed():
    return [
        # the targets of a batch by type
        dict(_GROUPED, name="group_1024_of_4", op="group"),
        # the input vertices of a large batch by type, some of no type that counts
        dict(_GROUPED, name="group_1000003_of_64", op="group", rows=1000003, groups=64, skew=1.0, left_out=0.1),
        # answers for a few vertices, each with the head of its type: latency is all of it
        dict(_GROUPED, name="forward_33_of_8_256x47", op="forward", rows=33, groups=8),
        # the batch of the large workload, heads by type, its classes
        dict(_GROUPED, name="forward_4096_of_16_256x172", op="forward", rows=4096, groups=16, skew=1.0, n_out=172),
        # projections of many rows that a sort has left in order
        dict(_GROUPED, name="forward_60000_of_8_512x512", op="forward", rows=60000, groups=8, skew=1.0, sorted=True, n_in=512,
             n_out=512),
        # experts' products of a large batch in bf16: the largest
        dict(_GROUPED, name="forward_65536_of_64_2048x2048_bf16", op="forward", rows=65536, groups=64, n_in=2048, n_out=2048,
             dtype="bf16"),
        # the gradients of the benchmark workload's batch, heads by type
        dict(_GROUPED, name="backward_1024_of_4_256x47", op="backward"),
        # odd sizes in padded buffers, bf16
        dict(_GROUPED, name="backward_20011_of_24_1000x1021_bf16", op="backward", rows=20011, groups=24, skew=1.0, left_out=0.05,
             n_in=1000, n_out=1021, pad=7, dtype="bf16"),
        # the weights of the tiny workload's model
        dict(_MATRICES, name="orth_sage_tiny", op="orth", shapes="2x64x64,2x64x16"),
        # a stack of experts' matrices
        dict(_MATRICES, name="orth_16_of_2048x1024_bf16", op="orth", shapes="16x2048x1024", dtype="bf16"),
        # the benchmark workload's model
        dict(_MATRICES, name="muon_sage_medium", op="muon", shapes="2x100x256,2x256x256,2x256x47"),
        # a large model's matrices of many shapes, bf16 parameters with a float copy among them
        dict(_MATRICES, name="muon_large_mixed", op="muon",
             shapes="1x4096x4096,2x2048x5000,8x1024x1000,3x1021x4095,24x512x512,6x128x2048", dtype="mixed"),
    ]


def draw(rng: random.Random):
    """One more case of the ranges the listed ones span."""
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["group", "forward", "forward", "backward", "backward", "orth", "muon"])
    if op in ("orth", "muon"):
        left, shapes = MOST_NEWTON * math.exp(rng.uniform(math.log(1e-5), 0.0)), []
        for _ in range(rng.randint(1, 8)):
            rows, cols = log_uniform(2, 4096), log_uniform(2, 5000)
            while _newton_madds(1, rows, cols) > left:
                rows, cols = max(2, rows * 2 // 3), max(2, cols * 2 // 3)
                if rows == cols == 2:
                    break
            count = min(log_uniform(1, 32), max(1, int(left / _newton_madds(1, rows, cols))))
            left = max(0.0, left - _newton_madds(count, rows, cols))
            shapes.append(f"{count}x{rows}x{cols}")
        return dict(_MATRICES, op=op, shapes=",".join(shapes),
                    dtype=rng.choice(["f32", "bf16"] if op == "orth" else ["f32", "bf16", "mixed"]))
    c = dict(_GROUPED, op=op, groups=log_uniform(1, 256), skew=rng.choice([0.0, 0.5, 1.0, 2.0]),
             left_out=rng.choice([0.0, 0.0, 0.1, 0.5]))
    if op == "group":
        return dict(c, rows=log_uniform(1, 2_000_000))
    c.update(rows=log_uniform(1, 100_000), n_in=log_uniform(3, 2500), n_out=log_uniform(2, 2500), pad=rng.choice([0, 0, 1, 8]),
             dtype=rng.choice(["f32", "bf16"]), sorted=rng.random() < 0.3)
    most = MOST_PRODUCT // (2 if op == "backward" else 1) // (2 if c["dtype"] == "f32" else 1)
    c["groups"] = max(1, min(c["groups"], 100_000_000 // (c["n_in"] * c["n_out"])))
    c["rows"] = max(1, min(c["rows"], most // (c["n_in"] * c["n_out"])))
    return c


# -- what a case consists of -------------------------------------------------------------------

def _shapes(c):
    return [tuple(int(x) for x in s.split("x")) for s in c["shapes"].split(",")]


def _newton_madds(count, rows, cols):
    """Multiply-adds of the steps, those of the symmetric products counted once for both triangles."""
    m, n = min(rows, cols), max(rows, cols)
    return count * STEPS * (m * (m + 1) // 2 * n + m * (m + 1) // 2 * m + m * m * n)


def _group_of(c, seed):
    """Every row's group, -1 for a row that belongs to none (on the CPU, so that the sizes are known)."""
    gen = torch.Generator().manual_seed(seed * 7919 + 3)
    share = torch.arange(1, c["groups"] + 1, dtype=torch.float64) ** -c["skew"]
    share = share[torch.randperm(c["groups"], generator=gen)].cumsum(0)
    g = torch.searchsorted(share, torch.rand(c["rows"], dtype=torch.float64, generator=gen) * share[-1], right=True)
    g = g.clamp(max=c["groups"] - 1).to(torch.int32)
    g[torch.rand(c["rows"], generator=gen) < c["left_out"]] = -1
    return g


def _half_types(c):
    """Which stacks are bf16."""
    return [c["dtype"] == "bf16" or (c["dtype"] == "mixed" and i % 2 == 1) for i in range(len(_shapes(c)))]


def work(c):
    if c["op"] == "group":
        return {"bytes": 4 * (2 * c["rows"] + c["groups"] + 1), "flops": c["rows"]}
    if c["op"] in ("forward", "backward"):
        size = 4 if c["dtype"] == "f32" else 2
        rows = c["rows"] * (1.0 - c["left_out"])
        groups = min(c["groups"], c["rows"])        # (a gradient of W is written for those without rows too)
        x, y, w, b = rows * c["n_in"], rows * c["n_out"], groups * c["n_in"] * c["n_out"], c["groups"] * c["n_out"]
        dw = c["groups"] * c["n_in"] * c["n_out"]
        index = 4 * (rows + c["groups"] + 1)
        if c["op"] == "forward":
            return {"bytes": size * (x + y + w) + 4 * b + index, "flops": 2 * x * c["n_out"]}
        return {"bytes": size * (2 * x + y + w) + 4 * (dw + b) + index, "flops": 4 * x * c["n_out"]}
    each = [(k * r * q, h) for (k, r, q), h in zip(_shapes(c), _half_types(c))]
    flops = 2 * sum(_newton_madds(*s) for s in _shapes(c))
    if c["op"] == "orth":
        return {"bytes": sum(n * (4 if h else 8) for n, h in each), "flops": flops}
    # parameter (or its float copy) and momentum read and written; the gradient read, or it and the bf16 parameter at half the size
    return {"bytes": sum(20 * n for n, _ in each), "flops": flops}


_kept = {}


def _context():
    """The program's context.  These calls need no batch of it, so its graph is a single vertex."""
    if "ctx" not in _kept:
        from paper_2303_13775_amd import Context
        dev = torch.device("cuda")
        _kept["ctx"] = Context(torch.zeros(2, dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev),
                               torch.zeros(1, dtype=torch.uint8, device=dev), 1, [1], 1)
    return _kept["ctx"]


def _prepare_grouped(s, c, seed, gen):
    dev = torch.device("cuda")
    group = _group_of(c, seed)
    if c["sorted"]:
        group = group.sort()[0]
    counts = torch.bincount((group + 1).long(), minlength=c["groups"] + 1)
    first = torch.cat([torch.zeros(1, dtype=torch.int64), counts[1:].cumsum(0)])
    if c["op"] == "group":
        s.group = group.to(dev)
        s.ptr = torch.zeros(c["groups"] + 1, dtype=torch.int32, device=dev)
        s.order = torch.full((c["rows"],), -1, dtype=torch.int32, device=dev)       # the places behind the last group stay
        return
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    rows, k, n = c["rows"], c["n_in"], c["n_out"]
    if c["sorted"]:
        # the rows of no group come first in the sort and are not among those handed over
        rows = int(first[-1])
        s.order = None
    else:
        order = group.long().sort(stable=True)[1]
        # (those of no group behind the last one, where nobody asks for them)
        s.order = torch.roll(order, -int(counts[0])).to(torch.int32).to(dev)
    s.sizes = counts[1:].tolist()
    s.ptr = first.to(torch.int32).to(dev)

    def buffer(width, fill):
        t = torch.empty((rows, width + c["pad"]), device=dev, dtype=torch.float32)
        t = (t.normal_(generator=gen) if fill else t.zero_()).to(dt)
        return t[:, :width]

    s.x = buffer(k, True)
    s.w = (torch.randn((c["groups"], k, n), device=dev, generator=gen) * k ** -0.5).to(dt)
    if c["op"] == "forward":
        s.bias = torch.randn((c["groups"], n), device=dev, generator=gen).mul_(0.1)
        s.y = buffer(n, False)
    else:
        s.dy = buffer(n, True)
        s.dx = buffer(k, False)
        s.dw = torch.zeros((c["groups"], k, n), device=dev)
        s.db = torch.zeros((c["groups"], n), device=dev)


def _matrices(shapes, halves, gen, scale):
    """What gradients look like: a few strong directions over a floor of noise."""
    out = []
    for (count, rows, cols), half in zip(shapes, halves):
        rank = min(12, rows, cols)
        fall = 2.0 ** -torch.arange(rank, device="cuda", dtype=torch.float32)
        u = torch.randn((count, rows, rank), device="cuda", generator=gen) * fall
        v = torch.randn((count, rank, cols), device="cuda", generator=gen)
        g = torch.matmul(u, v).add_(torch.randn((count, rows, cols), device="cuda", generator=gen), alpha=0.3).mul_(scale)
        out.append(g.bfloat16() if half else g)
    return out


def prepare(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000003 + 29)
    s = SimpleNamespace(c=c)
    if c["op"] in ("group", "forward", "backward"):
        _prepare_grouped(s, c, seed, gen)
    else:
        shapes, s.half = _shapes(c), _half_types(c)
        s.grads = _matrices(shapes, s.half, gen, 1e-3)
        if c["op"] == "orth":
            s.outs = [torch.zeros_like(g) for g in s.grads]
        else:
            s.momenta = [m.mul_(0.5) for m in _matrices(shapes, [False] * len(shapes), gen, 1e-3)]
            # float: the parameters, and the copies of the bfloat16 ones
            s.params = [torch.randn(x, device="cuda", generator=gen).mul_(0.05) for x in shapes]
            s.halves = [p.bfloat16() if h else None for p, h in zip(s.params, s.half)]
    if own:
        s.ctx = _context()
        if c["op"] == "backward":
            s.room = s.ctx.gsplit_grouped_linear_work(s.x, s.w)
        elif c["op"] == "orth":
            from paper_2303_13775_amd import MatrixTensors
            s.table = MatrixTensors(s.grads, s.outs)
        elif c["op"] == "muon":
            from paper_2303_13775_amd import MuonTensors
            s.table = MuonTensors([p if h is None else h for p, h in zip(s.params, s.halves)], s.grads, s.momenta,
                                  [None if h is None else p for p, h in zip(s.params, s.halves)])
    return s


# -- the plain forms ---------------------------------------------------------------------------

def _plain_group(s):
    g = s.group.long()
    order = torch.sort(torch.where(g < 0, s.c["groups"], g), stable=True)[1]
    counts = torch.zeros(s.c["groups"] + 1, dtype=torch.int64, device=g.device).scatter_add_(0, g + 1, torch.ones_like(g))
    s.ptr[1:] = counts[1:].cumsum(0)
    place = torch.arange(g.numel(), device=g.device)
    return {"ptr": s.ptr, "order": torch.where(place < s.ptr[-1], order, -1).int()}


def _blocks(s):
    """(group, its rows) of the groups that have any."""
    at = 0
    for g, n in enumerate(s.sizes):
        if n:
            yield g, slice(at, at + n) if s.order is None else s.order[at:at + n].long()
        at += n


def _plain_forward(s):
    y = torch.zeros(s.y.shape, device=s.y.device)
    for g, rows in _blocks(s):
        y[rows] = s.x[rows].float() @ s.w[g].float() + s.bias[g]
    return {"y": y.to(s.x.dtype)}


def _plain_backward(s):
    dx = torch.zeros(s.x.shape, device=s.x.device)
    dw, db = torch.zeros(s.w.shape, device=s.x.device), torch.zeros(s.db.shape, device=s.x.device)
    for g, rows in _blocks(s):
        x, dy = s.x[rows].float(), s.dy[rows].float()
        dx[rows] = dy @ s.w[g].float().t()
        dw[g] = x.t() @ dy
        db[g] = dy.sum(0)
    return {"dx": dx.to(s.x.dtype), "dw": dw, "db": db}


def _plain_orthogonal(g):
    tall = g.shape[1] > g.shape[2]
    x = g.transpose(1, 2).contiguous() if tall else g
    norm = (x * x).sum((1, 2), keepdim=True, dtype=torch.float64).sqrt().float()
    x = x / (norm + EPS)
    for _ in range(STEPS):
        a = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = A * x + torch.matmul(B * a + C * torch.matmul(a, a), x)
    return x.transpose(1, 2) if tall else x


def _plain_orth(s):
    return {f"out{i}": _plain_orthogonal(g.float()).to(g.dtype).contiguous() for i, g in enumerate(s.grads)}


def _muon_scale(shape):
    """An update of the size of the output: the matrices are n_in x n_out."""
    return math.sqrt(max(1.0, shape[2] / shape[1]))


def _muon_outputs(s):
    return {**{f"param{i}": p for i, p in enumerate(s.params)}, **{f"momentum{i}": m for i, m in enumerate(s.momenta)},
            **{f"half{i}": h for i, h in enumerate(s.halves) if h is not None}}


def _plain_muon(s):
    for p, h, g, m in zip(s.params, s.halves, s.grads, s.momenta):
        g = g.float()
        m.mul_(MOMENTUM).add_(g * (1 - MOMENTUM))
        o = _plain_orthogonal(MOMENTUM * m + (1 - MOMENTUM) * g)
        p.mul_(1 - LR * DECAY).sub_(o * (LR * _muon_scale(p.shape)))
        if h is not None:
            h.copy_(p)
    return _muon_outputs(s)


_PLAIN = {"group": _plain_group, "forward": _plain_forward, "backward": _plain_backward, "orth": _plain_orth, "muon": _plain_muon}


def run(s):
    op = s.c["op"]
    if not own:
        return _PLAIN[op](s)
    if op == "group":
        s.ctx.gsplit_group_rows(s.group, s.ptr, s.order)
        return {"ptr": s.ptr, "order": s.order}
    if op == "forward":
        s.ctx.gsplit_grouped_linear_fwd(s.x, s.ptr, s.order, s.w, s.bias, s.y)
        return {"y": s.y}
    if op == "backward":
        s.ctx.gsplit_grouped_linear_bwd(s.x, s.ptr, s.order, s.w, s.dy, s.dx, s.dw, s.db, s.room)
        return {"dx": s.dx, "dw": s.dw, "db": s.db}
    if op == "orth":
        s.ctx.gsplit_orthogonalize(s.table, steps=STEPS, coefficients=(A, B, C), eps=EPS)
        return {f"out{i}": o for i, o in enumerate(s.outs)}
    s.ctx.gsplit_muon_step(s.table, lr=LR, momentum=MOMENTUM, nesterov=True, weight_decay=DECAY, scaling="shape", steps=STEPS,
                           coefficients=(A, B, C), eps=EPS)
    return _muon_outputs(s)


# -- the definition in 64 bits -------------------------------------------------------------------

def _exact_polar(g):
    """Newton-Schulz of one matrix, by its definition: X <- (a I + b (X X^T) + c (X X^T)^2) X."""
    x = g.double()
    x = x / (torch.linalg.matrix_norm(x) + EPS)
    if x.shape[0] > x.shape[1]:         # (X X^T) X = X (X^T X): the smaller of the two
        return _exact_steps(x.t().contiguous()).t()
    return _exact_steps(x)


def _exact_steps(x):
    one = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for _ in range(STEPS):
        q = torch.mm(x, x.t())
        x = torch.mm(A * one + B * q + C * torch.mm(q, q), x)
    return x


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "group":
        return None
    if c["op"] in ("forward", "backward"):
        of = torch.full((s.x.shape[0],), -1, dtype=torch.int64)
        place = torch.arange(s.x.shape[0]) if s.order is None else s.order.cpu().long()
        ptr = s.ptr.tolist()
        for g in range(c["groups"]):
            of[place[ptr[g]:ptr[g + 1]]] = g
        of = of.to(s.x.device)
        if c["op"] == "forward":
            y = torch.zeros(s.y.shape, dtype=torch.float64, device=of.device)
            for g in range(c["groups"]):
                r = (of == g).nonzero()[:, 0]
                y[r] = torch.addmm(s.bias[g].double(), s.x[r].double(), s.w[g].double())
            return {"y": y}
        out = {"dx": torch.zeros(s.x.shape, dtype=torch.float64, device=of.device),
               "dw": torch.zeros(s.w.shape, dtype=torch.float64, device=of.device),
               "db": torch.zeros(s.db.shape, dtype=torch.float64, device=of.device)}
        for g in range(c["groups"]):
            r = (of == g).nonzero()[:, 0]
            d = s.dy[r].double()
            out["dx"][r] = torch.mm(d, s.w[g].double().t().contiguous())
            out["dw"][g] = torch.mm(s.x[r].double().t().contiguous(), d)
            out["db"][g] = d.sum(0)
        return out
    if c["op"] == "orth":
        return {f"out{i}": torch.stack([_exact_polar(x) for x in g]) for i, g in enumerate(s.grads)}
    out = {}
    for i, (p, h, g, m) in enumerate(zip(s.params, s.halves, s.grads, s.momenta)):
        m, g = m.double(), g.double()
        m = MOMENTUM * m + (1 - MOMENTUM) * g
        o = torch.stack([_exact_polar(x) for x in MOMENTUM * m + (1 - MOMENTUM) * g])
        change = LR * math.sqrt(max(1.0, p.shape[2] / p.shape[1])) * o
        out[f"param{i}"], out[f"momentum{i}"] = p.double() * (1 - LR * DECAY) - change, m
        if h is not None:
            out[f"half{i}"] = out[f"param{i}"]
    return out
