"""Rows sorted by group and the products by group against their plain float64 forms: odd and ragged sizes, groups without rows, rows
without a group, padded and misaligned buffers, values that floats' parts cannot carry, and the ways a caller may run them.

Tolerances, with u = 2^-24 and s = the sum of the sizes of an element's terms.  A product of floats goes through three parts of
either factor; what is dropped reaches u of it.  A float sum of n terms taken 16 at a time by the matrix unit rounds at most
n / 16 + 5 times (16 terms inside the unit: 4), each at most u s, and so do the sums of its chunks (less than 64) and the bias:
(n / 16 + 5 + 64 + 2) u s bounds a float result; the tests take the rounding errors' usual growth with the root of their number, times 4:
4 (sqrt(n / 16 + 64) + 2) u s, which is at most the bound from n = 1 on (4 (8 + 2) = 40 < 71, and 4 sqrt(x) < x from x = 16 on).  Results
in bfloat16 are rounded once more (2^-8 of them)."""
import numpy as np
import pytest
import torch

import row_loss_check as K
from oracle import grouped as O

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = K.U


@pytest.fixture(scope="module")
def ctx():
    c = K.context()
    yield c
    c.close()


def _draw_groups(rng, rows, groups, skew=0.0, left_out=0.0, empty=()):
    p = np.arange(1, groups + 1.0) ** -skew
    p = rng.permutation(p)
    p[list(empty)] = 0.0
    g = rng.choice(groups, size=rows, p=p / p.sum()).astype(np.int32)
    g[rng.random(rows) < left_out] = rng.choice([-1, groups, -(1 << 31), (1 << 31) - 1])
    return g


def _group(ctx, group, n_groups, gap=3):
    dev = torch.from_numpy(group).cuda()
    ptr = torch.full((n_groups + 1 + gap,), 77, dtype=torch.int32, device="cuda")
    rows = torch.full((len(group) + gap,), 88, dtype=torch.int32, device="cuda")
    ctx.gsplit_group_rows(dev, ptr[:n_groups + 1], rows[:len(group)])
    assert bool((ptr[n_groups + 1:] == 77).all()) and bool((rows[len(group):] == 88).all())
    return ptr[:n_groups + 1], rows[:len(group)]


@pytest.mark.parametrize("rows, groups", [(0, 1), (0, 7), (1, 1), (1, 512), (63, 3), (64, 64), (65, 2), (1000, 1), (1024, 4), (1025, 512), (4096, 8),
                                          (4097, 8), (5000, 511), (70_001, 5), (300_000, 33), (1_000_003, 64), (2_500_000, 512), (20_000, 1)])
@pytest.mark.parametrize("skew, left_out", [(0.0, 0.0), (2.0, 0.3)])
def test_group_rows(ctx, rows, groups, skew, left_out):
    rng = np.random.default_rng(rows + groups)
    group = _draw_groups(rng, rows, groups, skew, left_out)
    ptr, order = _group(ctx, group, groups)
    ok = (group >= 0) & (group < groups)
    key = np.where(ok, group, groups)
    want = np.argsort(key, kind="stable")[:ok.sum()]
    got = order.cpu().numpy()
    assert (ptr.cpu().numpy() == np.concatenate([[0], np.bincount(key, minlength=groups + 1)[:groups].cumsum()])).all()
    assert (got[:len(want)] == want).all() and (got[len(want):] == 88).all()
    if rows <= 5000:
        p, r = O.group_rows(group, groups)
        assert (p == ptr.cpu().numpy()).all() and (r == want).all()


def test_rows_that_all_share_a_group_or_have_none(ctx):
    for rows in (100, 4097, 200_000):
        ptr, order = _group(ctx, np.full(rows, 3, np.int32), 5)
        assert ptr.tolist() == [0, 0, 0, 0, rows, rows] and bool((order == torch.arange(rows, device="cuda")).all())
        ptr, order = _group(ctx, np.full(rows, -1, np.int32), 5)
        assert ptr.tolist() == [0] * 6 and bool((order == 88).all())


@pytest.mark.parametrize("rows", [256, 1000, 4096, 4097, 90_001, 700_000])
@pytest.mark.parametrize("groups", [1, 2, 3, 61, 512])
def test_counters_that_pass_from_lane_to_lane(ctx, rows, groups):
    """The lane that counts for a group is its first of 64 rows; here it is another one in every 64."""
    i = np.arange(rows)
    lane, turn = i % 64, i // 64
    group = ((lane - 7 * turn) % 64 * groups // 64).astype(np.int32)            # a rotating pattern of runs
    group[(lane == turn % 64) & (turn % 3 == 0)] = groups - 1                   # one row by itself
    group[lane < turn % 5] = -1
    ptr, order = _group(ctx, group, groups)
    key = np.where(group >= 0, group, groups)
    want = np.argsort(key, kind="stable")[:(group >= 0).sum()]
    assert (ptr.cpu().numpy() == np.concatenate([[0], np.bincount(key, minlength=groups + 1)[:groups].cumsum()])).all()
    assert (order.cpu().numpy()[:len(want)] == want).all() and bool((order[len(want):] == 88).all())


def _tol(size, n):
    return 4 * (np.sqrt(n / 16 + 64) + 2) * U * size


def _check(name, got, want, tol, dtype=F32):
    """K.check; what lies beyond the largest float is infinite in either type."""
    with np.errstate(over="ignore"):
        want = np.where(np.isinf(want.astype(np.float32)), want.astype(np.float32).astype(np.float64), want)
    K.check(name, got, want, tol, dtype)


def _values(rng, shape, dtype, scale=1.0):
    """(tensor values as float64 after rounding to the type)"""
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(dtype).double().numpy()


def _case(ctx, rows, groups, n_in, n_out, dtype, *, skew=0.0, left_out=0.0, empty=(), pad=0, offset=0, listed=True, bias=True, seed=0,
          values=None, parts=("fwd", "bwd")):
    rng = np.random.default_rng(seed + 7 * rows + groups + n_in * 3 + n_out)
    group = _draw_groups(rng, rows, groups, skew, left_out, empty)
    if not listed:
        group = np.sort(group[(group >= 0) & (group < groups)])
        rows = len(group)
    ptr, order = _group(ctx, group, groups, 0)
    p, r = O.group_rows(group, groups)
    x, dy = _values(rng, (rows, n_in), dtype), _values(rng, (rows, n_out), dtype)
    w = _values(rng, (groups, n_in, n_out), dtype, n_in ** -0.5)
    b = _values(rng, (groups, n_out), F32)
    if values:
        values(x, w, dy)
    as_rows = lambda v: K.rows_buffer(torch.from_numpy(v), dtype, pad, offset)
    (xb, xt), (dyb, dyt) = as_rows(x), as_rows(dy)
    (yb, yt), (dxb, dxt) = as_rows(np.full((rows, n_out), 7.0)), as_rows(np.full((rows, n_in), 7.0))
    wt, bt = torch.from_numpy(w).to(dtype).cuda(), torch.from_numpy(b).float().cuda()
    order = order if listed else None
    if "fwd" in parts:
        ctx.gsplit_grouped_linear_fwd(xt, ptr, order, wt, bt if bias else None, yt)
        want, size, used = O.linear(x, p, r, w, b if bias else None)
        want[~used], size[~used] = 7.0, 0.0             # rows of no group are left as they were
        _check("y", yt, want, _tol(size, n_in), dtype)
        assert K.untouched(yb, yt)
    if "bwd" in parts:
        dw, db = torch.full((groups, n_in, n_out), 9.0, device="cuda"), torch.full((groups, n_out), 9.0, device="cuda")
        work = ctx.gsplit_grouped_linear_work(xt, wt)
        room = torch.full((work.numel() + 8,), 5.0, device="cuda")
        ctx.gsplit_grouped_linear_bwd(xt, ptr, order, wt, dyt, dxt, dw, db, room[:work.numel()])
        (dx, dxs), (dw0, dws), (db0, dbs) = O.linear_grad(x, p, r, w, dy)
        used = np.zeros(rows, bool)
        used[r] = True
        dx[~used], dxs[~used] = 7.0, 0.0
        most = int(np.diff(p).max())
        _check("dx", dxt, dx, _tol(dxs, n_out), dtype)
        _check("dw", dw, dw0, _tol(dws, most))
        _check("db", db, db0, _tol(dbs, most))
        assert K.untouched(dxb, dxt) and bool((room[work.numel():] == 5.0).all())
        again = [torch.empty_like(t) for t in (dw, db)]
        ctx.gsplit_grouped_linear_bwd(xt, ptr, order, wt, dyt, None, *again, room[:work.numel()])
        assert all(torch.equal(a, b) or bool(((a == b) | (a.isnan() & b.isnan())).all()) for a, b in zip((dw, db), again))
        only = K.rows_buffer(torch.full((rows, n_in), 7.0), dtype, pad, offset)[1]
        ctx.gsplit_grouped_linear_bwd(xt, ptr, order, wt, dyt, only, None, None)
        assert bool(((only == dxt) | (only.isnan() & dxt.isnan())).all())
    assert K.untouched(xb, xt) and K.untouched(dyb, dyt)


SHAPES = [      # rows, groups, n_in, n_out
    (1, 1, 1, 1), (1, 3, 2, 5), (5, 2, 3, 1), (7, 7, 1, 9), (33, 8, 256, 47), (64, 1, 32, 64), (65, 2, 33, 65), (100, 5, 31, 63), (129, 1, 64, 129),
    (200, 3, 65, 2), (257, 2, 129, 131), (300, 40, 17, 3), (1024, 4, 256, 47), (1000, 2, 100, 172), (4096, 16, 256, 172), (513, 100, 5, 7), (777, 512, 40, 30)]


@pytest.mark.parametrize("rows, groups, n_in, n_out", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kw", [dict(), dict(skew=2.0, left_out=0.3, pad=1, offset=1), dict(listed=False, pad=8, bias=False)])
def test_products(ctx, rows, groups, n_in, n_out, dtype, kw):
    _case(ctx, rows, groups, n_in, n_out, dtype, **kw)


LARGE = [
    (9000, 3, 512, 512, dict(skew=1.0)), (20_011, 24, 300, 261, dict(skew=1.0, left_out=0.05, pad=7)), (3000, 1, 1000, 1021, dict(offset=3)),
    (40_000, 2, 64, 16, dict(skew=2.0)), (2500, 9, 640, 520, dict(empty=(0, 4, 8))), (70_000, 300, 24, 40, dict(listed=False)),
    (5000, 2, 100, 60, dict()), (6000, 512, 300, 129, dict(pad=3)), (250, 300, 96, 100, dict())]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, groups, n_in, n_out, kw", LARGE)
def test_large_products(ctx, rows, groups, n_in, n_out, kw, dtype):
    _case(ctx, rows, groups, n_in, n_out, dtype, **kw)


# bfloat16 rows of whole granules, enough for the large tiles: edges of the rows, of the contraction, of the columns; groups of a few rows
LARGE_TILES = [
    (17_000, 5, 264, 520, dict(skew=1.0, left_out=0.1, pad=8, offset=8)), (33_000, 1, 128, 1000, dict(listed=False)), (20_000, 300, 512, 256, dict(skew=2.0)),
    (35_000, 40, 136, 1288, dict(skew=1.0, pad=16, bias=False)), (16_500, 2, 1000, 504, dict(empty=(0,))), (40_000, 7, 392, 136, dict(left_out=0.5)), (20_000, 3, 520, 128, dict(skew=2.0))]


@pytest.mark.parametrize("rows, groups, n_in, n_out, kw", LARGE_TILES)
def test_large_tiles(ctx, rows, groups, n_in, n_out, kw):
    _case(ctx, rows, groups, n_in, n_out, BF16, **kw)


# Weight gradients whose chunks are dealt in pieces: tiles that no piece divides (17 of 64, 25 of 64 and of 128, 18 of 256), groups of no rows among them
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, groups, n_in, n_out", [(3000, 30, 17 * 64, 40), (2500, 20, 300, 310), (1500, 17, 600, 580), (9000, 40, 264, 9 * 256)])
def test_chunks_in_pieces(ctx, rows, groups, n_in, n_out, dtype):
    _case(ctx, rows, groups, n_in, n_out, dtype, skew=1.0, left_out=0.1, empty=(0, 9, groups - 1))


# Contractions that end inside a granule, short of one, and rows whose last is the buffer's last: what lies past a row's end is its neighbour's
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, groups", [(300, 2), (9000, 5), (40_000, 3)])
@pytest.mark.parametrize("n_in, n_out", [(7, 9), (8, 200), (9, 17), (11, 15), (31, 33), (41, 71), (63, 65), (66, 201), (69, 130), (76, 8), (127, 257)])
def test_contractions_that_end_anywhere(ctx, rows, groups, n_in, n_out, dtype):
    _case(ctx, rows, groups, n_in, n_out, dtype, skew=0.5)


@pytest.mark.parametrize("bad", [np.inf, np.nan])
def test_large_tiles_keep_values_that_are_not_finite_where_they_belong(ctx, bad):
    rows, n_in, n_out = 17_000, 264, 520

    def values(x, w, dy):
        x[3, 1], x[rows - 1, n_in - 1] = bad, bad
        w[1, n_in - 1, n_out - 2], w[0, 0, 0] = bad, bad
        dy[rows - 2, 5], dy[4, n_out - 1] = bad, bad
    _case(ctx, rows, 3, n_in, n_out, BF16, values=values)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_groups_without_rows_and_no_rows_at_all(ctx, dtype):
    _case(ctx, 50, 6, 40, 24, dtype, empty=(0, 2, 3, 5))
    w = torch.ones((3, 5, 7), dtype=dtype, device="cuda")
    ptr, x = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros((0, 5), dtype=dtype, device="cuda")
    y, dw, db = torch.zeros((0, 7), dtype=dtype, device="cuda"), torch.ones((3, 5, 7), device="cuda"), torch.ones((3, 7), device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    for order in (None, none):
        ctx.gsplit_grouped_linear_fwd(x, ptr, order, w, None, y)
        ctx.gsplit_grouped_linear_bwd(x, ptr, order, w, y, x.clone(), dw, db)
        assert not dw.any() and not db.any()
        dw.fill_(1.0)
    x, y = torch.ones((9, 5), dtype=dtype, device="cuda"), torch.ones((9, 7), dtype=dtype, device="cuda")        # rows, none of them in a group
    dx, order = x.clone(), torch.full((9,), 1 << 30, dtype=torch.int32, device="cuda")
    ctx.gsplit_grouped_linear_fwd(x, ptr, order, w, None, y)
    ctx.gsplit_grouped_linear_bwd(x, ptr, order, w, y, dx, dw, db, ctx.gsplit_grouped_linear_work(x, w))
    assert bool((y == 1).all()) and bool((dx == 1).all()) and not dw.any() and not db.any()


@pytest.mark.parametrize("scale", [1e-36, 1e-30, 1e15])
def test_floats_of_any_size(ctx, scale):
    rows, groups, n_in, n_out = 200, 3, 70, 66

    def rounded(x, w, dy):
        for t in (x, dy):
            t[:] = (t * scale).astype(np.float32).astype(np.float64)
    _case(ctx, rows, groups, n_in, n_out, F32, values=rounded)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan, 3e38])
@pytest.mark.parametrize("rows, n_in, n_out", [(40, 30, 20), (700, 200, 150)])
def test_values_that_are_not_finite_stay_where_they_belong(ctx, dtype, bad, rows, n_in, n_out):
    """A row of x reaches its row of y and its group's dW, an element of W its column of y: no further, and infinities stay infinities."""
    v = float(torch.tensor(bad, dtype=F32).to(dtype).double()) if np.isfinite(bad) else bad

    def values(x, w, dy):
        x[3, 1] = v
        w[1, n_in - 1, n_out - 2] = v
        dy[rows - 1, 5] = v
    _case(ctx, rows, 3, n_in, n_out, dtype, values=values)


def test_offsets_and_rows_that_make_no_sense_stay_inside_the_buffers(ctx):
    """What the kernels are given by the device is held inside the buffers: the results are wrong, their surroundings untouched."""
    rows, groups, n_in, n_out = 300, 5, 40, 24
    for dtype in (F32, BF16):
        (xb, x), (yb, y), (dxb, dx) = (K.rows_buffer(torch.ones((rows, n)), dtype, 3, 1) for n in (n_in, n_out, n_in))
        w = torch.ones((groups, n_in, n_out), dtype=dtype, device="cuda")
        dw, db = torch.zeros((groups, n_in, n_out), device="cuda"), torch.zeros((groups, n_out), device="cuda")
        work = ctx.gsplit_grouped_linear_work(x, w)
        room = torch.full((work.numel() + 64,), 5.0, device="cuda")
        for ptr in ([-5, 100, 50, 4000, 200, 300], [300, 0, 300, 0, 300, 0], [0, 300, 300, 2 ** 31 - 1, -2 ** 31, 7], [0, 2 ** 31 - 1] * 3):
            for order in (None, [0] * rows, [-1, rows, 2 ** 31 - 1] * 100, list(range(rows))):
                pt = torch.tensor(ptr, dtype=torch.int32, device="cuda")
                ot = None if order is None else torch.tensor(order, dtype=torch.int32, device="cuda")
                ctx.gsplit_grouped_linear_fwd(x, pt, ot, w, None, y)
                ctx.gsplit_grouped_linear_bwd(x, pt, ot, w, y, dx, dw, db, room[:work.numel()])
                assert K.untouched(yb, y) and K.untouched(dxb, dx) and bool((room[work.numel():] == 5.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_against_differences(ctx, dtype):
    """The gradients of sum(y * dy) against the differences of the forward pass in float64 (the product is linear in each factor)."""
    rng = np.random.default_rng(5)
    rows, groups, n_in, n_out = 60, 3, 11, 9
    group = _draw_groups(rng, rows, groups)
    ptr, order = _group(ctx, group, groups, 0)
    p, r = O.group_rows(group, groups)
    x, dy, w = _values(rng, (rows, n_in), dtype), _values(rng, (rows, n_out), dtype), _values(rng, (groups, n_in, n_out), dtype)
    b = np.zeros((groups, n_out))
    dev = lambda v: torch.from_numpy(v).to(dtype).cuda()
    xt, wt, dyt, dx = dev(x), dev(w), dev(dy), dev(x)
    dw, db = torch.zeros(w.shape, device="cuda"), torch.zeros(b.shape, device="cuda")
    ctx.gsplit_grouped_linear_bwd(xt, ptr, order, wt, dyt, dx, dw, db, ctx.gsplit_grouped_linear_work(xt, wt))
    value = lambda x, w, b: float((O.linear(x, p, r, w, b)[0] * dy).sum())
    for t, got, args in ((x, dx, 0), (w, dw, 1), (b, db, 2)):
        for _ in range(20):
            at = tuple(int(rng.integers(n)) for n in t.shape)
            sides = []
            for h in (0.5, -0.5):
                moved = [x.copy(), w.copy(), b.copy()]
                moved[args][at] += h
                sides.append(value(*moved))
            want = sides[0] - sides[1]
            tol = 200 * U * (np.abs(x).max() + 1) * (np.abs(w).max() + 1) * (np.abs(dy).max() + 1) + (K.EPS[dtype] * abs(want) if args == 0 else 0)
            assert abs(float(got[at]) - want) <= tol, (args, at)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_captured_calls(ctx, dtype):
    """Sorting, the products and their gradients captured once and replayed on other groups and values, with eager calls of the same
    context between: the bits of eager calls."""
    rng = np.random.default_rng(6)
    rows, groups, n_in, n_out = 6000, 6, 130, 70
    dev = lambda *shape: torch.zeros(shape, dtype=dtype, device="cuda")
    group, ptr, order = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (rows, groups + 1, rows))
    x, w, dy, b = dev(rows, n_in), dev(groups, n_in, n_out), dev(rows, n_out), torch.zeros((groups, n_out), device="cuda")
    outs = lambda: [dev(rows, n_out), dev(rows, n_in), torch.zeros((groups, n_in, n_out), device="cuda"), torch.zeros((groups, n_out), device="cuda")]
    got, want = outs(), outs()
    rooms = [ctx.gsplit_grouped_linear_work(x, w) for _ in range(2)]

    def step(o, room):
        ctx.gsplit_group_rows(group, ptr, order)
        ctx.gsplit_grouped_linear_fwd(x, ptr, order, w, b, o[0])
        ctx.gsplit_grouped_linear_bwd(x, ptr, order, w, dy, o[1], o[2], o[3], room)

    step(want, rooms[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(got, rooms[0])
    for k in range(5):
        group.copy_(torch.from_numpy(_draw_groups(rng, rows, groups, float(k % 3), 0.1 * k)))
        for t in (x, w, dy, b):
            t.copy_(torch.from_numpy(rng.standard_normal(t.shape).astype(np.float32)))
        for t in (*got, *want):
            t.zero_()
        step(want, rooms[1])
        graph.replay()
        if k % 2:
            torch.cuda.synchronize()
        ctx.gsplit_grouped_linear_fwd(x, ptr, order, w, b, want[0])
        assert all(torch.equal(a, c) for a, c in zip(got, want)), k


def test_other_streams(ctx):
    rng = np.random.default_rng(8)
    rows, groups, n_in, n_out = 3000, 4, 96, 80
    group = torch.from_numpy(_draw_groups(rng, rows, groups)).cuda()
    x, w = torch.randn((rows, n_in), device="cuda"), torch.randn((groups, n_in, n_out), device="cuda")
    res = []
    for s in (torch.cuda.current_stream(), *[torch.cuda.Stream() for _ in range(4)]):      # (a stream for every hardware queue)
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            ptr, order = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (groups + 1, rows))
            y, dx, dw, db = torch.zeros((rows, n_out), device="cuda"), torch.zeros_like(x), torch.zeros_like(w), torch.zeros((groups, n_out), device="cuda")
            ctx.gsplit_group_rows(group, ptr, order)
            ctx.gsplit_grouped_linear_fwd(x, ptr, order, w, None, y)
            ctx.gsplit_grouped_linear_bwd(x, ptr, order, w, y, dx, dw, db, ctx.gsplit_grouped_linear_work(x, w))
            torch.cuda.synchronize()
            res.append((ptr, order, y, dx, dw, db))
    assert all(torch.equal(a, b) for r in res[1:] for a, b in zip(res[0], r))


def test_more_than_32_bits_of_elements(ctx):
    """Rows and matrices whose elements lie past 2^31 and 2^32."""
    rows, n_in, n_out = 1_100_000, 2000, 3        # 2.2e9 values
    x = torch.zeros((rows, n_in), dtype=BF16, device="cuda")
    at = [0, 7, 1_073_742, rows - 2, rows - 1]
    x[at, 5] = 2.0
    w = torch.zeros((2, n_in, n_out), dtype=BF16, device="cuda")
    w[0, 5], w[1, 5] = 1.0, 3.0
    ptr = torch.tensor([0, 100, rows], dtype=torch.int32, device="cuda")
    y = torch.zeros((rows, n_out), dtype=BF16, device="cuda")
    ctx.gsplit_grouped_linear_fwd(x, ptr, None, w, None, y)
    assert int(torch.count_nonzero(y)) == 3 * len(at) and y[at, 1].tolist() == [2.0, 2.0, 6.0, 6.0, 6.0]
    dw, db = torch.zeros((2, n_in, n_out), device="cuda"), torch.zeros((2, n_out), device="cuda")
    dx = torch.zeros_like(x)
    ctx.gsplit_grouped_linear_bwd(x, ptr, None, w, y, dx, dw, db, ctx.gsplit_grouped_linear_work(x, w))
    assert int(torch.count_nonzero(dw)) == 6 and dw[:, 5, 0].tolist() == [8.0, 36.0] and db[:, 2].tolist() == [4.0, 18.0]
    assert int(torch.count_nonzero(dx)) == len(at) and dx[at, 5].tolist() == [6.0, 6.0, 54.0, 54.0, 54.0]
    del x, dx, y
    groups, n_in, n_out = 3, 40_000, 20_000         # 2.4e9 values
    w = torch.zeros((groups, n_in, n_out), dtype=BF16, device="cuda")
    w[2, n_in - 1, n_out - 1], w[2, 0, 0], w[1, 9, 9] = 4.0, 2.0, 1.0
    x = torch.ones((2, n_in), dtype=BF16, device="cuda")
    y = torch.zeros((2, n_out), dtype=BF16, device="cuda")
    ctx.gsplit_grouped_linear_fwd(x, torch.tensor([0, 0, 1, 2], dtype=torch.int32, device="cuda"), None, w, None, y)
    assert int(torch.count_nonzero(y)) == 3 and y[0, 9] == 1 and y[1, 0] == 2 and y[1, -1] == 4


def test_results_in_the_place_of_what_is_read(ctx):
    x, w, dw = torch.ones((9, 6), device="cuda"), torch.ones((2, 6, 6), device="cuda"), torch.zeros((2, 6, 6), device="cuda")
    dy, group, ptr = torch.ones((9, 6), device="cuda"), torch.zeros(9, dtype=torch.int32, device="cuda"), torch.tensor([0, 4, 9], dtype=torch.int32, device="cuda")
    for call in (lambda: ctx.gsplit_group_rows(group, ptr, group), lambda: ctx.gsplit_grouped_linear_fwd(x, ptr, None, w, None, x),
                 lambda: ctx.gsplit_grouped_linear_bwd(x, ptr, None, w, dy, x, dw, None), lambda: ctx.gsplit_grouped_linear_bwd(x, ptr, None, w, dy, dy, None, None)):
        with pytest.raises(AssertionError):
            call()
    both = torch.ones((9, 12), device="cuda")           # columns of one buffer side by side are apart
    ctx.gsplit_grouped_linear_fwd(both[:, :6], ptr, None, w, None, both[:, 6:])
    assert bool((both[:, :6] == 1).all()) and bool((both[:, 6:] == 6).all())


def test_refusals(ctx):
    from paper_2303_13775_amd import GsplitError
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    with pytest.raises(GsplitError) as e:
        ctx.gsplit_group_rows(i32(4), i32(514), i32(4))
    assert e.value.code == -1 and "gsplit_group_rows" in str(e.value)
    x, w, y = torch.zeros((6, 4), device="cuda"), torch.zeros((2, 4, 3), device="cuda"), torch.zeros((6, 3), device="cuda")
    ptr, order = i32(3), i32(6)
    with pytest.raises(GsplitError) as e:
        ctx.gsplit_grouped_linear_bwd(x, ptr, order, w, y, None, None, None)
    assert "gsplit_grouped_linear_bwd" in str(e.value)
    with pytest.raises(GsplitError):
        ctx.gsplit_grouped_linear_bwd(x, ptr, order, w, y, x.clone(), None, torch.zeros((2, 3), device="cuda"))
    with pytest.raises(GsplitError):
        ctx.gsplit_grouped_linear_fwd(x, i32(514), order, torch.zeros((513, 4, 3), device="cuda"), None, y)
    with pytest.raises(GsplitError):
        ctx.gsplit_grouped_linear_fwd(x.expand(6, 4).as_strided((6, 4), (2, 1)), ptr, order, w, None, y)
    bad = [lambda: ctx.gsplit_group_rows(i32(4).long(), i32(3), i32(4)), lambda: ctx.gsplit_group_rows(i32(4), i32(3), i32(5)),
           lambda: ctx.gsplit_grouped_linear_fwd(x, i32(4), order, w, None, y), lambda: ctx.gsplit_grouped_linear_fwd(x, ptr, i32(5), w, None, y),
           lambda: ctx.gsplit_grouped_linear_fwd(x, ptr, order, w.bfloat16(), None, y), lambda: ctx.gsplit_grouped_linear_fwd(x, ptr, order, w, None, y.bfloat16()),
           lambda: ctx.gsplit_grouped_linear_fwd(x, ptr, order, w, None, y[:5]), lambda: ctx.gsplit_grouped_linear_fwd(x.cpu(), ptr, order, w, None, y),
           lambda: ctx.gsplit_grouped_linear_fwd(x.t().contiguous().t(), ptr, order, w, None, y), lambda: ctx.gsplit_grouped_linear_fwd(x, ptr, order, w, y, y)]
    for f in bad:
        with pytest.raises(AssertionError):
            f()
    big = torch.zeros((3000, 64), device="cuda")
    wb = torch.zeros((1, 64, 64), device="cuda")
    assert ctx.gsplit_grouped_linear_work(big, wb).numel() > 0
    with pytest.raises(AssertionError):
        ctx.gsplit_grouped_linear_bwd(big, i32(2), None, wb, big.clone(), None, wb.clone(), None, torch.zeros(8, device="cuda"))


def test_outputs_that_overlap_in_part(ctx):
    from paper_2303_13775_amd import GsplitError
    rows, n = 300, 8
    buf, ptr = torch.ones((rows + 1, n), device="cuda"), torch.tensor([0, 100, rows], dtype=torch.int32, device="cuda")
    w, ints = torch.ones((2, n, n), device="cuda"), torch.zeros(2 * rows + 2, dtype=torch.int32, device="cuda")
    dy, dw, room = torch.ones((rows, n), device="cuda"), torch.zeros((4, n, n), device="cuda"), torch.zeros((5000, n), device="cuda")
    assert ctx.gsplit_grouped_linear_work(dy, w).numel() <= room.numel()
    parts = dw.view(-1)
    calls = [lambda: ctx.gsplit_group_rows(ints[:rows], ptr, ints[rows - 1:2 * rows - 1]), lambda: ctx.gsplit_group_rows(ints[:rows], ints[rows:rows + 3], ints[rows + 2:2 * rows + 2]),
             lambda: ctx.gsplit_grouped_linear_fwd(buf[:-1], ptr, None, w, None, buf[1:]),
             lambda: ctx.gsplit_grouped_linear_bwd(buf[:-1], ptr, None, w, dy, buf[1:], None, None),
             lambda: ctx.gsplit_grouped_linear_bwd(buf[:-1], ptr, None, w, dy, None, w, None, room),
             lambda: ctx.gsplit_grouped_linear_bwd(buf[:-1], ptr, None, w, dy, None, dw[:2], parts[2 * n * n - 2:2 * n * n + 2 * n - 2].view(2, n), room),
             lambda: ctx.gsplit_grouped_linear_bwd(buf[:-1], ptr, None, dw[1:3], dy, None, dw[:2], None, room)]
    for k, call in enumerate(calls):
        with pytest.raises(GsplitError) as e:
            call()
        assert e.value.code == -1 and "overlaps" in str(e.value), k
    assert bool((buf == 1).all()) and bool((w == 1).all()) and not dw.any() and not ints.any()        # nothing was written
    # several chunks of rows, whose gradients go through the working memory: not in the place of an output
    big, wide = torch.ones((70_000, 64), device="cuda"), torch.ones((1, 64, 64), device="cuda")
    one = torch.tensor([0, 70_000], dtype=torch.int32, device="cuda")
    need = ctx.gsplit_grouped_linear_work(big, wide)
    assert need.numel() > 64 * 64
    with pytest.raises(GsplitError) as e:
        ctx.gsplit_grouped_linear_bwd(big, one, None, wide, big, None, need[:64 * 64].view(1, 64, 64), None, need)
    assert "overlaps" in str(e.value)
    # what lies side by side is taken: columns of one buffer, neighbours in one allocation
    both = torch.ones((rows, 2 * n), device="cuda")
    ctx.gsplit_grouped_linear_fwd(both[:, n:], ptr, None, w, None, both[:, :n])
    ctx.gsplit_grouped_linear_bwd(both[:, n:], ptr, None, w, dy, None, dw[:2], parts[2 * n * n:2 * n * n + 2 * n].view(2, n), room)
    assert bool((both[:, :n] == n).all()) and dw[:2, 0, 0].tolist() == [100, 200] and parts[2 * n * n].item() == 100 and not dw[2:].view(-1)[2 * n:].any()


@pytest.mark.parametrize("dtype, n_in, n_out", [(F32, 64, 64), (F32, 200, 301), (BF16, 64, 63), (BF16, 256, 256)])
def test_bias_gradients_of_many_chunks(ctx, dtype, n_in, n_out):
    """One large row, then ones too far apart to share a chunk: added to it one by one in float, each would be lost."""
    rows, apart = 70_000, 1500
    x, dy = torch.zeros((rows, n_in), dtype=dtype, device="cuda"), torch.zeros((rows, n_out), dtype=dtype, device="cuda")
    dy[0], dy[apart::apart] = 2.0**24, 1.0
    w, ptr = torch.zeros((1, n_in, n_out), dtype=dtype, device="cuda"), torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    dw, db = torch.full((1, n_in, n_out), 7.0, device="cuda"), torch.zeros((1, n_out), device="cuda")
    work = ctx.gsplit_grouped_linear_work(x, w)
    assert work.numel() > n_in * n_out                      # (there are chunks)
    ctx.gsplit_grouped_linear_bwd(x, ptr, None, w, dy, None, dw, db, work)
    want = np.float32(2.0**24 + (rows - 1) // apart)        # sums of whole numbers are exact in double: one rounding
    assert bool((db == float(want)).all()) and want > 2.0**24 and not dw.any()
