"""The rules by which the losses over rows and the update take their form: a form holds the rows it is chosen for, parts fit the
scratch they are kept in, and the sizes of the GPU tests reach every form."""
import itertools

import numpy as np
import pytest

import row_rules as R

WIDTHS = sorted({1, 2, 3, 4, 7, 8, 9} | {b + d for b in (128, 256, 512, 1024, 2048, 4096, 8192, 16384, 32768, 65536, 131072) for d in (-1, 0, 1, 3, 4, 7, 8)}
                | {140001, 1 << 20, 2 ** 31 - 1})


@pytest.mark.parametrize("piece", [4, 8])
def test_a_form_holds_its_rows(piece):
    for rows, C in itertools.product((1, 100, 257, 10 ** 6), WIDTHS):
        f = R.form(rows, C, piece)
        if f == "STREAMED":
            assert C > 65536
            continue
        lanes, elements = (int(x) for x in f.replace("_RAW", "").split("x"))
        assert C // piece * piece <= lanes * elements, (C, f)       # the whole pieces
        assert C % piece < 16 <= lanes and elements % piece == 0     # and a lane each for what is behind them
        assert not f.endswith("RAW") or piece == 8


def test_parts_fit_the_scratch():
    L = R.lib()
    for rows, C in itertools.product((1, 2, 3, 7, 64, 127, 200, 255), (8193, 10000, 65536, 65537, 131072, 10 ** 6, 2 ** 31 - 1)):
        n = L.chunks(rows, C, R.N_CU)
        assert 1 <= n <= 64 and n * rows <= L.parts_held()
        step = -(-(-(-C // n)) // 8) * 8            # elements of a part, as the launch rounds them
        assert -(-C // step) <= n
        # every part has an element: the last one begins inside the row
        assert (-(-C // step) - 1) * step < C
    for rows, C, piece in itertools.product((1, 100, 127, 128, 255, 256, 10 ** 5), WIDTHS, (4, 8)):
        if L.policy_parts(rows, C, piece, R.N_CU):
            assert rows < R.N_CU and C > 65536
        if L.preference_parts(rows, C, R.N_CU):
            assert rows < R.N_CU and C > 8192


def test_workgroups_of_pairs():
    L = R.lib()
    for rows, pairs, C in itertools.product((1, 2, 64, 1000, 10 ** 5, 10 ** 9), (1, 2, 100, 512, 10 ** 5, 1 << 24, 10 ** 9), (1, 47, 256, 257, 4096, 4097, 65536)):
        t = L.whole(rows, pairs, C, R.N_CU)
        assert t in (0, 64, 256, 1024) and (not t or t >= L.part(C)) and (t in (0, 256) or L.part(C) < 256)
        assert not t or pairs * t < 2 ** 32


def test_chunks_of_the_update():
    L = R.lib()
    for total in (0, 1, 1000, 10 ** 6, 10 ** 9, 2 ** 46):
        for c, most in ((L.chunk(total, 4096, R.N_CU), 2 ** 23), (L.chunk(total, 2048, R.N_CU), 2 ** 23), (L.chunk_norm(total, R.N_CU), 2 ** 30)):
            assert c % 1024 == 0 and total / c <= most and c < 2 ** 31 // 16
        assert not L.clip_small(total) or total <= 32768


def test_gpu_tests_reach_every_form():
    """The sizes that tests/test_gpu_row_losses.py runs, as (rows, classes)."""
    import test_gpu_row_losses as G
    policy = [(37 if C > 300 else 333, C) for C in G.WIDTHS] + [(n, C) for n in (1, 5) for C in (16383, 32768, 65536, 65537, 131071, 140001)]
    policy += [(300, 16385), (270, 33001), (600, 9000)] + G.POLICY_FORMS
    seen = {(R.form(n, C, piece), piece) for n, C in policy for piece in (4, 8) if not R.lib().policy_parts(n, C, piece, R.N_CU)}
    want = {(f, p) for f in R.FORMS for p in (4, 8)} - {("64x32", 4), ("256x8", 8), ("512x128_RAW", 4), ("1024x128_RAW", 4)}
    assert seen == want, want ^ seen
    assert any(R.lib().policy_parts(n, C, p, R.N_CU) for n, C in policy for p in (4, 8))
    pairs = [(len(l) // 2, int(np.sum(l)), C) for l, C in G.PREFERENCE_FORMS]
    got = {(R.lib().part(C), R.lib().whole(n, p, C, R.N_CU)) for p, n, C in pairs}
    assert got == {(16, 64), (16, 256), (16, 1024), (16, 0), (64, 64), (64, 256), (64, 1024), (64, 0), (256, 256), (256, 0)}, got
    parts = {bool(R.lib().preference_parts(n, C, R.N_CU)) for p, n, C in pairs if not R.lib().whole(n, p, C, R.N_CU) and R.lib().part(C) == 256}
    assert parts == {False, True}


@pytest.mark.parametrize("rows, pairs, C", [(8 * 512, 512, 65536), (8 * 512, 512, 20000), (4 * 512, 512, 20000), (2 * 512 - 100, 512, 65536), (190, 100, 8000), (64 * 16, 16, 2048),
                                            (32 * 128, 128, 2048), (32 * 256, 256, 2048), (32 * 1024, 1024, 2048), (64 * 1024, 1024, 172), (128 * 64, 64, 172)])
def test_pairs_whose_longest_may_be_all_of_the_call(rows, pairs, C):
    """Pairs of which one alone keeps a workgroup busy for several rounds: the host knows their mean only, a batch of ragged ones would
    wait for the longest (512 pairs of 65536 classes, one of them with half of 4096 rows: 57.6 ms, 0.55 by three launches)."""
    assert R.lib().whole(rows, pairs, C, R.N_CU) == 0


@pytest.mark.parametrize("rows, pairs, C", [(2 * 512, 512, 47), (33 * 256, 256, 172), (2 * 512, 512, 65536), (2, 1, 5000), (64 * 512, 512, 172), (32 * 2048, 2048, 172),
                                            (8 * 4096, 4096, 2048), (16 * 16384, 16384, 172), (2 * 4096, 4096, 20000), (8 * 512, 512, 172)])
def test_pairs_of_a_workgroup_each(rows, pairs, C):
    assert R.lib().whole(rows, pairs, C, R.N_CU)
