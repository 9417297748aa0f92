"""What bench.py --update goes with, and the entries of its work table (no GPU)."""
import sys

import pytest

import bench
import workloads


@pytest.mark.parametrize("args", [["--update", "--graph"], ["--update", "--redundancy"]])
def test_update_is_refused(monkeypatch, args):
    """Where two models would be trained in turn, or a step repeated, the update has no meaning."""
    monkeypatch.setattr(sys, "argv", ["bench.py"] + args)
    with pytest.raises(SystemExit):
        bench.parse()


@pytest.mark.parametrize("args", [["--update"], ["--update", "--model", "gat"], ["--redundancy"]])
def test_update_is_taken(monkeypatch, args):
    monkeypatch.setattr(sys, "argv", ["bench.py"] + args)
    assert bench.parse().update == ("--update" in args)


@pytest.mark.parametrize("model, separate, update, want", [
    ("sage", False, False, ["sample_split", "gather", "sage_step"]),
    ("sage", False, True, ["sample_split", "gather", "sage_step", "update"]),
    ("sage", True, False, ["sample_split", "gather", "sage_fwd", "loss_grad", "sage_bwd"]),
    ("gat", False, True, ["sample_split", "gather", "gat_fwd", "loss_grad", "gat_bwd", "update"])])
def test_stages_of_a_step(monkeypatch, model, separate, update, want):
    """The update is a stage of its own, not a part of the backward pass."""
    monkeypatch.setattr(bench.Runner, "separate_calls", separate)
    monkeypatch.setattr(bench.Runner, "with_update", update)
    assert bench.stage_names(model) == want


def test_work_of_the_update():
    """Bytes of the update's kernels: each gradient read, and parameter and moments read and written beside it."""
    w = workloads.tiny(device="cpu")
    rows, edges, mixed = [4000, 900, 128], [3000, 800], [10, 5]
    work, _ = bench.algorithmic_work(w, "sage", None, rows, edges, mixed, 256, 4, w.n_splits)
    assert not {"adamw", "grad_norm", "sum_slots"} & set(work)
    work, _ = bench.algorithmic_work(w, "sage", None, rows, edges, mixed, 256, 4, w.n_splits, n_params=1000)
    assert work["adamw"] == ("bytes", 28000) and work["grad_norm"] == ("bytes", 4000) and work["sum_slots"][1] > 0
