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
