"""The example that runs the calls around the 8-bit cache together with truncation and tree verification."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rounds_run_and_stay_inside_their_budget(tslt):
    spec = importlib.util.spec_from_file_location("cached_tree_rounds", os.path.join(ROOT, "examples", "cached_tree_rounds.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    a = example.main(rounds=60, B=3, report=lambda _: None)
    assert all(60 <= n <= 60 * 4 for n in a["emitted"]) and sum(a["emitted"]) > 3 * 60          # (some candidates are accepted)
    assert all(example.KEEP // 2 < n <= example.BUDGET for n in a["length"])
    assert a["attend"]["status"].tolist() == [0, 0, 0] and a["verify"]["status"].tolist() == [0, 0, 0]
    assert torch.isfinite(a["attend"]["out"].float()).all()
    assert example.main(rounds=60, B=3, report=lambda _: None)["emitted"] == a["emitted"]        # the same seed: the same tokens


def test_path_of_a_tree_follows_the_accepted_children(tslt):
    spec = importlib.util.spec_from_file_location("cached_tree_rounds", os.path.join(ROOT, "examples", "cached_tree_rounds.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    slots = torch.full((2, 15), -1, dtype=torch.int32)
    slots[0, 0], slots[0, 2], slots[0, 5] = 1, 0, 1                # 0 -> 2 -> 5 -> 12
    slots[1, 0] = 0                                                # 0 -> 1, whose candidates are rejected
    path = example.verified_path(slots, torch.tensor([4, 2], dtype=torch.int32), (2, 2, 2))
    assert path[0].tolist() == [0, 2, 5, 12] and path[1, :2].tolist() == [0, 1]
