"""The example's runs: one with the same seed is the same run, also in the same process."""
import importlib.util
import pathlib

import pytest

pytestmark = pytest.mark.gpu
PATH = pathlib.Path(__file__).resolve().parents[1] / "examples" / "token_policy.py"


def test_a_seed_gives_the_same_answers():
    spec = importlib.util.spec_from_file_location("token_policy_runs", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    runs = [example.main(["--vocab", "300", "--steps", "2", "--answers", "64", "--seed", s]) for s in "556"]
    first = [[m["reward_first"] for m in r["members"]] for r in runs]
    assert first[0] == first[1]                          # of each member's first answers
    assert first[0] != first[2]
