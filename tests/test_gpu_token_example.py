"""The example that uses the token losses together: its policies learn."""
import importlib.util
import pathlib

import pytest

pytestmark = pytest.mark.gpu
PATH = pathlib.Path(__file__).resolve().parents[1] / "examples" / "token_policy.py"


def test_example_learns():
    spec = importlib.util.spec_from_file_location("token_policy", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(["--vocab", "1000", "--steps", "20", "--answers", "256"])
    chance = 1 / example.CLASSES
    for member in r["members"]:
        assert abs(member["reward_first"] - chance) < 0.08          # 256 answers of about 4 tokens: 5 deviations
        assert member["reward_last"] > member["reward_first"] + 0.1
    assert abs(r["pref"]["losses"][0] - 0.6931) < 0.02              # the policy is its own reference: ln 2
    assert r["pref"]["losses"][-1] < r["pref"]["losses"][0] - 0.1
    assert r["distill"]["losses"][-1] < 0.5 * r["distill"]["losses"][0]
    assert r["distill"]["reward"] > 2 * chance
