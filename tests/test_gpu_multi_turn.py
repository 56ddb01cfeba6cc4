"""The example of a multi-turn rollout: rotation, prefill, append and attention of chunks, drafts and single tokens together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "multi_turn.py")
    spec = importlib.util.spec_from_file_location("multi_turn", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("kv,seqs,turns,answer,draft", [("bf16", 9, 3, (1, 60), 4), ("bf16", 4, 1, (100, 150), 12), ("e4m3", 9, 2, (1, 60), 4)])
def test_turns_equal_one_pass(kv, seqs, turns, answer, draft):
    """Two layers, each of which rounds what it adds to the residual to bf16 a few times (2^-8 each, up to eight of them on the
    way): 2 * 8 * 2^-8 of the norm.  An e4m3 cache: codes are off by up to 2^-4, a third of that on average, in scores and
    values of one side alone: 0.1 for two layers."""
    worst = example().run(seqs, turns, kv, prompt=(3, 200), answer=answer, draft=draft, singles=3, seed=turns)
    assert worst <= (2 * 8 * 2.0 ** -8 if kv == "bf16" else 0.1)
