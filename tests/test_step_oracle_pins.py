"""The reference of both ends of a step, held against what follows from the definitions alone (CPU only)."""
import numpy as np
import pytest

import step_util as su


@pytest.mark.parametrize("greedy", [False, True])
def test_tokens_are_distributed_as_the_target_s(greedy):
    """Over every number on a grid (accept and draw) and every draft weighed by q, the first token of one draft's verification has the
    target's probabilities: the identity that speculative sampling rests on.  K points on each axis move a probability by at most two of
    their cells for each of the V tokens."""
    r = np.random.default_rng(3)
    V, K = 5, 60
    logits, draft = r.normal(0, 1, (2, V)), r.normal(0, 1, (1, V))
    T = [0.0 if greedy else 0.8]
    p, q = su.distribution(logits[0], T[0]), su.distribution(draft[0], T[0])
    got = np.zeros(V)
    grid = (np.arange(K) + 0.5) / K
    for x in range(V):
        for u in grid:
            for v in grid if u * q[x] >= p[x] else grid[:1]:
                _, out, _, _ = su.verify(logits, [0, 2], [0, x], [u, 0.5], [v], T, draft, [0])
                got[out[0]] += q[x] / K / (K if u * q[x] >= p[x] else 1)
    assert np.abs(got - p).max() <= (2 * V / K if not greedy else 1e-12)


def test_guesses_and_last_rows():
    logits = np.log(np.array([[0.1, 0.6, 0.3], [0.2, 0.3, 0.5]]))
    # a guess that holds by 0.6: then the second row's token
    assert su.verify(logits, [0, 2], [9, 1], [0.59, 0], [0.1]) [:2] == ([1], [1, 0])
    # one that does not: from 0.1 and 0.3 alone
    assert su.verify(logits, [0, 2], [9, 1], [0.61, 0], [0.24])[:2] == ([0], [0, -1])
    assert su.verify(logits, [0, 2], [9, 1], [0.61, 0], [0.26])[:2] == ([0], [2, -1])


def test_places_by_hand():
    table = np.array([[7, -1, -1], [3, -1, -1], [5, 6, -1]], dtype=np.int32)
    got = su.place([15, 16, 20], [2, 1, 12], [1, 1, 2], table, [10, 11, 12, 13], 3, 16)
    assert got["block_table"].tolist() == [[7, 12, -1], [3, 11, -1], [5, 6, -1]]
    assert got["cu_seqlens"].tolist() == [0, 2, 3, 15] and got["free_count_out"].tolist() == [1]
    assert got["slots"].tolist()[:4] == [7 * 16 + 15, 12 * 16, 11 * 16, 6 * 16 - 16 + 20] and got["slots"][-1] == -1
    back = su.release([15, 0, 20], [2, 1, 2], got["block_table"], [10, 11, 12, 13], 1)
    assert back["free_pages"].tolist() == [10, 12, 3, 13] and back["free_count_out"].tolist() == [3] and back["held_out"].tolist() == [1, 0, 2]
