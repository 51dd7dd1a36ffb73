"""Host side of the operators around a step's attention, and their oracle against first principles: no device needed."""
import ctypes

import numpy as np
import pytest

from oracle import step
from paper_2609_14237_b200 import binding as B


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()


def test_null_stages_are_refused():
    L = B.lib()
    assert L.opw_norm_rope_append(None, 0, 1, 64, 0, 16, 16, 64, 16, 64, 16, 64, 16, 16, 0, ctypes.c_float(1e-6), 16, 16, 16, 1, 16, 16,
                                  None) == B.OPW_ERR_INVALID_ARG
    assert L.opw_tree_verify(None, 1, 4, 8, 0, 0, 16, 8, 16, 8, *[16] * 7, None) == B.OPW_ERR_INVALID_ARG
    assert L.opw_kv_extend(None, 1, 16, 16, 16, 1, 16, 16, 1, 16, 1, 16, None, None, None, None, 0, None, None, None) == B.OPW_ERR_INVALID_ARG


def test_the_oracle_of_head_norms():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 64))
    y = step.head_norm(x, None, 1e-12)
    assert np.allclose((y * y).sum(-1), 64) and np.allclose(step.head_norm(4 * x, None, 1e-12), y)
    assert np.allclose(step.head_norm(x, np.full(64, 0.5), 1e-12), y / 2)


@pytest.mark.parametrize("draw", ["again", "distinct"])
def test_the_oracle_of_verification_keeps_the_targets_distribution(draw):
    """Whatever the drafter proposes, the first new token is distributed as the target's: summed exactly over the proposals of two siblings
    and over the intervals of the uniforms in which the decisions agree."""
    V = 4
    p, q = np.array([0.1, 0.5, 0.15, 0.25]), np.array([0.4, 0.1, 0.3, 0.2])
    got = np.zeros(V)
    mid = (np.arange(400) + 0.5) / 400                       # midpoints: the accepted share of a uniform is exact to 1/800
    for a in range(V):
        for b in range(V):
            if draw == "distinct" and a == b:
                continue
            chance = q[a] * (q[b] if draw == "again" else q[b] / (1 - q[a]))
            take = min(1.0, p[a] / q[a])
            got[a] += chance * take
            left = np.maximum(p - q, 0)
            left /= left.sum()
            q2 = q.copy()
            if draw == "distinct":
                q2[a] = 0
                q2 /= q2.sum()
            ratio = min(1.0, left[b] / q2[b]) if q2[b] > 0 else 0.0
            got[b] += chance * (1 - take) * ratio
            rest = np.maximum(left - q2, 0)
            rest = rest / rest.sum() if rest.sum() > 0 else left
            got += chance * (1 - take) * (1 - ratio) * rest
            # the oracle decides as this enumeration does
            args = (np.array([[p, p, p]]), np.array([[q, q, q]]), [[0, a, b]], [[-1, 0, 0]], [3])
            taken = [step.verify(*args, [[0.3, u, 0.999999]], draw)[0][0, 1] == 1 for u in mid]
            assert abs(np.mean(taken) - take) <= 1 / 400
            if take < 1:
                second = [step.verify(*args, [[0.3, 0.999999, u]], draw)[0][0, 1] == 2 for u in mid]
                assert abs(np.mean(second) - ratio) <= 1 / 400
                follows = [step.verify(*args, [[u, 0.999999, 0.9999999]], draw)[2][0] for u in mid]
                if ratio < 0.99:
                    assert np.abs(np.bincount(follows, minlength=V) / 400 - rest).max() <= 1 / 200
    assert np.allclose(got, p)


def test_the_oracle_of_extending():
    table, counts = np.full((3, 4), -1), np.zeros(8, np.int64)
    table[0, 0], counts[5] = 5, 1
    starts, lens, seq, slots, end, bad = step.extend([0, 2, 1], [15, 0, 0], [2, 33, 40], table, counts, [1, 2, 3, 4, 6], 5, 0, 80)
    assert starts.tolist() == [0, 2, 35, 75] and lens.tolist() == [17, 33, 0] and end == 4 and not bad
    assert table.tolist() == [[5, 1, -1, -1], [-1] * 4, [2, 3, 4, -1]] and counts.tolist() == [0, 1, 1, 1, 1, 1, 0, 0]
    assert seq.tolist() == [0] * 2 + [2] * 33 + [-1] * 45 and slots.tolist() == [15, 16, *range(33)] + [-1] * 45


def test_null_prefix_handles_are_refused():
    L, h = B.lib(), ctypes.c_void_p()
    assert L.opw_prefix_attn_workspace_bytes(None) == 0
    assert L.opw_prefix_attn_create(None, 0, 256, 1 << 30, ctypes.byref(h)) == B.OPW_ERR_INVALID_ARG and h.value is None
    assert L.opw_prefix_attention(None, 0, 1, 1, *[16] * 6, None, None) == B.OPW_ERR_INVALID_ARG
    assert L.opw_prefix_attn_destroy(None) == B.OPW_OK
