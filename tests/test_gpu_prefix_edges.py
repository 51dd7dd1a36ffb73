"""Decode attention behind shared prefixes: groups that are empty, and lengths that are cut where the groups take every block."""
import numpy as np
import pytest
import torch

from oracle import step
from paper_2609_14237_b200 import binding as B
from test_gpu_prefix import P, check, run, shared_batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()
    assert torch.cuda.is_available()


@pytest.mark.parametrize("Hq,Hkv,D,members", [(32, 8, 128, 40), (8, 2, 64, 64), (16, 1, 128, 9)])
@pytest.mark.parametrize("where", ["front", "behind", "around"])
def test_empty_groups_change_nothing(Hq, Hkv, D, members, where):
    """A captured step has as many groups as it may ever need: the empty ones neither change the result nor which kernel takes the others
    (the two would differ in their last bits)."""
    rng = np.random.default_rng(9100 + members)
    lens = [int(700 + rng.integers(1, 200)) for _ in range(members)]
    pool, tab, q, starts = shared_batch(rng, [members], [700], lens, Hq, Hkv, D)
    want, want_lse, rc = run(pool, tab, q, lens, starts, [700], Hq, Hkv, D)
    assert rc == B.OPW_OK
    check(want, want_lse, step.decode_attention(pool, Hq, Hkv, D, q, lens, tab), 900)
    front = {"front": members - 1, "behind": 0, "around": members // 2}[where]
    behind = members - 1 - front
    out, lse, rc = run(pool, tab, q, lens, [0] * (front + 1) + [members] * (behind + 1), [700] * members, Hq, Hkv, D)
    assert rc == B.OPW_OK and torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("Hq,Hkv,D,members", [(8, 2, 64, 8), (8, 1, 128, 5), (16, 4, 128, 6), (32, 8, 128, 5), (6, 2, 256, 4)])
@pytest.mark.parametrize("window", [0, 200])
def test_lengths_beyond_the_table_are_recorded_where_all_keys_are_shared(Hq, Hkv, D, members, window):
    """A prefix as long as the table: no row has keys of its own, and the groups may take every block there is."""
    rng = np.random.default_rng(9200 + Hkv + members)
    width = 320
    full = width * P
    lens = [full - 16 * b for b in range(members)]
    pool, tab, q, starts = shared_batch(rng, [members], [full], lens, Hq, Hkv, D, width=width)
    want, want_lse, rc = run(pool, tab, q, lens, starts, [full], Hq, Hkv, D, window)
    assert rc == B.OPW_OK
    check(want, want_lse, step.decode_attention(pool, Hq, Hkv, D, q, lens, tab, window), full)
    for long in (full + 1, (1 << 31) - 1):
        out, lse, rc = run(pool, tab, q, [long] + lens[1:], starts, [full], Hq, Hkv, D, window)
        assert rc == B.OPW_ERR_BAD_PAGE and torch.equal(out, want) and torch.equal(lse, want_lse)
