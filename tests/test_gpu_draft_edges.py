"""GPU tests of the drafted-token and page operators where their protocols and choices have edges: runs of short key ranges,
scores that rise along the keys, layers that differ, many layers, values at the ends of their types."""
import math

import numpy as np
import pytest
import torch

import oracle
from helpers import P, out_to_f64, rand_bits
from oracle import draft
from paper_2609_14237_b200 import binding as B
from test_gpu_draft import check_tree, dev, host_bits, make_stage, random_tree, tree_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()
    assert torch.cuda.is_available()


# ---------------------------------------------------------------------------- tree attention ---

@pytest.mark.parametrize("Hq,Hkv,D,T", [(32, 8, 128, 5), (8, 2, 64, 9), (32, 8, 128, 40)])
@pytest.mark.parametrize("long", [0, 7])
def test_runs_of_row_blocks_of_one_key_tile(Hq, Hkv, D, T, long):
    """Workers whose shares are row blocks of a single key tile, one after the other (`long`: every so many sequences one of three
    tiles between them): of two slots that take turns only one has a tile.  Thirty sequences, many times over."""
    rng = np.random.default_rng(2000 + Hq + T + long)
    kinds, times = 30, 16
    ctx = [int(x) for x in rng.integers(0, 60 - min(T, 24), size=kinds)]
    size = [int(x) for x in rng.integers(max(1, min(T, 24) // 2), min(T, 24) + 1, size=kinds)]
    if long:
        ctx[::long] = [150] * len(ctx[::long])
    pool, tab, q, mask, pos = tree_inputs(rng, ctx, size, T, Hq, Hkv, D)
    ref = draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, ctx, size, tab)
    st = make_stage([dev(pool, True)], Hq, Hkv, D, kinds * times, tab.shape[1])
    tree = B.TreeAttention(st, T)
    many = lambda a: np.concatenate([a] * times)  # noqa: E731
    i32 = lambda a: dev(many(np.asarray(a, np.int32)))  # noqa: E731
    args = (dev(many(q), True), dev(many(mask)), i32(pos), i32(ctx), i32(size), i32(tab))
    first = None
    for _ in range(5):
        out = torch.full_like(args[0], float("nan"))
        lse = torch.full(out.shape[:3], float("nan"), device="cuda")
        tree.attention(0, *args, out, lse)
        if first is None:
            first = out.clone(), lse.clone()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    assert st.poll_error() == B.OPW_OK
    check_tree(first[0], first[1], [many(a) for a in ref], 300)
