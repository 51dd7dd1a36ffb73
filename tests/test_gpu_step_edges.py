"""The operators around a step's attention where they are easiest to get wrong: drafters that are sure of themselves, uniforms of 0 behind refused
tokens, groups that are empty, lengths that are cut where no row has keys of its own, maps at the end of 32 bits."""
import numpy as np
import pytest
import torch

from paper_2609_14237_b200 import binding as B
from test_gpu_step import run_verify, same_as_oracle, small_stage

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()
    assert torch.cuda.is_available()


# ---------------------------------------------------------------------------- verification ---

def sure_drafter(rng, n, T, V, tail, kind, near):
    """A drafter that gives all but `tail` to one token and the rest to seven others, a target that spreads over a dozen; the drafted siblings
    are the likely ones, drawn without replacement.  `near`: all of them among the first tokens, else anywhere."""
    target, q = np.zeros((n, T, V)), np.zeros((n, T, V))
    tokens, parents = np.zeros((n, T), np.int64), np.zeros((n, T), np.int64)
    parents[:, 0] = -1
    for b in range(n):
        pick = rng.permutation(min(V, 40) if near else V)[:16]
        for i in range(T):
            target[b, i, pick[:12]] = rng.dirichlet(np.ones(12))
            q[b, i, pick[0]] = 1.0
            q[b, i, pick[1:8]] = tail * rng.dirichlet(np.ones(7))
        way = np.concatenate([pick[:1], rng.permutation(pick[1:8])])
        for i in range(1, T):
            if b % 3 == 2 and i > T // 2:                                 # (some below the first child)
                parents[b, i] = 1
            tokens[b, i] = way[(parents[b, :i] == parents[b, i]).sum()]
    u = rng.random((n, T))
    u[:, 1] = np.where(rng.random(n) < 0.8, 1 - 2.0 ** -24, u[:, 1])      # the likeliest is refused unless the target has nothing else
    f = lambda x: torch.from_numpy(x).to(kind).cuda()  # noqa: E731
    return f(target), f(q), tokens, parents, np.full(n, T), u


@pytest.mark.parametrize("tail", [1e-6, 1e-13, 1e-16, 1e-17, 1e-22, 1e-30])
@pytest.mark.parametrize("n,V,near", [(40, 40, True), (64, 4099, True), (1, 70001, False), (300, 1000, False)])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_verify_distinct_behind_a_sure_drafter(tail, n, V, near, kind):
    """What the drafter has left once its likeliest token is refused is not lost beside it: the next sibling counts with its share of that."""
    rng = np.random.default_rng(9000 + V)
    st = small_stage()
    for T in (3, 6, 9):
        args = sure_drafter(rng, n, T, V, tail, kind, near)
        same_as_oracle(run_verify(st, *args, distinct=True), *args, "distinct")
    assert st.poll_error() == B.OPW_OK


@pytest.mark.parametrize("V,batch", [(257, 200), (4099, 64), (70001, 3)])
@pytest.mark.parametrize("draw", ["distinct", "certain"])
def test_verify_draws_behind_parts_of_refused_tokens(V, batch, draw):
    """Uniforms of 0 where nothing but refused tokens come first: the token that follows is the first that is left, never one of those and never
    none, whatever the rounding of sums over them."""
    rng = np.random.default_rng(9100 + V)
    st, T = small_stage(), 7
    parents = np.zeros((batch, T), np.int64)
    parents[:, 0] = -1
    target, q = np.zeros((batch, T, V)), np.zeros((batch, T, V))
    tokens, u = np.zeros((batch, T), np.int64), np.full((batch, T), 1 - 2.0 ** -24)
    u[:, 0] = 0.0
    for b in range(batch):
        kids = rng.permutation(min(V - 5, 200))[:T - 1]
        small = 10.0 ** -rng.uniform(0.5, 14, size=T - 1)
        target[b, :, kids] = np.minimum(0.4 * small / small.sum(), 0.1)[:, None]     # less than the drafter's, whose rest is 0.6 at most:
        target[b, :, V - 3:V - 1] = 0.3                                              # refused, and left nothing
        q[b, :, kids] = 0.9 / (T - 1)
        q[b, :, 0] += 0.1
        tokens[b, 1:] = kids
    f = lambda x: torch.from_numpy(x).to(torch.float32).cuda()  # noqa: E731
    args = (f(target), None if draw == "certain" else f(q), tokens, parents, np.full(batch, T), u)
    got = run_verify(st, *args, distinct=draw == "distinct")
    want = same_as_oracle(got, *args, draw)
    assert (want[1] == 1).all() and (want[2] == V - 3).all() and st.poll_error() == B.OPW_OK


@pytest.mark.parametrize("draw", ["distinct", "certain"])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("batch,V", [(3, 1031), (2, 4099), (1, 70001)])
def test_verify_leaves_out_tokens_wherever_they_lie(draw, kind, batch, V):
    """Refused tokens at the ends of the row, of words, of a warp's steps and of the blocks' parts, many of them side by side; rows that begin
    anywhere, alike and not."""
    rng = np.random.default_rng(9300 + V)
    st, T = small_stage(), 40
    spots = np.unique(np.clip([0, 1, 2, 3, 4, 7, 8, 9, 15, 16, 31, 32, 63, 64, 126, 127, 128, 129, 255, 256, 257, 511, 512, 513, 514, 515, 1023, 1024, 1025,
                               V // 2 - 1, V // 2, V // 2 + 1, 4095, 4096, V - 4, V - 3, V - 2, V - 1], 0, V - 1))
    soft = lambda z: np.exp(z) / np.exp(z).sum(-1, keepdims=True)  # noqa: E731
    for pad, off, off_q in ((0, 0, 0), (5, 1, 1), (3, 3, 2)):
        x = rng.standard_normal((batch, T, V))
        y = x + rng.standard_normal((batch, T, V))
        x[:, :, spots] += -3.0 if draw == "distinct" else 2.0             # (refused: the drafter likes them more)
        y[:, :, spots] += 3.0
        tokens, parents = np.zeros((batch, T), np.int64), np.zeros((batch, T), np.int64)
        parents[:, 0] = -1
        for b in range(batch):
            way = rng.permutation(spots)[:T - 1]
            tokens[b, 1:1 + len(way)] = way
            tokens[b, 1 + len(way):] = way[0]                             # (a token that is refused already)
        u = np.full((batch, T), 1 - 2.0 ** -24)
        u[:, 0] = rng.random(batch)
        views = []
        for z, o in ((x, off), (y, off_q)):
            flat = torch.full((batch * T * (V + pad) + o + 64,), float("nan"), dtype=kind, device="cuda")
            view = flat[o:o + batch * T * (V + pad)].view(batch, T, V + pad)[..., :V]
            view.copy_(torch.from_numpy(soft(z)))
            views.append(view)
        args = (views[0], None if draw == "certain" else views[1], tokens, parents, np.full(batch, T), u)
        same_as_oracle(run_verify(st, *args, distinct=draw == "distinct"), *args, draw)
    assert st.poll_error() == B.OPW_OK


# ---------------------------------------------------------------------------- pages for requests ---

@pytest.mark.parametrize("room,off", [((1 << 31) - 1, 0), ((1 << 31) - 1, 1), ((1 << 31) - 65536 + 8, 0)])
def test_extend_with_maps_at_the_end_of_32_bits(room, off):
    """The largest maps there can be: a thread's next rows lie beyond 32 bits and are not written.  (Also at an odd address, word by word.)"""
    st = small_stage(width=8)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    tab = torch.full((4, 8), -1, dtype=torch.int32, device="cuda")
    refs, free, starts, lens = torch.zeros(40, dtype=torch.int32, device="cuda"), torch.arange(40, device="cuda").int(), i32([0] * 4), i32([0] * 3)
    seq, slots = (torch.full((room + off,), -77, dtype=torch.int32, device="cuda") for _ in range(2))
    st.kv_extend(i32([2, 0, 3]), i32([0, 0, 0]), i32([100, 1, 17]), tab, refs, free, i32([40]), row_starts=starts, new_lens=lens, seq=seq[off:],
                 slots=slots[off:])
    assert st.poll_error() == B.OPW_OK and starts.tolist() == [0, 100, 101, 118] and lens.tolist() == [100, 1, 17]
    assert seq[off:off + 118].tolist() == [2] * 100 + [0] + [3] * 17 and slots[off:off + 118].tolist() == [*range(100), 0, *range(17)]
    for x in (seq, slots):
        assert (x[:off] == -77).all()
        for lo in range(off + 118, room + off, 1 << 28):
            assert (x[lo:lo + (1 << 28)] == -1).all()
