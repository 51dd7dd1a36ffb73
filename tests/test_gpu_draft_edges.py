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


@pytest.mark.parametrize("Hq,Hkv,D", [(32, 8, 128), (8, 2, 64), (16, 2, 256)])
def test_positions_far_below_the_context_count_as_its_length(Hq, Hkv, D):
    """A position below the context's length counts as that length, the type's lowest value too: the same bits.  (A hidden key would
    show, and so would another path through the kernel: the infinity sits at a key whose weight has left the range of 32 bits.)"""
    rng = np.random.default_rng(2100 + D)
    T, ctx, size = 5, [1000, 300], [5, 4]
    pool, tab, q, mask, _ = tree_inputs(rng, ctx, size, T, Hq, Hkv, D)
    q = oracle.f32_to_bf16_bits(np.ones((2, T, Hq, D), np.float32))
    far = oracle.f32_to_bf16_bits(np.full((Hkv, D), -32.0, np.float32))
    for b in range(2):
        v = rand_bits(rng, (Hkv, D))
        v[:, 3] = 0x7F80
        draft._put_row(pool, Hkv, D, tab[b, 0], 5, far, v)
    st = make_stage([dev(pool, True)], Hq, Hkv, D, 2, tab.shape[1], window=2000)
    tree, res = B.TreeAttention(st, T), []
    for low in (None, 0, -(1 << 31)):
        at = np.tile(np.asarray(ctx, np.int32)[:, None], (1, T)) if low is None else np.full((2, T), low, np.int32)
        out, lse = torch.empty(2, T, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(2, T, Hq, device="cuda")
        tree.attention(0, dev(q, True), dev(mask), dev(at), dev(np.array(ctx, np.int32)), dev(np.array(size, np.int32)), dev(tab), out, lse)
        res.append((out.view(torch.int16), lse.view(torch.int32)))
    assert st.poll_error() == B.OPW_OK
    for out, lse in res[1:]:
        assert torch.equal(out, res[0][0]) and torch.equal(lse, res[0][1])


def test_masks_of_full_trees_as_unsigned_words():
    """The words that opw_tree_mask returns for a tree of 64 do not all fit a signed 64-bit integer: as torch.uint64 they are taken as
    they are."""
    rng = np.random.default_rng(2150)
    Hq, Hkv, D, T = 8, 2, 64, 64
    pool, tab, q, _, _ = tree_inputs(rng, [40], [T], T, Hq, Hkv, D)
    words, depth = B.opw_tree_mask([i - 1 for i in range(T)])
    mask = torch.tensor([words], dtype=torch.uint64, device="cuda")
    pos = 40 + np.array([depth], np.int32)
    ref = draft.tree_attention(pool, Hq, Hkv, D, q, np.array([words], np.uint64), pos, [40], [T], tab)
    st = make_stage([dev(pool, True)], Hq, Hkv, D, 1, tab.shape[1])
    tree = B.TreeAttention(st, T)
    out, lse = torch.empty(1, T, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(1, T, Hq, device="cuda")
    args = dev(pos), dev(np.array([40], np.int32)), dev(np.array([T], np.int32)), dev(tab)
    tree.attention(0, dev(q, True), mask, *args, out, lse)
    assert st.poll_error() == B.OPW_OK
    check_tree(out, lse, ref, 104)
    signed = torch.empty_like(out)
    tree.attention(0, dev(q, True), mask.view(torch.int64), *args, signed)
    assert torch.equal(signed, out)
    with pytest.raises(ValueError):
        tree.attention(0, dev(q, True), mask.view(torch.float64), *args, out)


def test_rotary_append_ignores_strides_of_single_rows_and_heads():
    """The stride of an axis of one element says nothing: torch calls such tensors contiguous whatever it is."""
    g = torch.Generator(device="cuda")
    g.manual_seed(21)
    x = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    rope, tab = B.Rope(64), i32([[0, 1]])
    for Hq, Hkv, rows in ((4, 1, 3), (4, 2, 1), (1, 1, 5), (1, 1, 1)):
        q, k, v = (x(h, rows, 64).transpose(0, 1) for h in (Hq, Hkv, Hkv))
        if rows > 1 and Hq > 1:
            q = q.contiguous()
        pools = [torch.zeros(2 * Hkv * 2 * 16 * 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        at, seq, res = i32(list(range(7, 7 + rows))), i32([0] * rows), []
        for pool, plain in zip(pools, (True, False)):
            st = make_stage([pool], Hq, Hkv, 64, 1, 2)
            plain_of = lambda t: torch.empty(t.shape, dtype=t.dtype, device="cuda").copy_(t)  # noqa: E731
            a, b, c = (plain_of(t) if plain else t for t in (q, k, v))
            out = torch.empty(rows, Hq, 64, dtype=torch.bfloat16, device="cuda")
            st.rope_append(0, rope, a, b, c, seq, at, at, tab, out)
            assert st.poll_error() == B.OPW_OK
            res.append(out)
            if rows == 1 and not plain:                          # in place too
                st.rope_append(0, rope, a, b, c, seq, at, at, tab, a)
                assert torch.equal(a, out)
        assert torch.equal(res[0], res[1]) and torch.equal(pools[0], pools[1])


@pytest.mark.parametrize("D", [64, 128, 256])
def test_commit_records_rows_in_place_on_bad_pages(D):
    """An accepted row that is in its place already has nothing to move, but a page or a slot that does not exist is recorded."""
    rng = np.random.default_rng(2300 + D)
    Hkv, T, width = 2, 6, 3
    pool = rand_bits(rng, oracle.pool_elems(8, Hkv, P, D))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for table, ctx, took, status in (([[5, 2, 7]], 14, 4, B.OPW_OK), ([[5, -1, 7]], 14, 4, B.OPW_ERR_BAD_PAGE), ([[5, -1, 7]], 14, 2, B.OPW_OK),
                                     ([[5, 8, 7]], 15, 3, B.OPW_ERR_BAD_PAGE), ([[5, 2, 7]], 46, 2, B.OPW_OK),
                                     ([[5, 2, 7]], 46, 3, B.OPW_ERR_BAD_PAGE)):
        d_pool = dev(pool, True)
        st = make_stage([d_pool], Hkv, Hkv, D, 1, width)
        new = i32([-9])
        st.kv_commit([0], i32([list(range(T))]), i32([took]), i32([ctx]), i32(table), new)
        assert st.poll_error() == status, (table, ctx, took)
        assert new.item() == ctx + took and (host_bits(d_pool) == pool).all()


def test_commit_refuses_lengths_that_overlap_what_it_reads():
    """new_lens is written while other blocks still read the path and the page table."""
    st = make_stage([torch.zeros(4 * 2 * 16 * 64, dtype=torch.bfloat16, device="cuda")], 1, 1, 64, 4, 2)
    buf = torch.zeros(64, dtype=torch.int32, device="cuda")
    base, h = buf.data_ptr(), B.lib()
    layers = (B.ctypes.c_int32 * 1)(0)
    # accepted [2, 3] at 0..5, accepted_lens at 8, ctx_lens at 12, page table [2, 2] at 16..19
    call = lambda new: h.opw_kv_commit(st.handle, layers, 1, 2, 3, base, base + 32, base + 48, base + 64, new, None)  # noqa: E731
    for at in (0, 1, 5, 7, 8, 9, 11, 12, 13, 15, 16, 19):
        assert call(base + 4 * at) == B.OPW_ERR_INVALID_ARG, at
    assert st.launch_count() == 0
    for at in (6, 10, 14, 20):
        assert call(base + 4 * at) == B.OPW_OK, at
    torch.cuda.synchronize()


def test_tree_attention_refuses_outputs_that_overlap():
    """out and lse are written while other blocks still read the inputs."""
    st = make_stage([torch.zeros(4 * 2 * 16 * 64, dtype=torch.bfloat16, device="cuda")], 1, 1, 64, 2, 2)
    tree = B.TreeAttention(st, 3)
    buf = torch.zeros(8192, dtype=torch.uint8, device="cuda")
    base, h = buf.data_ptr(), B.lib()
    at = dict(q=0, mask=1024, pos=1088, ctx=1120, sizes=1136, table=1152, out=2048, lse=4096)    # [2, 3, 1, 64]: q and out 768 bytes

    def call(**other):
        a = {k: base + v for k, v in {**at, **other}.items()}
        return h.opw_tree_attention(tree.handle, 0, 2, 3, a["q"], a["mask"], a["pos"], a["ctx"], a["sizes"], a["table"], a["out"], a["lse"],
                                    None)

    for other in (dict(lse=0), dict(lse=764), dict(lse=1024), dict(lse=1068), dict(lse=1088), dict(lse=1120), dict(lse=1136), dict(lse=1164),
                  dict(lse=2048), dict(lse=2812), dict(out=512), dict(out=1024), dict(out=1152), dict(out=400)):
        assert call(**other) == B.OPW_ERR_INVALID_ARG, other
    assert st.launch_count() == 0
    assert call() == call(lse=2816) == call(lse=1168) == B.OPW_OK
    torch.cuda.synchronize()
    assert st.poll_error() == B.OPW_OK


def test_rotary_append_refuses_queries_over_what_it_reads():
    """q_out is written while other rows' numbers are still read."""
    st = make_stage([torch.zeros(4 * 2 * 16 * 64, dtype=torch.bfloat16, device="cuda")], 1, 1, 64, 2, 2)
    buf = torch.zeros(8192, dtype=torch.uint8, device="cuda")
    base, h = buf.data_ptr(), B.lib()
    at = dict(table=64, q=512, k=1152, v=1792, seq=2448, slots=2480, pos=2512, pages=2544, out=4096)    # 5 rows of 128 bytes
    buf[2448:2448 + 20] = 255                                    # padding rows: nothing is read or written for them

    def call(out):
        a = {k: base + x for k, x in at.items()}
        return h.opw_rope_append(st.handle, 0, 5, 64, 0, a["table"], a["q"], 64, a["k"], 64, a["v"], 64, a["seq"], a["slots"], a["pos"], 2,
                                 a["pages"], base + out, None)

    for out in (0, 320, 528, 1104, 1776, 1936, 2432, 2464, 2480, 2496, 2544):
        assert call(out) == B.OPW_ERR_INVALID_ARG, out
    assert st.launch_count() == 0
    assert call(512) == call(2560) == call(4096) == B.OPW_OK
    torch.cuda.synchronize()
    assert st.poll_error() == B.OPW_OK


def rising_case(rng, shape, ctx, T, Hq, Hkv, D, gain):
    """Keys along one direction that the queries share, with a factor per key: scores go as `shape` says, `gain` log2 units (at the
    default scale) from its 0 to its 1."""
    size = [T] * len(ctx)
    pool, tab, q, mask, pos = tree_inputs(rng, ctx, size, T, Hq, Hkv, D)
    u = np.sign(rng.standard_normal((Hkv, D)))
    f32 = lambda x: oracle.f32_to_bf16_bits(x.astype(np.float32))  # noqa: E731
    q = f32(np.repeat(u, Hq // Hkv, 0) * (1 + 0.05 * rng.standard_normal((len(ctx), T, Hq, D))))
    unit = gain / (math.sqrt(D) * math.log2(math.e))             # of the keys' factor: a score of 1 is sqrt(D) at the default scale
    for b, c in enumerate(ctx):
        n = c + T
        at = np.arange(n)
        a = {"rise": at / n, "fall": 1 - at / n, "alternate": ((at // 64) % 2).astype(float), "steps": np.floor(at / 64) * 64 / n,
             "spike": (at == n // 2).astype(float)}[shape]
        k = f32(u[None] * (unit * a)[:, None, None] + 0.3 * rng.standard_normal((n, Hkv, D)))
        _, v = oracle.gather_logical(pool, Hkv, P, D, tab[b], 0, n)
        oracle.scatter_logical(pool, Hkv, P, D, tab[b], k, v)
    return pool, tab, q, mask, pos, size


@pytest.mark.parametrize("Hq,Hkv,D,T", [(32, 8, 128, 6), (32, 8, 128, 40), (8, 2, 64, 6), (8, 2, 64, 40), (32, 8, 128, 3), (16, 2, 256, 3)])
@pytest.mark.parametrize("shape,gain", [("rise", 30), ("rise", 400), ("fall", 60), ("alternate", 11), ("alternate", 40), ("steps", 200),
                                        ("spike", 25)])
@pytest.mark.parametrize("times", [1, 14])
def test_scores_that_rise_and_fall_along_the_keys(Hq, Hkv, D, T, shape, gain, times):
    """A row's maximum is raised many times, by little and by much, in the middle of what a worker holds and between the parts that are
    merged (alternate tiles of two slots, partials of many workers).  `times`: once, a few tiles a worker; many times over, dozens."""
    rng = np.random.default_rng(2500 + Hq + D + T + gain)
    ctx = [1290, 517, 96]
    pool, tab, q, mask, pos, size = rising_case(rng, shape, ctx, T, Hq, Hkv, D, gain)
    ref = draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, ctx, size, tab)
    if shape != "fall":                                          # the maximum does pass the kernel's threshold of 2^8 from tile to tile
        k, _ = oracle.gather_logical(pool, Hkv, P, D, tab[0], 0, ctx[0])
        x = oracle.bf16_bits_to_f64(k)[:, 0] @ oracle.bf16_bits_to_f64(q)[0, 0, 0] / math.sqrt(D) * math.log2(math.e)
        tops = np.maximum.accumulate([x[i:i + 64].max() for i in range(0, len(x), 64)])
        assert tops[-1] > tops[0] + 8
    many = lambda a: np.concatenate([a] * times)  # noqa: E731
    i32 = lambda a: dev(many(np.asarray(a, np.int32)))  # noqa: E731
    st = make_stage([dev(pool, True)], Hq, Hkv, D, 3 * times, tab.shape[1])
    tree = B.TreeAttention(st, T)
    out = torch.empty(3 * times, T, Hq, D, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(3 * times, T, Hq, device="cuda")
    tree.attention(0, dev(many(q), True), dev(many(mask)), i32(pos), i32(ctx), i32(size), i32(tab), out, lse)
    assert st.poll_error() == B.OPW_OK
    check_tree(out, lse, [many(a) for a in ref], 1400)


@pytest.mark.parametrize("scale", [0.02, 1.0, 4.0])
@pytest.mark.parametrize("Hq,Hkv,D,T", [(32, 8, 128, 9), (8, 2, 64, 64), (6, 2, 256, 5)])
def test_other_softmax_scales(Hq, Hkv, D, T, scale):
    rng = np.random.default_rng(2600 + D + T)
    ctx, size = [700, 31, 0, 200], [T, max(1, T - 3), T, 1]
    pool, tab, q, mask, pos = tree_inputs(rng, ctx, size, T, Hq, Hkv, D)
    ref = draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, ctx, size, tab, scale=scale)
    st = make_stage([dev(pool, True)], Hq, Hkv, D, 4, tab.shape[1], softmax_scale=scale)
    tree = B.TreeAttention(st, T)
    out, lse = torch.empty(4, T, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(4, T, Hq, device="cuda")
    tree.attention(0, dev(q, True), dev(mask), dev(pos), dev(np.array(ctx, np.int32)), dev(np.array(size, np.int32)), dev(tab), out, lse)
    assert st.poll_error() == B.OPW_OK
    check_tree(out, lse, ref, 800)


@pytest.mark.parametrize("Hq,Hkv,D,T", [(32, 8, 128, 7), (8, 2, 64, 40), (6, 2, 256, 5)])
def test_every_layer_has_its_own_window_pool_and_pages(Hq, Hkv, D, T):
    """Tree attention and rotary append on the layers of a stage that differ in all of these, out of order."""
    rng = np.random.default_rng(2700 + D)
    ctx, size, windows = [200, 37, 90], [T, T, max(1, T - 2)], [0, 33, 7, 0]
    layers = [tree_inputs(rng, [c + 16 * i for c in ctx], size, T, Hq, Hkv, D) for i in range(4)]
    width = max(x[1].shape[1] for x in layers)
    d_pools = [dev(x[0], True) for x in layers]
    assert len({p.numel() for p in d_pools}) == 4
    st = B.Stage(pools=d_pools, layer_window=windows, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, max_batch=3, max_pages_per_seq=width)
    tree, rope = B.TreeAttention(st, T), B.Rope(D)
    i32 = lambda a: dev(np.asarray(a, np.int32))  # noqa: E731
    for i in (2, 0, 3, 1):
        pool, tab, q, mask, pos = layers[i]
        tab = np.concatenate([tab, np.full((3, width - tab.shape[1]), -1, np.int32)], 1)
        at = [c + 16 * i for c in ctx]
        out, lse = torch.empty(3, T, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(3, T, Hq, device="cuda")
        tree.attention(i, dev(q, True), dev(mask), dev(pos), i32(at), i32(size), i32(tab), out, lse)
        assert st.poll_error() == B.OPW_OK
        check_tree(out, lse, draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, at, size, tab, windows[i]), 300)
        # three rows at position 0, where the rotation leaves every bit: only this layer's pool changes
        k, v = rand_bits(rng, (3, Hkv, D)), rand_bits(rng, (3, Hkv, D))
        slots = [5, 17, 2]
        st.rope_append(i, rope, None, dev(k, True), dev(v, True), i32([0, 1, 2]), i32(slots), i32([0, 0, 0]), i32(tab), None)
        draft.append_rows(pool, Hkv, D, [0, 1, 2], slots, tab, k, v)
        for j in range(4):
            assert (host_bits(d_pools[j]) == layers[j][0]).all(), (i, j)
    # a page that the largest pool has and the smallest has not
    small, large = 0, max(range(4), key=lambda i: d_pools[i].numel())
    last = d_pools[large].numel() // (2 * Hkv * 16 * D) - 1
    bad = i32([[last] * width] * 3)
    row = dev(rand_bits(rng, (1, Hkv, D)), True)
    for i, status in ((large, B.OPW_OK), (small, B.OPW_ERR_BAD_PAGE)):
        _, _, q, mask, pos = layers[i]
        tree.attention(i, dev(q, True), dev(mask), dev(pos), i32([0, 3, 6]), i32(size), bad, out, lse)
        assert st.poll_error() == status, i
        st.rope_append(i, rope, None, row, row, i32([1]), i32([3]), i32([3]), bad, None)
        assert st.poll_error() == status, i


# ----------------------------------------------------------------------------- many layers ---

@pytest.mark.parametrize("layers", [64, 65, 130])
def test_commit_and_fork_over_more_layers_than_a_launch_takes(layers):
    """Beside good ones a fork that is refused in every launch (its target is named twice), and one whose page lies beyond the smallest
    pool; the path of one sequence crosses pages."""
    rng = np.random.default_rng(2800 + layers)
    Hkv, D, T, rows, width = 1, 64, 9, 8, 3
    sizes = [14 + (i * 5) % 3 for i in range(layers)]
    pools = [rand_bits(rng, oracle.pool_elems(n, Hkv, P, D)) for n in sizes]
    order = [int(x) for x in rng.permutation(layers)]
    tab, counts = np.full((rows, width), -1, np.int32), np.zeros(min(sizes), np.int32)
    tab[:2] = rng.permutation(12)[:6].reshape(2, 3)
    counts[tab[:2].ravel()] = 1
    d_pools, d_tab, d_counts = [dev(p, True) for p in pools], dev(tab), dev(counts)
    st = make_stage(d_pools, Hkv, Hkv, D, rows, width)
    i32 = lambda a: dev(np.asarray(a, np.int32))  # noqa: E731
    acc, took, ctx, new = [[0, 2, 3, 8, 1, 0, 0, 0, 0], [4, 4, 7, 0, 0, 0, 0, 0, 0]], [4, 3], [11, 30], i32([-1, -1])
    st.kv_commit(order, i32(acc), i32(took), i32(ctx), i32(tab[:2]), new)
    assert st.poll_error() == B.OPW_OK and st.launch_count() == (layers + 63) // 64
    for p in pools:
        want = draft.commit(p, Hkv, D, np.array(acc), np.array(took), np.array(ctx), tab[:2], T)
    assert (new.cpu().numpy() == want).all()
    for p, d in zip(pools, d_pools):
        assert (host_bits(d) == p).all()
    fresh = [int(x) for x in np.nonzero(counts == 0)[0]]
    src, dst, lens, pages = [0, 1, 0, 1, 1], [4, 5, 6, 6, 7], [21, 37, 16, 16, 5], [fresh[0], fresh[1], 0, 0, min(sizes)]
    before = st.launch_count()
    st.kv_fork(order, i32(src), i32(dst), i32(lens), i32(pages), d_tab, d_counts)
    assert st.poll_error() == B.OPW_ERR_BAD_PAGE and st.launch_count() - before == (layers + 63) // 64
    draft.fork(pools, Hkv, D, src[:2], dst[:2], lens[:2], pages[:2], tab, counts)
    assert (d_tab.cpu().numpy() == tab).all() and (d_counts.cpu().numpy() == counts).all()
    for p, d in zip(pools, d_pools):
        assert (host_bits(d) == p).all()


# ------------------------------------------------------------------------------ a whole step ---

def test_a_captured_step_equals_the_oracle_and_records_exactly_what_it_should():
    """Fork, rotary append, tree attention, commit, release and the free list in one graph, replayed with other lengths: the status is
    known for each, and where every row has its page the results are the oracle's."""
    rng = np.random.default_rng(2900)
    Hq, Hkv, D, T, width, total, rot = 32, 8, 128, 6, 6, 40, 64
    i32 = lambda a: dev(np.asarray(a, np.int32))  # noqa: E731
    pool0 = rand_bits(rng, oracle.pool_elems(total, Hkv, P, D))
    tab0, refs0 = np.full((4, width), -1, np.int32), np.zeros(total, np.int32)
    tab0[:2] = rng.permutation(total)[:12].reshape(2, 6)
    refs0[tab0[:2].ravel()] = 1
    spare = np.nonzero(refs0 == 0)[0][[3, 8]].astype(np.int32)
    parents = random_tree(rng, T)
    words, depth = B.opw_tree_mask(parents)
    mask, seq = np.array([words] * 4, np.uint64), np.repeat(np.arange(4), T)
    q0, k0, v0 = rand_bits(rng, (4 * T, Hq, D)), rand_bits(rng, (4 * T, Hkv, D)), rand_bits(rng, (4 * T, Hkv, D))
    size, acc, took = [T, 3, 2, T], [[1, 4, 5, 0, 0, 0], [2, 0, 0, 0, 0, 0], [0, 1, 0, 0, 0, 0], [0, 2, 5, 0, 0, 0]], [3, 1, 2, 3]
    pool, tab, refs = dev(pool0, True), dev(tab0), dev(refs0)
    st = make_stage([pool], Hq, Hkv, D, 4, width)
    tree, rope = B.TreeAttention(st, T), B.Rope(rot)
    q, k, v, d_mask, d_seq, dep = dev(q0, True), dev(k0, True), dev(v0, True), dev(mask), i32(seq), i32([depth] * 4)
    ctx, lens, new = i32([41, 61, 0, 0]), i32([0, 0]), i32([0] * 4)
    pos, slots, qr = i32([0] * 4 * T), i32([0] * 4 * T), torch.empty_like(q)
    out, lse = torch.empty(4, T, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(4, T, Hq, device="cuda")
    lst, cnt, ar = i32([-7] * total), i32([0]), torch.arange(T, dtype=torch.int32, device="cuda")
    ids = [i32(x) for x in ([0, 1], [2, 3], [0], size, acc, took)]
    d_spare = dev(spare)

    def step():
        st.kv_fork([0], ids[0], ids[1], lens, d_spare, tab, refs)
        ctx[2:].copy_(lens)
        pos.copy_((ctx[:, None] + dep).view(-1))
        slots.copy_((ctx[:, None] + ar).view(-1))
        st.rope_append(0, rope, q, k, v, d_seq, slots, pos, tab, qr)
        tree.attention(0, qr.view(4, T, Hq, D), d_mask, pos.view(4, T), ctx, ids[3], tab, out, lse)
        st.kv_commit([0], ids[4], ids[5], ctx, tab, new)
        st.kv_release(ids[2], None, tab, refs)
        st.kv_free_pages(refs, lst, cnt)

    def reset(change):
        pool.copy_(dev(pool0, True)), tab.copy_(dev(tab0)), refs.copy_(dev(refs0)), lst.fill_(-7), out.fill_(0), lse.fill_(0)
        lens.copy_(i32(list(change)))

    reset((21, 37)), step()
    assert st.poll_error() == B.OPW_OK
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    freq = draft.frequencies(rot)
    # whole pages are shared and the drafted rows need room behind the copied rest: 21, 37 and 26 leave it, 16 and 0 have no page of
    # their own, 28 runs over its end
    for change, status in (((21, 37), B.OPW_OK), ((16, 33), B.OPW_ERR_BAD_PAGE), ((26, 34), B.OPW_OK), ((0, 41), B.OPW_ERR_BAD_PAGE),
                           ((21, 28), B.OPW_ERR_BAD_PAGE), ((5, 26), B.OPW_OK)):
        reset(change), g.replay()
        assert st.poll_error() == status, change
        if status != B.OPW_OK:
            continue
        w_pool, w_tab, w_refs = pool0.copy(), tab0.copy(), refs0.copy()
        draft.fork([w_pool], Hkv, D, [0, 1], [2, 3], change, spare, w_tab, w_refs)
        at = np.array([41, 61, *change])
        w_pos, w_slots = (at[:, None] + np.array(depth)).ravel(), (at[:, None] + np.arange(T)).ravel()
        # what was rotated, to its rounding (half a step of bf16, and fp32 products of a pair): the bits of keys come from a cache of
        # their own, so that what follows can be exact
        own_pool, own_tab = torch.zeros(4 * T * 2 * Hkv * 16 * D, dtype=torch.bfloat16, device="cuda"), i32([[i] for i in range(4 * T)])
        own = make_stage([own_pool], Hq, Hkv, D, 4 * T, 1)
        q_own = torch.empty_like(q)
        own.rope_append(0, rope, q, k, v, i32(range(4 * T)), i32([0] * 4 * T), i32(w_pos), own_tab, q_own)
        k_bits = np.concatenate([oracle.gather_logical(host_bits(own_pool), Hkv, P, D, np.array([i]), 0, 1)[0] for i in range(4 * T)])
        for bits, x0 in ((k_bits, k0), (host_bits(q_own), q0)):
            x = oracle.bf16_bits_to_f64(x0)
            want = draft.rotate(x, w_pos, freq, "half")
            near = 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * np.abs(x).max()
            assert (np.abs(oracle.bf16_bits_to_f64(bits) - want) <= near).all()
        assert torch.equal(q_own, qr)
        draft.append_rows(w_pool, Hkv, D, seq, w_slots, w_tab, k_bits, v0)
        ref = draft.tree_attention(w_pool, Hq, Hkv, D, host_bits(qr).reshape(4, T, Hq, D), mask, w_pos.reshape(4, T), at, size, w_tab)
        check_tree(out, lse, ref, 128)
        w_new = draft.commit(w_pool, Hkv, D, np.array(acc), np.array(took), at, w_tab, T)
        draft.release([0], None, w_tab, w_refs)
        free = np.nonzero(w_refs == 0)[0]
        assert (host_bits(pool) == w_pool).all() and (new.cpu().numpy() == w_new).all()
        assert (tab.cpu().numpy() == w_tab).all() and (refs.cpu().numpy() == w_refs).all()
        assert cnt.item() == len(free) and (lst[:len(free)].cpu().numpy() == free).all() and (lst[len(free):] == -7).all()


@pytest.mark.parametrize("Hq,Hkv,D,T", [(32, 8, 128, 5), (8, 2, 64, 40), (16, 2, 256, 3)])
def test_contexts_at_the_end_of_32_bits(Hq, Hkv, D, T):
    """A window at the far end of the longest table that is taken equals, bit for bit, the same window near the start; a table whose
    last key tile could pass 32 bits is refused."""
    rng = np.random.default_rng(2400 + D)
    window, width, far = 100, 30, (1 << 27) - 9
    cap = far * 16
    assert cap <= (1 << 31) - 1 - 128 < (far + 1) * 16
    near = width * 16 - 3 - T                                    # drafted rows end three slots before the table does
    pool, tab, q, mask, pos = tree_inputs(rng, [near], [T], T, Hq, Hkv, D)
    d_pool, i32 = dev(pool, True), lambda a: dev(np.asarray(a, np.int32))  # noqa: E731
    junk = rand_bits(rng, (3, Hkv, D))
    junk[:] = 0x7FC0
    draft.append_rows(pool, Hkv, D, [0] * 3, [width * 16 - 3 + i for i in range(3)], tab, junk, junk)
    d_pool.copy_(dev(pool, True))
    res = []
    for pages in (width, far):
        shift = (pages - width) * 16
        st = make_stage([d_pool], Hq, Hkv, D, 1, pages, window)
        tree = B.TreeAttention(st, T)
        table = torch.full((1, pages), -1, dtype=torch.int32, device="cuda")
        table[0, pages - width:] = i32(tab[0])
        out, lse = torch.empty(1, T, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(1, T, Hq, device="cuda")
        tree.attention(0, dev(q, True), dev(mask), i32(pos.astype(np.int64) + shift), i32([near + shift]), i32([T]), table, out, lse)
        assert st.poll_error() == B.OPW_OK
        res.append((out, lse))
        tree.close(), st.close()
        del table
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])
    ref = draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, [near], [T], tab, window)
    check_tree(*res[1], ref, 200)
    st = make_stage([d_pool], Hq, Hkv, D, 1, far + 1, window)
    assert B.opw_tree_attn_workspace_bytes(st.handle, T) == 0
    h = B.ctypes.c_void_p()
    ws = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    assert B.lib().opw_tree_attn_create(st.handle, T, 0, ws.data_ptr(), 1 << 28, B.ctypes.byref(h)) == B.OPW_ERR_UNSUPPORTED and h.value is None
