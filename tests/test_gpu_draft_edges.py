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
