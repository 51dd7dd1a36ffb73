"""GPU parity of the drafted-token operators (rotary append, tree attention, commit) and of the page operators (fork,
release, free list) against the 64-bit oracle, their refusals, and a whole draft-verify-commit run."""
import ctypes
import math

import numpy as np
import pytest
import torch

import oracle
from helpers import P, make_case, out_to_f64, rand_bits
from oracle import draft
from paper_2609_14237_b200 import binding as B

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 64), (32, 8, 128), (64, 8, 128), (5, 1, 64), (16, 1, 128), (4, 4, 64), (16, 2, 256), (6, 2, 256)]


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()
    assert torch.cuda.is_available()


def dev(a, bf16=False):
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint64:
        a = a.view(np.int64)
    t = torch.from_numpy(a)
    return (t.view(torch.int16).view(torch.bfloat16) if bf16 else t).cuda()


def host_bits(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


def make_stage(pools, Hq, Hkv, D, rows, width, window=0, **kw):
    return B.Stage(pools=pools, layer_window=[window] * len(pools), num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, max_batch=rows,
                   max_pages_per_seq=width, **kw)


def random_tree(rng, n):
    return [int(rng.integers(-1, i)) if i else -1 for i in range(n)]


def tree_inputs(rng, ctx, size, T, Hq, Hkv, D, general=False, spare_pages=0):
    """Cache, queries, masks and positions; row b's drafted rows are cached behind its context."""
    n = [max(c, 0) + max(t, 0) for c, t in zip(ctx, size)]
    pool, tab, _, _, _ = make_case(rng, [max(x, 1) for x in n], Hq, Hkv, D)
    if spare_pages:
        tab = np.concatenate([tab, np.full((len(ctx), spare_pages), -1, np.int32)], 1)
    B_ = len(ctx)
    mask, pos = np.zeros((B_, T), np.uint64), np.zeros((B_, T), np.int32)
    for b in range(B_):
        t = max(0, min(size[b], T))
        if general:       # any words: rows that see nothing, rows without their own bit, bits behind the tree
            mask[b] = rng.integers(0, 1 << 63, size=T, dtype=np.uint64) * np.uint64(2) + rng.integers(0, 2, size=T).astype(np.uint64)
            mask[b, ::3] = 0
            pos[b] = max(ctx[b], 0) + rng.integers(-3, 20, size=T)
        elif t:
            m, d = B.opw_tree_mask(random_tree(rng, t))
            mask[b, :t], pos[b, :t] = m, max(ctx[b], 0) + np.array(d)
    q = rand_bits(rng, (B_, T, Hq, D))
    return pool, tab.astype(np.int32), q, mask, pos


def gpu_tree(pool, tab, q, mask, pos, ctx, size, Hq, Hkv, D, window=0, scale=0.0):
    st = make_stage([dev(pool, True)], Hq, Hkv, D, len(ctx), tab.shape[1], window, softmax_scale=scale)
    tree = B.TreeAttention(st, q.shape[1])
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:3], float("nan"), dtype=torch.float32, device="cuda")
    tree.attention(0, dev(q, True), dev(mask), dev(pos), dev(np.asarray(ctx, np.int32)), dev(np.asarray(size, np.int32)), dev(tab), out, lse)
    rc = st.poll_error()
    tree.close()
    st.close()
    return out, lse, rc


def check_tree(out, lse, ref, n):
    """The tolerance counts roundings (half a step of bf16 is 2^-8 of the value, of fp32 2^-24):
    * each p_j is rounded to bf16 for the product with V: off by at most 2^-8 sum p|V| / sum p = 2^-8 spread;
    * the output is rounded to bf16 once: 2^-8 |out|, and 2^-16 of the cross term;
    * the scores are fp32 sums of D exact products, scaled: ds = (D + 4) 2^-24 bound, which moves each p_j by a factor
      e^(+-2 ds) against its neighbours; 2^x is good to 2^-21 relative; sums of n terms and their rescalings add n 2^-23."""
    want, want_lse, spread, bound = ref
    D = want.shape[-1]
    got, got_lse = out_to_f64(out), lse.cpu().numpy().astype(np.float64)
    ds = (D + 4) * 2.0 ** -24 * bound
    noise = (2 * ds + 2.0 ** -21 + n * 2.0 ** -23)[..., None] * spread
    tol = 2.0 ** -8 * (np.abs(want) + spread) + 2.0 ** -14 * spread + 2 * noise
    fine = np.isfinite(want)
    assert (np.isnan(got) == np.isnan(want)).all()
    assert (got[np.isinf(want)] == want[np.isinf(want)]).all()
    err = np.abs(got - np.where(fine, want, 0.0))[fine]
    assert (err <= tol[fine] + 1e-30).all(), (err.max(), (err / (tol[fine] + 1e-30)).max())
    seen = np.isfinite(want_lse)
    assert (np.isneginf(got_lse) == np.isneginf(want_lse)).all()
    lse_tol = ds + 2.0 ** -21 + n * 2.0 ** -23 + 2.0 ** -22 * np.abs(np.where(seen, want_lse, 0.0))
    assert (np.abs(got_lse[seen] - want_lse[seen]) <= lse_tol[seen]).all()


# ---------------------------------------------------------------------------- tree attention ---

@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("T", [1, 3, 13, 64])
@pytest.mark.parametrize("window", [0, 37])
def test_tree_attention_matches_the_oracle(Hq, Hkv, D, T, window):
    rng = np.random.default_rng(1000 + Hq + D + T + window)
    ctx = [0, 1, 15, 16, 130, 700, -1, 33]
    size = [T, max(1, T // 2), T, 1, T, T, T, 0]
    pool, tab, q, mask, pos = tree_inputs(rng, ctx, size, T, Hq, Hkv, D)
    ref = draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, ctx, size, tab, window)
    out, lse, rc = gpu_tree(pool, tab, q, mask, pos, ctx, size, Hq, Hkv, D, window)
    assert rc == B.OPW_OK
    check_tree(out, lse, ref, 800)
    got = out_to_f64(out)
    assert (got[6:] == 0).all() and (got[1, size[1]:] == 0).all()


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (32, 8, 128), (6, 2, 256)])
@pytest.mark.parametrize("window", [0, 1, 9])
def test_any_mask_words_and_rows_that_see_nothing(Hq, Hkv, D, window):
    rng = np.random.default_rng(1100 + D + window)
    T = 29
    ctx, size = [0, 0, 5, 40, 200], [T, 3, T, T, 17]
    pool, tab, q, mask, pos = tree_inputs(rng, ctx, size, T, Hq, Hkv, D, general=True)
    ref = draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, ctx, size, tab, window)
    assert np.isneginf(ref[1][0]).any()
    out, lse, rc = gpu_tree(pool, tab, q, mask, pos, ctx, size, Hq, Hkv, D, window)
    assert rc == B.OPW_OK
    check_tree(out, lse, ref, 300)


@pytest.mark.parametrize("Hq,Hkv,D,T", [(8, 2, 64, 5), (32, 8, 128, 4), (32, 8, 128, 64), (8, 2, 64, 64), (6, 2, 256, 9)])
@pytest.mark.parametrize("window", [0, 20])
def test_what_a_node_does_not_see_may_hold_anything(Hq, Hkv, D, T, window):
    """NaN and infinities in slots behind the end, before the window, and in the keys and values of nodes that others
    do not see: only the rows that see them are touched, and those as the definition says."""
    rng = np.random.default_rng(1200 + D + T)
    ctx, size = [37, 21, 150], [T, T, max(1, T - 2)]
    pool, tab, q, mask, pos = tree_inputs(rng, ctx, size, T, Hq, Hkv, D)
    clean = draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, ctx, size, tab, window)
    junk = np.array([0x7FC0, 0x7F80, 0xFF80, 0xFFFF], np.uint16)          # NaN, +inf, -inf, NaN
    row = lambda: (junk[rng.integers(0, 4, size=(Hkv, D))], junk[rng.integers(0, 4, size=(Hkv, D))])  # noqa: E731
    for b in range(3):
        n = ctx[b] + size[b]
        for s in range(n, tab[b][tab[b] >= 0].size * P):
            draft._put_row(pool, Hkv, D, tab[b, s // P], s % P, *row())
        if window:
            for s in range(0, max(0, ctx[b] + 1 - window)):
                draft._put_row(pool, Hkv, D, tab[b, s // P], s % P, *row())
    same = draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, ctx, size, tab, window)
    assert (same[0] == clean[0]).all()
    out, lse, rc = gpu_tree(pool, tab, q, mask, pos, ctx, size, Hq, Hkv, D, window)
    assert rc == B.OPW_OK
    check_tree(out, lse, clean, 300)
    # now a value that some nodes see: one infinity in one dimension of one head, of the last drafted node
    for b in range(3):
        s = ctx[b] + size[b] - 1
        k, v = oracle.gather_logical(pool, Hkv, P, D, tab[b], s, s + 1)
        v[0, 0, 3], v[0, Hkv - 1, D - 1] = 0x7F80, 0x7FC0
        draft._put_row(pool, Hkv, D, tab[b, s // P], s % P, k[0], v[0])
    ref = draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, ctx, size, tab, window)
    assert np.isinf(ref[0]).any() and np.isnan(ref[0]).any()
    out, lse, rc = gpu_tree(pool, tab, q, mask, pos, ctx, size, Hq, Hkv, D, window)
    assert rc == B.OPW_OK
    check_tree(out, lse, ref, 300)
    # and a key: its score is NaN or infinite for the nodes that see it, their whole row with it
    for b in range(3):
        s = ctx[b] + size[b] - 1
        draft._put_row(pool, Hkv, D, tab[b, s // P], s % P, np.full((Hkv, D), 0x7FC0, np.uint16), rand_bits(rng, (Hkv, D)))
    out, lse, rc = gpu_tree(pool, tab, q, mask, pos, ctx, size, Hq, Hkv, D, window)
    got, got_lse = out_to_f64(out), lse.cpu().numpy()
    for b in range(3):
        t = size[b]
        hit = np.array([(int(mask[b, i]) >> (t - 1)) & 1 for i in range(t)], bool)
        assert np.isnan(got[b, :t][hit]).all() and np.isnan(got_lse[b, :t][hit]).all()
        assert np.isfinite(got[b, :t][~hit]).all()


@pytest.mark.parametrize("Hq,Hkv,D,T", [(32, 8, 128, 7), (32, 8, 128, 40), (8, 2, 64, 33), (16, 2, 256, 5)])
def test_long_context_splits_over_workers(Hq, Hkv, D, T):
    """One long sequence beside short ones: its rows are merged from many partials.  Checked at a few heads' worth of rows
    by a plain 64-bit computation on the device."""
    g = torch.Generator(device="cuda")
    g.manual_seed(77)
    ctx, size = [20011, 5, 300], [T, T, T]
    pages = [(c + t + 15) // 16 for c, t in zip(ctx, size)]
    total = sum(pages)
    perm = torch.randperm(total, generator=g, device="cuda").int()
    tab = torch.full((3, max(pages)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        tab[b, :n] = perm[at:at + n]
        at += n
    pool = torch.randn(total * Hkv * 2 * 16 * D, generator=g, device="cuda", dtype=torch.bfloat16)
    q = torch.randn(3, T, Hq, D, generator=g, device="cuda", dtype=torch.bfloat16)
    m, d = B.opw_tree_mask(random_tree(np.random.default_rng(3), T))
    mask = dev(np.array([m] * 3, np.uint64))
    pos = torch.tensor(ctx, device="cuda", dtype=torch.int32)[:, None] + torch.tensor(d, device="cuda", dtype=torch.int32)
    st = make_stage([pool], Hq, Hkv, D, 3, max(pages))
    tree = B.TreeAttention(st, 64)
    c, s = (torch.tensor(x, device="cuda", dtype=torch.int32) for x in (ctx, size))
    outs = []
    for _ in range(2):
        out, lse = torch.empty_like(q), torch.empty(3, T, Hq, device="cuda")
        tree.attention(0, q, mask, pos, c, s, tab, out, lse)
        outs.append((out, lse))
    assert st.poll_error() == B.OPW_OK
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])      # deterministic
    idx = torch.arange(16 * D, device="cuda").view(16, D // 8, 8)
    order = torch.stack([idx[t][torch.arange(D // 8, device="cuda") ^ (t & 7)].reshape(-1) for t in range(16)]).reshape(-1)
    for b in range(3):
        n = ctx[b] + size[b]
        kv = pool.view(total, Hkv, 2, 16 * D)[tab[b, :pages[b]].long()][..., order].view(pages[b], Hkv, 2, 16, D)
        kv = kv.permute(2, 1, 0, 3, 4).reshape(2, Hkv, pages[b] * 16, D)[:, :, :n].double()
        hide = torch.zeros(T, n, dtype=torch.bool, device="cuda")
        for i in range(T):
            for j in range(T):
                hide[i, ctx[b] + j] = not (m[i] >> j) & 1
        x = torch.einsum("thgd,hkd->hgtk", q[b].double().view(T, Hkv, -1, D), kv[0]) / math.sqrt(D)
        x = x.masked_fill(hide, -math.inf)
        p = torch.softmax(x, -1)
        want = torch.einsum("hgtk,hkd->thgd", p, kv[1]).reshape(T, Hq, D)
        spread = torch.einsum("hgtk,hkd->thgd", p, kv[1].abs()).reshape(T, Hq, D)
        big = (torch.einsum("thgd,hkd->hgtk", q[b].double().abs().view(T, Hkv, -1, D), kv[0].abs()).amax(-1) / math.sqrt(D))
        bound = big.permute(2, 0, 1).reshape(T, Hq)
        want_lse = torch.logsumexp(x, -1).permute(2, 0, 1).reshape(T, Hq)
        ref = [a.cpu().numpy() for a in (want, want_lse, spread, bound)]
        check_tree(outs[0][0][b], outs[0][1][b], ref, n)
    # the split follows from the lengths alone: other physical pages, same bits
    moved = torch.randperm(total, generator=g, device="cuda")
    pool2 = torch.empty_like(pool)
    pool2.view(total, -1)[moved] = pool.view(total, -1)
    tab2 = torch.where(tab >= 0, moved[tab.clamp(min=0).long()].int(), tab)
    st2 = make_stage([pool2], Hq, Hkv, D, 3, max(pages))
    tree2 = B.TreeAttention(st2, T)
    out2 = torch.empty_like(q)
    tree2.attention(0, q, mask, pos, c, s, tab2, out2)
    assert torch.equal(out2, outs[0][0])


@pytest.mark.parametrize("window", [0, 700, 4096])
@pytest.mark.parametrize("Hq,Hkv,D,T", [(32, 8, 128, 26), (64, 8, 128, 33), (8, 2, 64, 40), (32, 8, 128, 6), (16, 2, 256, 11)])
def test_many_ragged_sequences_each_of_many_tiles(Hq, Hkv, D, T, window):
    """Workers whose shares span several sequences of many key tiles, with masked tiles at both ends (window and tree)."""
    rng = np.random.default_rng(1600 + D + T + window)
    g = torch.Generator(device="cuda")
    g.manual_seed(78)
    n = 24
    ctx = rng.integers(500, 9000, size=n)
    size = rng.integers(T // 2, T + 1, size=n)
    first = np.maximum(0, ctx + 1 - window) // 16 if window else np.zeros(n, np.int64)
    pages = (ctx + size + 15) // 16
    total = int((pages - first).sum())
    perm = rng.permutation(total).astype(np.int32)
    tab, at = np.full((n, int(pages.max())), -1, np.int32), 0
    mask, pos = np.zeros((n, T), np.uint64), np.zeros((n, T), np.int32)
    for b in range(n):
        c = int(pages[b] - first[b])
        tab[b, first[b]:pages[b]] = perm[at:at + c]
        at += c
        m, d = B.opw_tree_mask(random_tree(rng, int(size[b])))
        mask[b, :size[b]], pos[b, :size[b]] = m, ctx[b] + np.array(d)
    pool = torch.randn(total * Hkv * 2 * 16 * D, generator=g, device="cuda", dtype=torch.bfloat16)
    q = torch.randn(n, T, Hq, D, generator=g, device="cuda", dtype=torch.bfloat16)
    st = make_stage([pool], Hq, Hkv, D, n, tab.shape[1], window)
    tree = B.TreeAttention(st, T)
    out, lse = torch.empty_like(q), torch.empty(n, T, Hq, device="cuda")
    args = (q, dev(mask), dev(pos), dev(ctx.astype(np.int32)), dev(size.astype(np.int32)), dev(tab))
    tree.attention(0, *args, out, lse)
    assert st.poll_error() == B.OPW_OK
    idx = torch.arange(16 * D, device="cuda").view(16, D // 8, 8)
    order = torch.stack([idx[t][torch.arange(D // 8, device="cuda") ^ (t & 7)].reshape(-1) for t in range(16)]).reshape(-1)
    for b in range(n):
        c, t, lo = int(ctx[b]), int(size[b]), int(first[b]) * 16
        ids = dev(tab[b, first[b]:pages[b]]).long()
        kv = pool.view(total, Hkv, 2, 16 * D)[ids][..., order].view(len(ids), Hkv, 2, 16, D)
        kv = kv.permute(2, 1, 0, 3, 4).reshape(2, Hkv, len(ids) * 16, D)[:, :, :c + t - lo].double()
        where = np.concatenate([np.arange(lo, c), pos[b, :t]])
        see = np.ones((t, c + t - lo), bool)
        for i in range(t):
            see[i, c - lo:] = [(int(mask[b, i]) >> j) & 1 for j in range(t)]
            if window:
                see[i] &= where > pos[b, i] - window
        x = torch.einsum("thgd,hkd->hgtk", q[b, :t].double().view(t, Hkv, -1, D), kv[0]) / math.sqrt(D)
        x = x.masked_fill(~dev(see), -math.inf)
        p = torch.softmax(x, -1)
        want = torch.einsum("hgtk,hkd->thgd", p, kv[1]).reshape(t, Hq, D)
        spread = torch.einsum("hgtk,hkd->thgd", p, kv[1].abs()).reshape(t, Hq, D)
        big = torch.einsum("thgd,hkd->hgtk", q[b, :t].double().abs().view(t, Hkv, -1, D), kv[0].abs()).amax(-1) / math.sqrt(D)
        ref = [a.cpu().numpy() for a in (want, torch.logsumexp(x, -1).permute(2, 0, 1).reshape(t, Hq), spread,
                                         big.permute(2, 0, 1).reshape(t, Hq))]
        check_tree(out[b, :t], lse[b, :t], ref, c + t)
        assert (out[b, t:] == 0).all() and torch.isneginf(lse[b, t:]).all()


def test_a_chain_of_one_is_a_decode_step():
    rng = np.random.default_rng(1300)
    Hq, Hkv, D, lens = 32, 8, 128, [0, 15, 16, 100, 999]
    pool, tab, q, mask, pos = tree_inputs(rng, lens, [1] * 5, 1, Hq, Hkv, D)
    out, lse, rc = gpu_tree(pool, tab, q, mask, pos, lens, [1] * 5, Hq, Hkv, D)
    st = make_stage([dev(pool, True)], Hq, Hkv, D, 5, tab.shape[1])
    o2, l2 = torch.empty(5, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(5, Hq, device="cuda")
    st.decode_attention(0, dev(q[:, 0], True), dev(np.array(lens, np.int32) + 1), dev(tab), o2, l2)
    assert st.poll_error() == B.OPW_OK
    ref = draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, lens, [1] * 5, tab)
    check_tree(o2[:, None], l2[:, None], ref, 1000)
    check_tree(out, lse, ref, 1000)


@pytest.mark.parametrize("T", [4, 64])
def test_bad_pages_and_lengths_beyond_the_table_are_masked_and_recorded(T):
    rng = np.random.default_rng(1400)
    Hq, Hkv, D = 32, 8, 128
    ctx, size = [100, 100, 100], [T, T, T]
    pool, tab, q, mask, pos = tree_inputs(rng, ctx, size, T, Hq, Hkv, D)
    good, _, rc = gpu_tree(pool, tab, q, mask, pos, ctx, size, Hq, Hkv, D)
    assert rc == B.OPW_OK
    bad = tab.copy()
    bad[1, 2] = 1 << 20
    out, lse, rc = gpu_tree(pool, bad, q, mask, pos, ctx, size, Hq, Hkv, D)
    assert rc == B.OPW_ERR_BAD_PAGE and torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])
    assert torch.isfinite(out).all()
    # page 2 hidden: the oracle on a context without those sixteen keys
    keep = [i for i in range(100) if i // 16 != 2]
    k, v = oracle.gather_logical(pool, Hkv, P, D, tab[1], 0, 100 + T)
    pool2, tab2 = pool.copy(), tab.copy()
    order = keep + list(range(100, 100 + T))
    draft.append_rows(pool2, Hkv, D, [1] * len(order), list(range(len(order))), tab2, k[order], v[order])
    ref = draft.tree_attention(pool2, Hq, Hkv, D, q[1:2], mask[1:2], pos[1:2], [84], [T], tab2[1:2])
    check_tree(out[1:2], lse[1:2], ref, 200)
    # lengths that do not fit
    out, lse, rc = gpu_tree(pool, tab, q, mask, pos, [100, tab.shape[1] * 16 + 5, 100], [T, T, T + 1], Hq, Hkv, D)
    assert rc == B.OPW_ERR_BAD_PAGE and torch.equal(out[0], good[0]) and torch.equal(out[2], good[2]) and torch.isfinite(out).all()


def test_tree_attention_refuses():
    Hq, Hkv, D = 8, 2, 64
    pool = torch.zeros(4 * Hkv * 2 * 16 * D, dtype=torch.bfloat16, device="cuda")
    st = make_stage([pool], Hq, Hkv, D, 2, 4)
    L, h = B.lib(), ctypes.c_void_p()
    assert B.opw_tree_attn_workspace_bytes(st.handle, 0) == B.opw_tree_attn_workspace_bytes(st.handle, 65) == 0
    n = B.opw_tree_attn_workspace_bytes(st.handle, 8)
    ws = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    base = (ws.data_ptr() + 255) // 256 * 256
    for args, want in (((0, 0, base, n), B.OPW_ERR_INVALID_ARG), ((65, 0, base, n), B.OPW_ERR_INVALID_ARG), ((8, 1, base, n), B.OPW_ERR_INVALID_ARG),
                       ((8, 0, base + 8, n), B.OPW_ERR_INVALID_ARG), ((8, 0, None, n), B.OPW_ERR_INVALID_ARG), ((8, 0, base, n - 1), B.OPW_ERR_CAPACITY)):
        assert L.opw_tree_attn_create(st.handle, *args, ctypes.byref(h)) == want and h.value is None
    tree = B.TreeAttention(st, 8)
    q, out = (torch.zeros(2, 8, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mask, pos = torch.zeros(2, 8, dtype=torch.int64, device="cuda"), torch.zeros(2, 8, dtype=torch.int32, device="cuda")
    ctx, size = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    tab = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    good = dict(layer=0, batch=2, nodes=8, q=q.data_ptr(), mask=mask.data_ptr(), pos=pos.data_ptr(), ctx=ctx.data_ptr(), size=size.data_ptr(),
                tab=tab.data_ptr(), out=out.data_ptr(), lse=None)
    call = lambda **kw: L.opw_tree_attention(tree.handle, *{**good, **kw}.values(), None)  # noqa: E731
    before = st.launch_count()
    for name in ("q", "mask", "pos", "ctx", "size", "tab", "out"):
        assert call(**{name: None}) == B.OPW_ERR_INVALID_ARG
        assert call(**{name: good[name] + (8 if name in ("q", "out") else 4 if name == "mask" else 2)}) == B.OPW_ERR_INVALID_ARG
    for kw, want in ((dict(layer=1), B.OPW_ERR_INVALID_ARG), (dict(layer=-1), B.OPW_ERR_INVALID_ARG), (dict(batch=-1), B.OPW_ERR_INVALID_ARG),
                     (dict(batch=3), B.OPW_ERR_CAPACITY), (dict(nodes=0), B.OPW_ERR_INVALID_ARG), (dict(nodes=9), B.OPW_ERR_CAPACITY),
                     (dict(out=good["q"]), B.OPW_ERR_INVALID_ARG), (dict(out=good["q"] + 64), B.OPW_ERR_INVALID_ARG), (dict(lse=good["ctx"] + 2), B.OPW_ERR_INVALID_ARG)):
        assert call(**kw) == want
    assert call(batch=0) == B.OPW_OK and st.launch_count() == before
    with pytest.raises(ValueError):
        tree.attention(0, q.float(), mask, pos, ctx, size, tab, out)
    with pytest.raises(ValueError):
        tree.attention(0, q, mask, pos.long(), ctx, size, tab, out)
    with pytest.raises(ValueError):
        tree.attention(0, q, mask, pos, ctx, size, tab[:, :3], out)
    with pytest.raises(ValueError):
        tree.attention(0, q, mask[:, :7], pos, ctx, size, tab, out)
    assert call() == B.OPW_OK and st.launch_count() == before + 2 and (out == 0).all()


def test_a_batch_beyond_the_tensor_core_kernels_reach():
    """More than 2048 sequences: the rows of wide trees go through the kernel of few rows, sixteen at a time."""
    rng = np.random.default_rng(1450)
    Hq, Hkv, D, T, n = 8, 1, 64, 5, 2100
    ctx = rng.integers(0, 40, size=n).tolist()
    size = rng.integers(0, T + 1, size=n).tolist()
    pool, tab, q, mask, pos = tree_inputs(rng, ctx, size, T, Hq, Hkv, D)
    out, lse, rc = gpu_tree(pool, tab, q, mask, pos, ctx, size, Hq, Hkv, D)
    assert rc == B.OPW_OK
    pick = list(range(0, n, 50)) + [n - 1]
    ref = draft.tree_attention(pool, Hq, Hkv, D, q[pick], mask[pick], pos[pick], [ctx[i] for i in pick], [size[i] for i in pick], tab[pick])
    check_tree(out[dev(np.array(pick))], lse[dev(np.array(pick))], ref, 60)
    # the same rows in a batch that the tensor cores take
    few, few_lse, rc = gpu_tree(pool, tab[:300], q[:300], mask[:300], pos[:300], ctx[:300], size[:300], Hq, Hkv, D)
    a, b = few.float(), out[:300].float()
    assert rc == B.OPW_OK and (a - b).abs().max() <= 4 * 2.0 ** -8 * b.abs().max()      # two roundings on either side


@pytest.mark.parametrize("T", [3, 20, 50])
def test_handles_of_their_own_run_side_by_side(T):
    """Two handles of one stage on two streams, launched without programmatic serialisation, against one after the other."""
    rng = np.random.default_rng(1460 + T)
    Hq, Hkv, D = 32, 8, 128
    ctx, size = [900, 37, 400], [T, max(1, T - 1), T]
    pool, tab, q, mask, pos = tree_inputs(rng, ctx, size, T, Hq, Hkv, D)
    ref = draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, ctx, size, tab)
    st = make_stage([dev(pool, True)], Hq, Hkv, D, 3, tab.shape[1], flags=B.OPW_FLAG_NO_PDL)
    args = (dev(q, True), dev(mask), dev(pos), dev(np.array(ctx, np.int32)), dev(np.array(size, np.int32)), dev(tab))
    jobs = [(B.TreeAttention(st, T), torch.cuda.Stream(), torch.empty_like(args[0]), torch.empty(3, T, Hq, device="cuda")) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for tree, stream, out, lse in jobs:
            with torch.cuda.stream(stream):
                tree.attention(0, *args, out, lse)
    torch.cuda.synchronize()
    for _, _, out, lse in jobs:
        check_tree(out, lse, ref, 1000)
    assert torch.equal(jobs[0][2], jobs[1][2]) and st.poll_error() == B.OPW_OK


def test_tree_attention_in_a_graph_on_another_stream_with_lengths_changed_between_replays():
    rng = np.random.default_rng(1500)
    Hq, Hkv, D, T = 32, 8, 128, 12
    ctx, size = [200, 90], [T, T]
    pool, tab, q, mask, pos = tree_inputs(rng, ctx, size, T, Hq, Hkv, D)
    st = make_stage([dev(pool, True)], Hq, Hkv, D, 2, tab.shape[1])
    tree = B.TreeAttention(st, T)
    d = dict(q=dev(q, True), mask=dev(mask), pos=dev(pos), tab=dev(tab))
    c, s = dev(np.array(ctx, np.int32)), dev(np.array(size, np.int32))
    out, lse = torch.empty_like(d["q"]), torch.empty(2, T, Hq, device="cuda")
    call = lambda: tree.attention(0, d["q"], d["mask"], d["pos"], c, s, d["tab"], out, lse)  # noqa: E731
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for cc, ss in (([200, 90], [T, T]), ([7, 90], [3, T]), ([-1, 33], [T, 1])):
        c.copy_(torch.tensor(cc, dtype=torch.int32))
        s.copy_(torch.tensor(ss, dtype=torch.int32))
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        ref = draft.tree_attention(pool, Hq, Hkv, D, q, mask, pos, cc, ss, tab)
        check_tree(out, lse, ref, 300)
    assert st.poll_error() == B.OPW_OK


@pytest.mark.parametrize("T", [2, 9, 64])
def test_the_longest_windows_hide_nothing(T):
    """Window arithmetic at the ends of 32 bits; positions far below and above the context."""
    rng = np.random.default_rng(1510 + T)
    Hq, Hkv, D = 32, 8, 128
    ctx, size = [2300, 0, 77], [T, T, max(1, T - 1)]
    pool, tab, q, mask, pos = tree_inputs(rng, ctx, size, T, Hq, Hkv, D)
    pos[2, ::2] = -(1 << 31)
    want = gpu_tree(pool, tab, q, mask, pos, ctx, size, Hq, Hkv, D)
    for window in (2400, (1 << 31) - 1):
        got = gpu_tree(pool, tab, q, mask, pos, ctx, size, Hq, Hkv, D, window)
        assert got[2] == B.OPW_OK and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_closed_stage_is_refused():
    st = make_stage([torch.zeros(2 * 2 * 16 * 64, dtype=torch.bfloat16, device="cuda")], 1, 1, 64, 1, 2)
    tree = B.TreeAttention(st, 1)
    q = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16, device="cuda")
    one = torch.ones(1, 1, dtype=torch.int32, device="cuda")
    st.close()
    with pytest.raises(ValueError):
        tree.attention(0, q, one.long(), one, one[0], one[0], one.repeat(1, 2), torch.empty_like(q))
    tree.close()


# --------------------------------------------------------------------------------- rotary ---

@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (32, 8, 128), (5, 1, 64), (6, 2, 256)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("part", ["full", "half", "odd", "two"])
@pytest.mark.parametrize("packed", [False, True])
def test_rope_append_matches_the_oracle(Hq, Hkv, D, layout, part, packed):
    rng = np.random.default_rng(2000 + D + Hq)
    rot = {"full": D, "half": D // 2, "odd": D // 4 + 2, "two": 2}[part]
    rows = 23
    tab = rng.permutation(8).astype(np.int32).reshape(4, 2)
    seq = np.array([0] * 7 + [-1] + [3] * 9 + [1] * 5 + [2], np.int32)
    slots = np.concatenate([np.arange(12, 19), [0], np.arange(9), np.arange(27, 32), [16]]).astype(np.int32)
    pos = rng.integers(0, 1 << 20, size=rows).astype(np.int32)
    pos[:3] = [0, 2 ** 31 - 1, 131071]
    qkv = rand_bits(rng, (rows, Hq + 2 * Hkv, D))
    pool = rand_bits(rng, oracle.pool_elems(8, Hkv, P, D))
    kw = dict(theta=10000.0, scaling="yarn", factor=8.0, original_context=8192.0)
    rope = B.Rope(rot, layout=layout, **kw)
    d_pool = dev(pool, True)
    st = make_stage([d_pool], Hq, Hkv, D, 4, 2)
    x = dev(qkv, True)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    q_out = torch.full((rows, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    args = (dev(seq), dev(slots), dev(pos), dev(tab))
    st.rope_append(0, rope, q, k, v, *args, q_out)
    assert st.poll_error() == B.OPW_OK and st.launch_count() == 1
    f, amp = draft.frequencies(rot, 10000.0, "yarn", 8.0, 8192.0), 1 + 0.1 * math.log(8.0)
    xf = oracle.bf16_bits_to_f64(qkv)
    turned = draft.rotate(xf[:, :Hq + Hkv], pos.astype(np.float64), f, layout, amp)

    def close(got, want, x):
        """bf16 half step of the value, fp32 cos/sin (2^-22) and three fp32 operations on |a| + |b| <= 2 max|x|, times the
        amplitude; the 64-bit angle itself is good to 2^31 * 2^-52 radians."""
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -20 + 2.0 ** -20) * 2 * amp * np.abs(x).max()
        assert (np.abs(got - want) <= tol).all(), np.abs(got - want).max()

    live = seq >= 0
    got_q = out_to_f64(q_out)
    close(got_q[live], turned[live, :Hq], xf)
    assert (got_q[live][..., rot:] == xf[live, :Hq, rot:]).all() and (got_q[~live] == 7.0).all()
    want_pool = pool.copy()
    got_pool = host_bits(d_pool)
    draft.append_rows(want_pool, Hkv, D, seq, slots, tab, qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:])
    gk = np.zeros((rows, Hkv, D))
    for r in np.nonzero(live)[0]:
        a, b = oracle.gather_logical(got_pool, Hkv, P, D, tab[seq[r]], slots[r], slots[r] + 1)
        gk[r] = oracle.bf16_bits_to_f64(a[0])
        assert (b[0] == qkv[r, Hq + Hkv:]).all()
        draft._put_row(want_pool, Hkv, D, tab[seq[r], slots[r] // P], slots[r] % P, a[0], b[0])
    close(gk[live], turned[live, Hq:], xf)
    assert (got_pool == want_pool).all()                       # nothing else in the cache moved
    # in place, and without queries
    if not packed:
        d2 = dev(pool, True)
        st2 = make_stage([d2], Hq, Hkv, D, 4, 2)
        q2 = q.clone()
        st2.rope_append(0, rope, q2, k, v, *args, q2)
        assert torch.equal(q2[dev(live)], q_out[dev(live)]) and torch.equal(q2[dev(~live)], q[dev(~live)]) and torch.equal(d2, d_pool)
        d3 = dev(pool, True)
        st3 = make_stage([d3], Hq, Hkv, D, 4, 2)
        st3.rope_append(0, rope, None, k, v, *args, None)
        assert torch.equal(d3, d_pool) and st3.poll_error() == B.OPW_OK


@pytest.mark.parametrize("layout,rot", [("half", 64), ("interleaved", 64), ("half", 10)])
def test_rope_append_skips_and_records_what_it_cannot_place(layout, rot):
    rng = np.random.default_rng(2100)
    Hq, Hkv, D, rows = 8, 2, 64, 5
    tab = np.array([[0, 1], [2, -1], [3, 99]], np.int32)
    seq, slots = np.array([0, 1, 2, 0, 3], np.int32), np.array([0, 16, 20, 32, 0], np.int32)
    pool = rand_bits(rng, oracle.pool_elems(4, Hkv, P, D))
    q, k, v = (dev(rand_bits(rng, (rows, h, D)), True) for h in (Hq, Hkv, Hkv))
    d_pool = dev(pool, True)
    st = make_stage([d_pool], Hq, Hkv, D, 8, 2)               # (row 3 is beyond the table, not beyond the stage)
    out = torch.zeros_like(q)
    pos = torch.zeros(rows, dtype=torch.int32, device="cuda")
    st.rope_append(0, B.Rope(rot, layout=layout), q, k, v, dev(seq), dev(slots), pos, dev(tab), out)
    assert st.poll_error() == B.OPW_ERR_BAD_PAGE and torch.equal(out, q)          # position 0 turns by nothing
    want = pool.copy()
    draft.append_rows(want, Hkv, D, [0], [0], tab, host_bits(k)[:1].reshape(1, Hkv, D), host_bits(v)[:1].reshape(1, Hkv, D))
    assert (host_bits(d_pool) == want).all()


def test_rotated_queries_must_not_overlap_the_inputs():
    Hq, Hkv, D, rows = 4, 2, 64, 5
    st = make_stage([torch.zeros(4 * Hkv * 2 * 16 * D, dtype=torch.bfloat16, device="cuda")], Hq, Hkv, D, 2, 2)
    rope, i = B.Rope(D), torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    tab = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    packed = torch.zeros(4 * rows, Hq + 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    q, k, v = (packed[:rows, a:b] for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    flat = packed.view(-1)
    size = rows * Hq * D
    for at in (0, 8, D, (rows - 1) * (Hq + 2 * Hkv) * D, rows * (Hq + 2 * Hkv) * D - 8):
        with pytest.raises(B.OpwError):
            st.rope_append(0, rope, q, k, v, i, i, i, tab, flat[at:at + size])
    own = torch.zeros(rows, Hq, D, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.OpwError):                                 # in place, but the keys lie there too
        st.rope_append(0, rope, own, own[:, :Hkv], v, i, i, i, tab, own)
    assert st.launch_count() == 0
    st.rope_append(0, rope, own, k, v, i, i, i, tab, own)           # in place
    end = rows * (Hq + 2 * Hkv) * D
    st.rope_append(0, rope, q, k, v, i, i, i, tab, flat[end:end + size])
    assert st.launch_count() == 2 and st.poll_error() == B.OPW_OK


def test_rope_append_refuses():
    Hq, Hkv, D, rows = 8, 2, 64, 3
    pool = torch.zeros(4 * Hkv * 2 * 16 * D, dtype=torch.bfloat16, device="cuda")
    st = make_stage([pool], Hq, Hkv, D, 2, 2)
    rope = B.Rope(64)
    q, k, v = (torch.zeros(rows, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    i = torch.zeros(rows, dtype=torch.int32, device="cuda")
    tab, out = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.zeros_like(q)
    good = dict(layer=0, rows=rows, rot=64, layout=0, table=rope.table.data_ptr(), q=q.data_ptr(), qs=Hq * D, k=k.data_ptr(), ks=Hkv * D,
                v=v.data_ptr(), vs=Hkv * D, seq=i.data_ptr(), slots=i.data_ptr(), pos=i.data_ptr(), num_rows=2, tab=tab.data_ptr(), out=out.data_ptr())
    call = lambda **kw: B.lib().opw_rope_append(st.handle, *{**good, **kw}.values(), None)  # noqa: E731
    for kw in (dict(layer=1), dict(rows=-1), dict(rot=0), dict(rot=63), dict(rot=66), dict(layout=2), dict(table=None), dict(table=good["table"] + 4),
               dict(q=None), dict(out=None), dict(k=None), dict(v=good["v"] + 2), dict(qs=Hq * D - 8), dict(qs=Hq * D + 4), dict(ks=Hkv * D - 8),
               dict(vs=Hkv * D + 1), dict(seq=None), dict(slots=good["slots"] + 2), dict(pos=None), dict(num_rows=0), dict(tab=None),
               dict(out=good["q"], qs=Hq * D + 8)):
        assert call(**kw) == B.OPW_ERR_INVALID_ARG, kw
    assert st.launch_count() == 0 and call(rows=0) == B.OPW_OK
    with pytest.raises(ValueError):
        st.rope_append(0, rope, q.half(), k, v, i, i, i, tab, out)
    with pytest.raises(ValueError):
        st.rope_append(0, rope, q, k, v, i, i, i, tab, out[:2])
    with pytest.raises(ValueError):
        st.rope_append(0, rope, q.transpose(0, 1).contiguous().transpose(0, 1), k, v, i, i, i, tab, out)


# --------------------------------------------------------------------------------- commit ---

@pytest.mark.parametrize("Hkv,D,layers,T", [(2, 64, 1, 1), (8, 128, 3, 7), (8, 128, 1, 64), (2, 256, 2, 64), (1, 64, 1, 33)])
def test_commit_gathers_the_accepted_rows(Hkv, D, layers, T):
    rng = np.random.default_rng(3000 + D + T)
    ctx = [0, 15, 16, 100, -1, 31, 7]
    pools, tab = [], None
    lens = [max(c, 0) + T for c in ctx]
    for _ in range(layers):
        pool, t, _, _, _ = make_case(np.random.default_rng(8), lens, Hkv, Hkv, D)
        pools.append(rand_bits(rng, pool.shape))
        tab = t.astype(np.int32)
    took = [T, max(1, T // 2), 0, T // 3, T, -3, 1]
    path = np.full((len(ctx), T), 1 << 20, np.int32)            # what lies behind the path is never read
    for b, m in enumerate(took):
        if m > 0:
            path[b, :m] = np.sort(rng.permutation(T)[:m])
    path[6, 0] = T - 1
    d_pools = [dev(p, True) for p in pools]
    st = make_stage(d_pools, Hkv, Hkv, D, len(ctx), tab.shape[1])
    new = torch.full((len(ctx),), 99, dtype=torch.int32, device="cuda")
    st.kv_commit(list(range(layers)), dev(path), dev(np.array(took, np.int32)), dev(np.array(ctx, np.int32)), dev(tab), new)
    assert st.poll_error() == B.OPW_OK and st.launch_count() == 1
    for p, d in zip(pools, d_pools):
        want = draft.commit(p, Hkv, D, path, took, ctx, tab, T)
        assert (host_bits(d) == p).all()
    assert (new.cpu().numpy() == want).all()


def test_commit_takes_any_list_of_rows_and_records_bad_ones():
    rng = np.random.default_rng(3100)
    Hkv, D, T = 2, 64, 9
    pool, tab, _, _, _ = make_case(rng, [20 + T, 5 + T], Hkv, Hkv, D)
    tab = tab.astype(np.int32)
    path = np.array([[3, 3, 0, 8, 1, 1, 0, 0, 0], [8, 7, 6, 5, 4, 3, 2, 1, 0]], np.int32)     # repeated; reversed
    want = pool.copy()
    draft.commit(want, Hkv, D, path, [5, 9], [20, 5], tab, T)
    d_pool = dev(pool, True)
    st = make_stage([d_pool], Hkv, Hkv, D, 2, tab.shape[1])
    ctx = dev(np.array([20, 5], np.int32))
    st.kv_commit([0], dev(path), dev(np.array([5, 9], np.int32)), ctx, dev(tab))
    assert st.poll_error() == B.OPW_OK and (host_bits(d_pool) == want).all()
    before = host_bits(d_pool).copy()
    for p in ([-1] + [0] * 8, [9] + [0] * 8):
        st.kv_commit([0], dev(np.array([p, p], np.int32)), dev(np.array([1, 0], np.int32)), ctx, dev(tab))
        assert st.poll_error() == B.OPW_ERR_BAD_PAGE and (host_bits(d_pool) == before).all()
    cut = tab.copy()
    cut[0, 1] = -1
    st.kv_commit([0], dev(np.array([[2] + [0] * 8, [1] + [0] * 8], np.int32)), dev(np.array([1, 0], np.int32)), ctx, dev(cut))
    assert st.poll_error() == B.OPW_ERR_BAD_PAGE and (host_bits(d_pool) == before).all()
    new = torch.zeros(2, dtype=torch.int32, device="cuda")
    ident = np.arange(T, dtype=np.int32)[None].repeat(2, 0)
    st.kv_commit([0], dev(ident), dev(np.array([T + 1, 2], np.int32)), ctx, dev(tab), new)
    assert st.poll_error() == B.OPW_ERR_BAD_PAGE and new.tolist() == [20 + T, 7] and (host_bits(d_pool) == before).all()


def test_commit_and_page_calls_refuse():
    Hkv, D = 2, 64
    pools = [torch.zeros(4 * Hkv * 2 * 16 * D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    st = make_stage(pools, Hkv, Hkv, D, 2, 2)
    L = B.lib()
    i = torch.zeros(64, dtype=torch.int32, device="cuda")
    a = [i.data_ptr() + 32 * n for n in range(8)]
    arr = lambda *x: (ctypes.c_int32 * len(x))(*x)  # noqa: E731
    commit = dict(layers=arr(0, 1), n=2, batch=2, nodes=4, path=a[0], took=a[1], ctx=a[2], tab=a[3], new=a[4])
    call = lambda f, good, **kw: f(st.handle, *{**good, **kw}.values(), None)  # noqa: E731
    for kw in (dict(layers=None), dict(n=0), dict(n=3), dict(layers=arr(0, 0)), dict(layers=arr(0, 2)), dict(layers=arr(-1, 0)), dict(batch=-1),
               dict(nodes=0), dict(nodes=65), dict(path=None), dict(took=None), dict(ctx=None), dict(tab=a[3] + 2), dict(new=a[2]), dict(new=a[1] + 4)):
        assert call(L.opw_kv_commit, commit, **kw) == B.OPW_ERR_INVALID_ARG, kw
    assert call(L.opw_kv_commit, commit, batch=3) == B.OPW_ERR_CAPACITY and call(L.opw_kv_commit, commit, batch=0) == B.OPW_OK
    fork = dict(layers=arr(0), n_layers=1, n=2, src=a[0], dst=a[1], lens=a[2], new=a[3], rows=2, tab=a[4], refs=a[5])
    for kw in (dict(layers=None), dict(n_layers=0), dict(layers=arr(5)), dict(n=-1), dict(src=None), dict(dst=None), dict(lens=a[2] + 1), dict(new=None),
               dict(rows=0), dict(tab=None), dict(refs=None)):
        assert call(L.opw_kv_fork, fork, **kw) == B.OPW_ERR_INVALID_ARG, kw
    assert call(L.opw_kv_fork, fork, n=65536) == B.OPW_ERR_CAPACITY and call(L.opw_kv_fork, fork, n=0) == B.OPW_OK
    drop = dict(n=2, rows=a[0], keep=None, num_rows=2, tab=a[1], refs=a[2], pages=4)
    for kw in (dict(n=-1), dict(rows=None), dict(keep=a[3] + 2), dict(num_rows=0), dict(tab=None), dict(refs=None), dict(pages=0), dict(pages=1 << 31)):
        assert call(L.opw_kv_release, drop, **kw) == B.OPW_ERR_INVALID_ARG, kw
    assert call(L.opw_kv_release, drop, n=65536) == B.OPW_ERR_CAPACITY and call(L.opw_kv_release, drop, n=0) == B.OPW_OK
    free = dict(refs=a[0], pages=4, lst=a[1], most=4, count=a[2])
    for kw in (dict(refs=None), dict(pages=0), dict(pages=1 << 31), dict(lst=None), dict(most=-1), dict(count=None), dict(count=a[2] + 1)):
        assert call(L.opw_kv_free_pages, free, **kw) == B.OPW_ERR_INVALID_ARG, kw
    assert st.launch_count() == 0
    with pytest.raises(ValueError):
        st.kv_fork([0], i[:2], i[:2], i[:2], i[:2], torch.zeros(2, 2, dtype=torch.int32, device="cuda"), i[:3])


# ---------------------------------------------------------------------------------- pages ---

@pytest.mark.parametrize("Hkv,D,layers", [(2, 64, 1), (8, 128, 3), (2, 256, 2)])
def test_fork_release_and_the_free_list(Hkv, D, layers):
    rng = np.random.default_rng(4000 + D)
    width, total, rows = 300, 900, 12
    tab = np.full((rows, width), -1, np.int32)
    order = rng.permutation(total).astype(np.int32)
    have = [290, 3, 40]
    counts, at = np.zeros(total, np.int32), 0
    for r, n in enumerate(have):
        tab[r, :n] = order[at:at + n]
        counts[order[at:at + n]] += 1
        at += n
    tab[2, :10] = -1                                            # a window layer's table: early pages are gone
    counts[order[have[0] + have[1]:have[0] + have[1] + 10]] = 0
    src = np.array([0, 0, 1, 2, 0, 1, 0], np.int32)
    dst = np.array([5, 3, 4, 11, 7, 8, 9], np.int32)
    lens = np.array([290 * 16, 4633, 33, 601, 0, 48, 7], np.int32)
    new = order[at:at + 7]
    pools = [rand_bits(rng, oracle.pool_elems(total, Hkv, P, D)) for _ in range(layers)]
    d_pools, d_tab, d_counts = [dev(p, True) for p in pools], dev(tab), dev(counts)
    st = make_stage(d_pools, Hkv, Hkv, D, rows, width)
    st.kv_fork(list(range(layers)), dev(src), dev(dst), dev(lens), dev(new), d_tab, d_counts)
    assert st.poll_error() == B.OPW_OK and st.launch_count() == 1
    draft.fork(pools, Hkv, D, src, dst, lens, new, tab, counts)
    assert (d_tab.cpu().numpy() == tab).all() and (d_counts.cpu().numpy() == counts).all()
    for p, d in zip(pools, d_pools):
        assert (host_bits(d) == p).all()

    def free_list():
        lst, n = torch.full((total,), -7, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        st.kv_free_pages(d_counts, lst, n)
        short, n2 = torch.full((4,), -7, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        st.kv_free_pages(d_counts, short[:3], n2)
        want = np.nonzero(counts == 0)[0]
        assert n.item() == n2.item() == len(want) and (lst[:len(want)].cpu().numpy() == want).all() and (lst[len(want):] == -7).all()
        assert short.tolist() == list(want[:3]) + [-7] * (4 - len(want[:3]))

    free_list()
    # drop a parent, cut a child, drop the others; a row named twice is dropped once
    for r, keep in (([0, 0], None), ([5, 3], [17, 0]), ([11, 4, 7, 11], [-5, 16, 3, 100])):
        keep_d = None if keep is None else dev(np.array(keep, np.int32))
        st.kv_release(dev(np.array(r, np.int32)), keep_d, d_tab, d_counts)
        draft.release(r, keep, tab, counts)
        assert (d_tab.cpu().numpy() == tab).all() and (d_counts.cpu().numpy() == counts).all()
    assert st.poll_error() == B.OPW_OK
    free_list()
    st.kv_release(dev(np.arange(rows, dtype=np.int32)), None, d_tab, d_counts)
    counts[:] = 0
    assert (d_tab == -1).all() and (d_counts == 0).all() and st.poll_error() == B.OPW_OK
    free_list()


def test_fork_refuses_bad_forks_as_a_whole():
    rng = np.random.default_rng(4100)
    Hkv, D, total, rows, width = 2, 64, 40, 10, 4
    pool = rand_bits(rng, oracle.pool_elems(total, Hkv, P, D))
    tab = np.full((rows, width), -1, np.int32)
    tab[0] = [0, 1, 2, 3]
    tab[1, :2] = [4, 77]
    counts = np.zeros(total, np.int32)
    counts[:5] = 1

    def forked(src, dst, lens, new):
        d_pool, d_tab, d_counts = dev(pool, True), dev(tab), dev(counts)
        st = make_stage([d_pool], Hkv, Hkv, D, rows, width)
        st.kv_fork([0], *(dev(np.array(x, np.int32)) for x in (src, dst, lens, new)), d_tab, d_counts)
        return st.poll_error(), d_tab.cpu().numpy(), d_counts.cpu().numpy(), host_bits(d_pool)

    for src, dst, ln, new in ((0, 10, 5, 30), (-1, 2, 5, 30), (10, 2, 5, 30), (0, -3, 5, 30), (0, 2, -1, 30), (0, 2, 65, 30), (0, 2, 5, 40),
                              (0, 2, 5, -1), (0, 0, 5, 30), (2, 3, 5, 30), (1, 3, 17, 30)):
        rc, t, c, p = forked([src, 0], [dst, 9], [ln, 20], [new, 31])
        assert rc == B.OPW_ERR_BAD_PAGE, (src, dst, ln, new)
        wp, wt, wc = pool.copy(), tab.copy(), counts.copy()
        if (src, dst) != (0, 0):
            draft.fork([wp], Hkv, D, [0], [9], [20], [31], wt, wc)
        else:                                                  # row 0 is named as a target: no fork may read it
            pass
        assert (t == wt).all() and (c == wc).all() and (p == wp).all(), (src, dst, ln, new)
    # one target twice, one new page twice, a target that is another's source
    for src, dst, lens, new in (([0, 0], [2, 2], [5, 5], [30, 31]), ([0, 0], [2, 3], [5, 5], [30, 30]), ([0, 3], [3, 5], [16, 0], [30, 31])):
        rc, t, c, p = forked(src, dst, lens, new)
        assert rc == B.OPW_ERR_BAD_PAGE and (t == tab).all() and (c == counts).all() and (p == pool).all()
    # the same new page is no conflict where only one fork needs it
    rc, t, c, p = forked([0, 0], [2, 3], [5, 16], [30, 30])
    assert rc == B.OPW_OK and t[2].tolist() == [30, -1, -1, -1] and t[3].tolist() == [0, -1, -1, -1] and c[0] == 2 and c[30] == 1
    # an entry beyond the pool is not handed on
    rc, t, c, p = forked([1], [3], [32], [30])
    assert rc == B.OPW_ERR_BAD_PAGE and t[3].tolist() == [4, -1, -1, -1] and c[4] == 2


def test_release_records_what_does_not_fit():
    tab = torch.tensor([[0, 1], [2, 9], [3, -1]], dtype=torch.int32, device="cuda")
    counts = torch.tensor([1, 0, 2, 1], dtype=torch.int32, device="cuda")
    st = make_stage([torch.zeros(4 * 2 * 16 * 64, dtype=torch.bfloat16, device="cuda")], 1, 1, 64, 3, 2)
    st.kv_release(dev(np.array([0], np.int32)), None, tab, counts)
    assert st.poll_error() == B.OPW_ERR_BAD_PAGE and counts.tolist() == [0, 0, 2, 1] and tab[0].tolist() == [-1, -1]
    st.kv_release(dev(np.array([1], np.int32)), None, tab, counts)
    assert st.poll_error() == B.OPW_ERR_BAD_PAGE and counts.tolist() == [0, 0, 1, 1]
    st.kv_release(dev(np.array([-1, 3], np.int32)), None, tab, counts)
    assert st.poll_error() == B.OPW_ERR_BAD_PAGE and counts.tolist() == [0, 0, 1, 1] and tab[2].tolist() == [3, -1]


@pytest.mark.parametrize("total", [1, 7, 8, 1023, 8192, 100003, 600001])
def test_free_list_of_any_length(total):
    rng = np.random.default_rng(total)
    counts = (rng.random(total) < 0.4).astype(np.int32) * rng.integers(1, 5, size=total).astype(np.int32)
    st = make_stage([torch.zeros(4 * 2 * 16 * 64, dtype=torch.bfloat16, device="cuda")], 1, 1, 64, 1, 1)
    lst, n = torch.full((total,), -7, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    st.kv_free_pages(dev(counts), lst, n)
    want = np.nonzero(counts == 0)[0]
    assert n.item() == len(want) and (lst[:len(want)].cpu().numpy() == want).all() and (lst[len(want):] == -7).all()


# ------------------------------------------------------------------------------ a whole run ---

def test_a_pool_of_more_than_32_bits_of_elements():
    """The same step on pages at the end of a pool of 4.6e9 elements and on a small one: equal bit for bit."""
    rng = np.random.default_rng(4900)
    Hq, Hkv, D, T, width, per = 32, 8, 128, 20, 8, 2 * 8 * 16 * 128
    big_pages = 140000
    assert big_pages * per > 1 << 32
    x = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda().bfloat16()  # noqa: E731
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    n = 75
    q, k, v = x(2, T, Hq, D), x(2 * n, Hkv, D), x(2 * n, Hkv, D)
    seq, at = i32([0] * n + [1] * n), i32(list(range(n)) * 2)
    ids = rng.permutation(3 * width).astype(np.int32)
    mask = dev(np.array([B.opw_tree_mask(random_tree(rng, T))[0] for _ in range(2)], np.uint64))
    acc = i32([[3, 5, 11] + [0] * (T - 3), [0, 1, 19] + [0] * (T - 3)])
    res = []
    for pages, base in ((3 * width, 0), (big_pages, big_pages - 3 * width)):
        pool = torch.empty(pages * per, dtype=torch.bfloat16, device="cuda")
        pool[-3 * width * per:] = 0
        st = make_stage([pool], Hq, Hkv, D, 4, width)
        tree = B.TreeAttention(st, T)
        tab = dev(np.concatenate([ids[:2 * width].reshape(2, width) + base, np.full((2, width), -1, np.int32)]).astype(np.int32))
        refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
        refs[tab[:2].long().view(-1)] = 1
        st.rope_append(0, B.Rope(D), None, k, v, seq, at, at, tab, None)
        out, few = torch.empty_like(q), torch.empty_like(q[:, :2])
        ctx, sizes = i32([n - T, n - T]), i32([T, T])
        tree.attention(0, q, mask, ctx[:, None] + i32([list(range(T))] * 2), ctx, sizes, tab, out)
        wide = [t.repeat(40, 1, *[1] * (t.dim() - 2)) for t in (q[:, :2], mask[:, :2])]     # many rows of few nodes: a warp per page
        st2 = make_stage([pool], Hq, Hkv, D, 80, width)
        tree2, few = B.TreeAttention(st2, 2), torch.empty_like(wide[0].contiguous())
        tree2.attention(0, wide[0].contiguous(), wide[1].contiguous(), i32([[n, n + 1]] * 80), ctx.repeat(40), i32([2] * 80),
                        tab[:2].repeat(40, 1).contiguous(), few)
        st.kv_commit([0], acc, i32([3, 3]), ctx, tab)
        st.kv_fork([0], i32([0, 1]), i32([2, 3]), i32([n - T + 3, n - T + 3]), dev(ids[2 * width:2 * width + 2] + np.int32(base)), tab, refs)
        assert st.poll_error() == B.OPW_OK and st2.poll_error() == B.OPW_OK
        res.append((out, few, pool[-3 * width * per:].clone(), torch.where(tab < 0, tab, tab - base), refs[-3 * width:].clone()))
        tree.close(), tree2.close(), st.close(), st2.close()
        del pool, refs
    torch.cuda.empty_cache()
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_a_whole_step_captured_and_replayed_equals_eager_calls():
    """Fork, rotary append, tree attention, commit, release and the free list in one graph, replayed with changed inputs."""
    rng = np.random.default_rng(4950)
    Hq, Hkv, D, T, width, total, n = 32, 8, 128, 6, 6, 48, 41
    per = 2 * Hkv * 16 * D
    x = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda().bfloat16()  # noqa: E731
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    start = x(total * per)
    first_tab = np.full((4, width), -1, np.int32)
    first_tab[0], first_tab[1] = rng.permutation(total)[:12].reshape(2, 6)
    first_refs = np.zeros(total, np.int32)
    first_refs[first_tab[:2].ravel()] = 1
    spare = i32([i for i in range(total) if not first_refs[i]][:2])
    pool = start.clone()
    tab, refs = dev(first_tab), dev(first_refs)
    st = make_stage([pool], Hq, Hkv, D, 4, width)
    tree, rope = B.TreeAttention(st, T), B.Rope(64, layout="interleaved")
    parents = random_tree(rng, T)
    m, depth = B.opw_tree_mask(parents)
    mask = dev(np.array([m] * 4, np.uint64))
    q, k, v = x(4 * T, Hq, D), x(4 * T, Hkv, D), x(4 * T, Hkv, D)
    ctx, sizes = i32([n, n + 20, 0, 0]), i32([T, 3, 2, 0])
    new, out, lse = torch.empty_like(ctx), torch.empty(4, T, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(4, T, Hq, device="cuda")
    took, acc = i32([2, 1, 1, 0]), i32([[1, 4, 0, 0, 0, 0], [2, 0, 0, 0, 0, 0], [0] * 6, [0] * 6])
    lens = i32([n, n + 5])
    seq, pos, slots = i32([b for b in range(4) for _ in range(T)]), torch.empty(4 * T, dtype=torch.int32, device="cuda"), None
    qr, dep = torch.empty_like(q), i32([depth] * 4)
    slots = torch.empty_like(pos)
    lst, cnt, gone = torch.full((total,), -7, dtype=torch.int32, device="cuda"), i32([0]), i32([0])

    def reset():
        pool.copy_(start), tab.copy_(dev(first_tab)), refs.copy_(dev(first_refs)), lst.fill_(-7), out.fill_(0), lse.fill_(0)

    def step():
        st.kv_fork([0], i2[0], i2[1], lens, spare, tab, refs)
        ctx[2:].copy_(lens)
        pos.copy_((ctx[:, None] + dep).view(-1))
        slots.copy_((ctx[:, None] + ar).view(-1))
        st.rope_append(0, rope, q, k, v, seq, slots, pos, tab, qr)
        tree.attention(0, qr.view(4, T, Hq, D), mask, pos.view(4, T), ctx, sizes, tab, out, lse)
        st.kv_commit([0], acc, took, ctx, tab, new)
        st.kv_release(gone, None, tab, refs)
        st.kv_free_pages(refs, lst, cnt)

    i2, ar = (i32([0, 1]), i32([2, 3])), torch.arange(T, dtype=torch.int32, device="cuda")
    state = lambda: [t.clone() for t in (pool, tab, refs, qr, out, lse, new, lst, cnt)]  # noqa: E731
    reset(), step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    reset()
    with torch.cuda.graph(g):
        step()
    for change in ((n, n + 5), (16, 33), (0, 47)):
        lens.copy_(i32(list(change)))
        q.copy_(x(*q.shape))
        reset(), step()
        eager = state()
        reset(), g.replay()
        for a, b in zip(eager, state()):
            assert torch.equal(a, b)
        assert (eager[1][0] == -1).all() and eager[8].item() == int((eager[2] == 0).sum())
    # rows of the forks without a page for the drafted tokens are recorded
    assert st.poll_error() in (B.OPW_OK, B.OPW_ERR_BAD_PAGE)


def test_empty_calls_do_nothing():
    st = make_stage([torch.zeros(2 * 2 * 16 * 64, dtype=torch.bfloat16, device="cuda")], 2, 1, 64, 2, 2)
    tree, rope = B.TreeAttention(st, 3), B.Rope(64)
    e = lambda *s, t=torch.int32: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
    h = lambda *s: e(*s, t=torch.bfloat16)  # noqa: E731
    tab, refs = e(2, 2).fill_(-1), e(2).fill_(0)
    st.rope_append(0, rope, h(0, 2, 64), h(0, 1, 64), h(0, 1, 64), e(0), e(0), e(0), tab, h(0, 2, 64))
    tree.attention(0, h(0, 3, 2, 64), e(0, 3, t=torch.int64), e(0, 3), e(0), e(0), tab, h(0, 3, 2, 64))
    st.kv_commit([0], e(0, 3), e(0), e(0), tab, e(0))
    st.kv_fork([0], e(0), e(0), e(0), e(0), tab, refs)
    st.kv_release(e(0), None, tab, refs)
    count = e(1)
    assert st.launch_count() == 0
    st.kv_free_pages(refs, e(0), count)          # only counted
    assert count.item() == 2 and st.poll_error() == B.OPW_OK


@pytest.mark.parametrize("window", [0, 24])
def test_draft_verify_commit_equals_token_by_token(window):
    """Two sequences forked from one prompt; each step drafts a tree, verifies it, accepts a path, commits.  Every accepted
    node's output equals (to rounding) what token-by-token decoding of the same tokens gives, and the caches are equal
    bit for bit."""
    rng = np.random.default_rng(5000 + window)
    Hq, Hkv, D, T, width, total = 32, 8, 128, 9, 12, 64
    pools = [torch.zeros(total * Hkv * 2 * 16 * D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kw = dict(Hq=Hq, Hkv=Hkv, D=D, rows=3, width=width, window=window)
    a, b = make_stage(pools[:1], **kw), make_stage(pools[1:], **kw)
    rope = B.Rope(D)
    tree = B.TreeAttention(a, T)
    x = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda().bfloat16()  # noqa: E731
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    tab = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
    tab[0, :3] = i32([9, 4, 30])
    counts = torch.zeros(total, dtype=torch.int32, device="cuda")
    counts[tab[0, :3].long()] = 1
    n = 37
    k, v = x(n, Hkv, D), x(n, Hkv, D)
    for st in (a, b):
        st.rope_append(0, rope, None, k, v, i32([0] * n), i32(list(range(n))), i32(list(range(n))), tab, None)
    other = tab.clone(), counts.clone()
    for st, (t, c) in ((a, (tab, counts)), (b, other)):
        st.kv_fork([0], i32([0, 0]), i32([1, 2]), i32([n, n]), i32([11, 12]), t, c)
        st.kv_release(i32([0]), None, t, c)
    assert torch.equal(tab, other[0]) and counts[9].item() == 2 and counts[30].item() == 0
    # pages for what comes, from the free list
    lst, cnt = torch.zeros(total, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    a.kv_free_pages(counts, lst, cnt)
    tab[1, 3:], tab[2, 3:] = lst[:width - 3], lst[width - 3:2 * width - 6]
    lens = i32([n, n])
    rows_tab = tab[1:].contiguous()
    ones = torch.empty(1, Hq, D, dtype=torch.bfloat16, device="cuda")
    for step in range(4):
        parents = [random_tree(rng, T) for _ in range(2)]
        both = [B.opw_tree_mask(p) for p in parents]
        mask, depth = dev(np.array([m for m, _ in both], np.uint64)), i32([d for _, d in both])
        pos = lens[:, None] + depth
        q, k, v = x(2, T, Hq, D), x(2, T, Hkv, D), x(2, T, Hkv, D)
        slots = lens[:, None] + torch.arange(T, dtype=torch.int32, device="cuda")
        seq = i32([0] * T + [1] * T)
        qr = torch.empty_like(q)
        a.rope_append(0, rope, q.view(2 * T, Hq, D), k.view(2 * T, Hkv, D), v.view(2 * T, Hkv, D), seq, slots.view(-1), pos.view(-1),
                      rows_tab, qr.view(2 * T, Hq, D))
        out = torch.empty_like(q)
        tree.attention(0, qr, mask, pos, lens, i32([T, T]), rows_tab, out)
        leaf = [int(rng.integers(0, T)) for _ in range(2)]
        path = [[i for i in range(T) if both[s][0][leaf[s]] >> i & 1] for s in range(2)]
        took = i32([len(p) for p in path])
        new = torch.empty_like(lens)
        a.kv_commit([0], i32([p + [0] * (T - len(p)) for p in path]), took, lens, rows_tab, new)
        for s in range(2):                                      # the same tokens one by one
            for j, i in enumerate(path[s]):
                at = i32([int(lens[s]) + j])
                q1, k1 = torch.empty(1, Hq, D, dtype=torch.bfloat16, device="cuda"), k[s, i][None]
                b.rope_append(0, rope, q[s, i][None], k1, v[s, i][None], i32([s]), at, at, rows_tab, q1)
                b.decode_attention(0, q1, at + 1, rows_tab[s:s + 1], ones)
                assert torch.equal(q1[0], qr[s, i])
                diff = (ones[0].float() - out[s, i].float()).abs()
                # two roundings of P and two of the output, each 2^-8 of values that are at most max|V| ~ 4.5
                assert diff.max() <= 4 * 2.0 ** -8 * 4.5
        lens = new
    assert a.poll_error() == B.OPW_OK and b.poll_error() == B.OPW_OK
    for s in range(2):
        for st_pool in ((pools[0], pools[1]),):
            got = [oracle.gather_logical(host_bits(p), Hkv, P, D, rows_tab[s].cpu().numpy(), 0, int(lens[s])) for p in st_pool]
            assert (got[0][0] == got[1][0]).all() and (got[0][1] == got[1][1]).all()
