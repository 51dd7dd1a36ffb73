"""A whole step in one graph, replayed on other states and compared with the oracles: nothing recorded, and every table entry, count, place, output,
path and committed row as they have to be."""
import numpy as np
import pytest
import torch

import oracle
from helpers import P, out_to_f64
from oracle import draft, step
from paper_2609_14237_b200 import binding as B
from test_gpu_prefix import check
from test_gpu_step import norm_reference, check_norm
from test_gpu_step_run import Server, bits, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()
    assert torch.cuda.is_available()


def sampled_state(rng, n, groups, width, pages):
    """Rows with lengths, and the table and counts of a server that has forked each group's first whole pages."""
    have = rng.integers(1, 90, size=n)
    table, counts, free, shared = np.full((n, width), -1, np.int64), np.zeros(pages, np.int64), list(rng.permutation(pages)), []
    for lo, hi in zip(groups, groups[1:]):
        shared.append(int(rng.integers(0, have[lo:hi].min() + 1)))
        whole = [free.pop() for _ in range(shared[-1] // P)]
        for b in range(lo, hi):
            table[b, :len(whole)] = whole
            for i in range(len(whole), -(-int(have[b]) // P)):
                table[b, i] = free.pop()
    np.add.at(counts, table[table >= 0], 1)
    return have, shared, table, counts


@pytest.mark.parametrize("Hq,Hkv,D", [(32, 8, 128), (8, 2, 64), (6, 2, 256)])
@pytest.mark.parametrize("draw", ["again", "distinct", "certain"])
def test_a_captured_step_matches_the_oracles(Hq, Hkv, D, draw):
    """Release, free list, a token for every sequence, its attention behind the prefix, a drafted tree for every sequence from the rest of the
    list, its attention, verification, commit, and the pages of what was not kept given back."""
    n, T, V, width, pages, groups = 6, 5, 900, 9, 70, [0, 3, 6]
    s = Server(Hq, Hkv, D, n, width, pages, 17)
    st = s.st
    parents = [-1, 0, 0, 1, 1]
    mask, depth = B.opw_tree_mask(parents)
    ints = lambda *k: torch.zeros(*k, dtype=torch.int32, device="cuda")  # noqa: E731
    rows, old, one, many, starts, shared, cursor = i32(range(n)), ints(n), i32([1] * n), i32([T] * n), i32(groups), ints(2), ints(1)
    room = n * T + 3                                          # the drafted rows', and some that stay padding
    seq1, slots1, lens, seq2, slots2, begins, longer = ints(n), ints(n), ints(n), ints(room), ints(room), ints(n + 1), ints(n)
    qkv1, qkv2 = (torch.empty(k, Hq + 2 * Hkv, D, dtype=torch.bfloat16, device="cuda") for k in (n, room))
    parts = lambda x: (x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:])  # noqa: E731
    q1, out1 = (torch.empty(n, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q2, out2 = (torch.empty(k, Hq, D, dtype=torch.bfloat16, device="cuda") for k in (room, n * T))
    lse1, lse2 = torch.empty(n, Hq, device="cuda"), torch.empty(n, T, Hq, device="cuda")
    masks, par, deep = torch.tensor([mask] * n, dtype=torch.uint64, device="cuda"), i32([parents] * n), i32(depth)
    at, pad = ints(n, T), ints(room)
    p, q, u = (torch.empty(*k, device="cuda") for k in ((n, T, V), (n, T, V), (n, T)))
    tokens, path, took, follows, after = ints(n, T), ints(n, T), ints(n), ints(n), ints(n)
    before_commit = torch.empty_like(s.pools[0])

    def one_step():
        cursor.zero_()
        st.kv_release(rows, old, s.table, s.counts)
        st.kv_free_pages(s.counts, s.free, s.n_free)
        st.kv_extend(rows, old, one, s.table, s.counts, s.free, s.n_free, new_lens=lens, seq=seq1, slots=slots1, free_begin=cursor, free_end=cursor)
        st.norm_rope_append(0, s.rope, *parts(qkv1), s.wq, s.wk, seq1, slots1, slots1, s.table, q1)
        s.prefix.attention(0, q1, lens, starts, shared, s.table, out1, lse1)
        st.kv_extend(rows, lens, many, s.table, s.counts, s.free, s.n_free, row_starts=begins, new_lens=longer, seq=seq2, slots=slots2,
                     free_begin=cursor, free_end=cursor)
        torch.add(lens[:, None], deep[None], out=at)
        pad[:n * T].copy_(at.view(-1))
        st.norm_rope_append(0, s.rope, *parts(qkv2), s.wq, s.wk, seq2, slots2, pad, s.table, q2)
        s.tree.attention(0, q2[:n * T].view(n, T, Hq, D), masks, at, lens, many, s.table, out2.view(n, T, Hq, D), lse2)
        before_commit.copy_(s.pools[0])
        st.tree_verify(p, None if draw == "certain" else q, tokens, par, many, u, path, took, follows, distinct=draw == "distinct")
        st.kv_commit([0], path, took, lens, s.table, after)
        st.kv_release(rows, after, s.table, s.counts)

    rng = np.random.default_rng(12 + D)
    f = draft.frequencies(D)
    graph = None
    accepted = 0
    for turn in range(4):
        have, pre, table, counts = sampled_state(rng, n, groups, width, pages)
        for x in (qkv1, qkv2):
            x.copy_(torch.randn(x.shape, generator=s.g, device="cuda"))
        p.copy_(torch.softmax(2 * torch.randn(p.shape, generator=s.g, device="cuda"), -1))
        q.copy_(torch.softmax(2 * torch.randn(p.shape, generator=s.g, device="cuda"), -1).add_(2 * p).div_(3))
        u.copy_(torch.rand(u.shape, generator=s.g, device="cuda"))
        pick = torch.multinomial(q.view(-1, V), 2, replacement=draw == "again", generator=s.g).view(n, T, 2)
        if draw == "certain":
            pick = torch.topk(p, 2, -1).indices
        for i, up in enumerate(parents[1:], 1):
            tokens[:, i] = pick[:, up, parents[:i].count(up)].int()

        def reset():
            old.copy_(i32(have)), shared.copy_(i32(pre)), s.table.copy_(i32(table)), s.counts.copy_(i32(counts))
            for x in (q1, out1, q2, out2, lse1, lse2):
                x.fill_(7.0)
        if graph is None:
            pool = s.pools[0].clone()
            reset(), one_step()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                one_step()
            s.pools[0].copy_(pool)
            assert st.poll_error() == B.OPW_OK
        reset()
        pool = bits(s.pools[0])
        graph.replay()
        assert st.poll_error() == B.OPW_OK
        # --- pages and places ---
        free = np.nonzero(counts == 0)[0]
        _, want_lens, want_seq, want_slots, end, bad = step.extend(range(n), have, [1] * n, table, counts, free, len(free), 0, n)
        assert not bad and (lens.cpu().numpy() == want_lens).all()
        assert (seq1.cpu().numpy() == want_seq).all() and (slots1.cpu().numpy() == want_slots).all()
        want_begins, want_longer, want_seq2, want_slots2, end, bad = step.extend(range(n), want_lens, [T] * n, table, counts, free, len(free), end, room)
        assert not bad and (longer.cpu().numpy() == want_longer).all() and (begins.cpu().numpy() == want_begins).all() and cursor.item() == end
        assert (seq2.cpu().numpy() == want_seq2).all() and (slots2.cpu().numpy() == want_slots2).all() and (want_seq2[n * T:] == -1).all()
        # --- queries, keys and values of both appends ---
        where = np.asarray(want_lens)[:, None] + np.asarray(depth)[None]
        final, mid = bits(s.pools[0]), bits(before_commit)
        for x, q_out, seq, slots, pos in ((qkv1, q1, want_seq, want_slots, want_slots), (qkv2, q2, want_seq2[:n * T], want_slots2[:n * T], where.reshape(-1))):
            m = len(seq)
            xf, pos = oracle.bf16_bits_to_f64(bits(x[:m])), pos.astype(np.float64)
            want, size = norm_reference(xf[:, :Hq], s.wq.double().cpu().numpy(), 1e-6, pos, f, "half", 1.0)
            check_norm(out_to_f64(q_out[:m]), want, size, D, pos)
            want, size = norm_reference(xf[:, Hq:Hq + Hkv], s.wk.double().cpu().numpy(), 1e-6, pos, f, "half", 1.0)
            kv = [oracle.gather_logical(mid, Hkv, P, D, table[b], int(t), int(t) + 1) for b, t in zip(seq, slots)]
            check_norm(np.stack([oracle.bf16_bits_to_f64(k[0]) for k, _ in kv]), want, size, D, pos)
            assert (np.stack([v[0] for _, v in kv]) == bits(x[:m])[:, Hq + Hkv:]).all()
            k, v = np.stack([k[0] for k, _ in kv]), np.stack([v[0] for _, v in kv])
            draft.append_rows(pool, Hkv, D, seq, slots, table, k, v)
        assert (pool == mid).all() and (out_to_f64(q2[n * T:]) == 7.0).all()             # nothing else in the cache moved; padding is left alone
        # --- attention ---
        check(out1, lse1, step.decode_attention(mid, Hq, Hkv, D, bits(q1), want_lens, table), 120)
        ref = draft.tree_attention(mid, Hq, Hkv, D, bits(q2[:n * T]).reshape(n, T, Hq, D), np.array([mask] * n, np.uint64), where, want_lens, [T] * n, table)
        check(out2.view(n, T, Hq, D), lse2, ref, 120)
        # --- the path, the rows that stay and the pages that go ---
        d = lambda x: x.double().cpu().numpy()  # noqa: E731
        want = step.verify(d(p), None if draw == "certain" else d(q), tokens.cpu().numpy(), par.cpu().numpy(), [T] * n, d(u), draw)
        assert all((a.cpu().numpy() == b).all() for a, b in zip((path, took, follows), want))
        accepted += int((want[1] > 1).sum())
        assert (after.cpu().numpy() == want_lens + want[1]).all()
        draft.commit(pool, Hkv, D, want[0], want[1], want_lens, table, T)
        assert (pool == final).all()
        draft.release(range(n), want_lens + want[1], table, counts)
        assert (s.table.cpu().numpy() == table).all() and (s.counts.cpu().numpy() == counts).all()
        assert (np.bincount(table[table >= 0], minlength=pages) == counts).all()
    assert accepted > 0
