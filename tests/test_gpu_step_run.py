"""The operators around a step's attention together, as a server calls them: prompts enter the cache, are sampled several times, decoded behind
their shared prefix, drafted ahead, verified and committed."""
import math

import numpy as np
import pytest
import torch

import oracle
from helpers import P, out_to_f64
from oracle import draft, step
from paper_2609_14237_b200 import binding as B
from test_gpu_prefix import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()
    assert torch.cuda.is_available()


def i32(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()


def bits(t):
    return t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


class Server:
    """Two layers (one with a window) over one page table, with the state a server keeps; every step goes by device tensors only."""

    def __init__(self, Hq, Hkv, D, rows, width, pages, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.g, self.Hq, self.Hkv, self.D, self.windows = g, Hq, Hkv, D, [0, 40]
        self.pools = [torch.randn(pages * Hkv * 2 * P * D, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
        self.st = B.Stage(pools=self.pools, layer_window=self.windows, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, max_batch=rows,
                          max_pages_per_seq=width)
        self.prefix, self.tree, self.rope = B.PrefixAttention(self.st), B.TreeAttention(self.st, 8), B.Rope(D)
        self.table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
        self.counts = torch.zeros(pages, dtype=torch.int32, device="cuda")
        self.free, self.n_free = torch.empty_like(self.counts), torch.zeros(1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.wq, self.wk = (1 + 0.1 * torch.randn(D, generator=g, device="cuda") for _ in range(2))

    def projections(self, n):
        x = torch.randn(n, self.Hq + 2 * self.Hkv, self.D, generator=self.g, device="cuda", dtype=torch.bfloat16)
        return x[:, :self.Hq], x[:, self.Hq:self.Hq + self.Hkv], x[:, self.Hq + self.Hkv:]

    def extend(self, rows, tokens, room):
        old, n = self.lens[rows.long()], rows.shape[0]
        out = {k: torch.empty(s, dtype=torch.int32, device="cuda") for k, s in (("seq", room), ("slots", room), ("row_starts", n + 1), ("new_lens", n))}
        self.st.kv_free_pages(self.counts, self.free, self.n_free)
        self.st.kv_extend(rows, old, tokens, self.table, self.counts, self.free, self.n_free, **out)
        return out

    def append(self, layer, qkv, seq, slots, positions=None):
        q_out = torch.zeros(qkv[0].shape, dtype=torch.bfloat16, device="cuda")
        self.st.norm_rope_append(layer, self.rope, *qkv, self.wq, self.wk, seq, slots, slots if positions is None else positions, self.table, q_out)
        return q_out


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (32, 8, 128), (6, 2, 256)])
def test_prompts_samples_and_drafts(Hq, Hkv, D):
    s = Server(Hq, Hkv, D, 16, 12, 96, 4)
    st, prompts, samples = s.st, [83, 50], 4
    # --- the prompts: pages, places, keys and values ---
    e = s.extend(i32([0, 1]), i32(prompts), sum(prompts) + 11)
    room = sum(prompts) + 11
    assert e["seq"].tolist() == [0] * 83 + [1] * 50 + [-1] * 11 and e["new_lens"].tolist() == prompts
    prompt_kv = [s.projections(room) for _ in range(2)]
    for layer in range(2):
        s.append(layer, prompt_kv[layer], e["seq"], e["slots"])
    s.lens[:2] = e["new_lens"]
    assert int(s.counts.sum()) == 6 + 4
    # --- each sampled: rows 2 .. 5 of the first, 6 .. 9 of the second ---
    src, dst = i32([0] * samples + [1] * samples), i32(range(2, 2 + 2 * samples))
    st.kv_free_pages(s.counts, s.free, s.n_free)
    st.kv_fork([0, 1], src, dst, s.lens[src.long()], s.free[:2 * samples].contiguous(), s.table, s.counts)
    s.lens[2:10] = s.lens[src.long()]
    starts, shared = i32([0, samples, 2 * samples]), i32(prompts)
    # --- decoded for a while behind the shared pages ---
    for t in range(18):
        e = s.extend(dst, i32([1] * 8), 8)
        for layer in range(2):
            q = s.append(layer, s.projections(8), e["seq"], e["slots"])
            out, lse = torch.empty_like(q), torch.empty(8, Hq, device="cuda")
            s.prefix.attention(layer, q, e["new_lens"], starts, shared, s.table[2:10], out, lse)
            if t % 6 == 5:
                ref = step.decode_attention(bits(s.pools[layer]), Hq, Hkv, D, bits(q), e["new_lens"].tolist(), s.table[2:10].cpu().numpy(),
                                            s.windows[layer])
                check(out, lse, ref, 120)
        s.lens[2:10] = e["new_lens"]
    assert st.poll_error() == B.OPW_OK
    # --- a tree of five drafted tokens for each: appended, attended to, verified, committed; what was not kept gives its pages back ---
    T, V = 5, 700
    parents = [-1, 0, 0, 1, 3]
    mask, depth = B.opw_tree_mask(parents)
    ctx = s.lens[2:10].clone()
    e = s.extend(dst, i32([T] * 8), 8 * T)
    at = ctx[:, None] + i32(depth)[None]
    masks, sizes = torch.tensor([mask] * 8, dtype=torch.uint64, device="cuda"), torch.full_like(ctx, T)
    drafted = [s.projections(8 * T) for _ in range(2)]
    for layer in range(2):
        q = s.append(layer, drafted[layer], e["seq"], e["slots"], at.reshape(-1).contiguous())
        out, lse = torch.empty(8, T, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(8, T, Hq, device="cuda")
        s.tree.attention(layer, q.view(8, T, Hq, D), masks, at, ctx, sizes, s.table[2:10], out, lse)
        ref = draft.tree_attention(bits(s.pools[layer]), Hq, Hkv, D, bits(q).reshape(8, T, Hq, D), np.array([mask] * 8, np.uint64),
                                   at.cpu().numpy(), ctx.tolist(), [T] * 8, s.table[2:10].cpu().numpy(), s.windows[layer])
        check(out, lse, ref, 120)
    p, q = (torch.softmax(3 * torch.randn(8, T, V, generator=s.g, device="cuda"), -1) for _ in range(2))
    q = 0.5 * (p + q)
    tokens = torch.multinomial(q[:, 0], T, replacement=True, generator=s.g).int()
    u = torch.rand(8, T, generator=s.g, device="cuda")
    par = i32([parents] * 8)
    path, took, follows, new = torch.empty_like(tokens), torch.empty_like(ctx), torch.empty_like(ctx), torch.empty_like(ctx)
    st.tree_verify(p, q, tokens, par, sizes, u, path, took, follows)
    want = step.verify(p.double().cpu().numpy(), q.double().cpu().numpy(), tokens.cpu().numpy(), par.cpu().numpy(), [T] * 8, u.double().cpu().numpy(), "again")
    assert all((a.cpu().numpy() == b).all() for a, b in zip((path, took, follows), want)) and took.max() > 1
    st.kv_commit([0, 1], path, took, ctx, s.table[2:10].contiguous(), new)
    assert torch.equal(new, ctx + took)
    st.kv_release(dst, new, s.table, s.counts)
    s.lens[2:10] = new
    assert st.poll_error() == B.OPW_OK
    held = [-(-int(n) // P) for n in s.lens[:10]]
    assert ((s.table >= 0).sum(1)[:10].tolist()) == held
    named = s.table[s.table >= 0].long()
    assert torch.equal(torch.bincount(named, minlength=s.counts.shape[0]).int(), s.counts)
    # the committed keys are those of the accepted nodes, rotated at their depth
    f = draft.frequencies(D)
    for b in range(8):
        c, way = int(ctx[b]), path[b, :int(took[b])].tolist()
        for layer in range(2):
            k, v = oracle.gather_logical(bits(s.pools[layer]), Hkv, P, D, s.table[2 + b].cpu().numpy(), c, c + len(way))
            x = out_to_f64(drafted[layer][1]).reshape(8, T, Hkv, D)[b, way]
            y = draft.rotate(step.head_norm(x, s.wk.double().cpu().numpy(), 1e-6), np.array([c + depth[i] for i in way], np.float64), f, "half")
            # half a step of bf16, and 2^-14 of the head's size for what fp32 adds (counted in the tests of the operator)
            assert (np.abs(oracle.bf16_bits_to_f64(k) - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -14 * math.sqrt(D)).all()
            assert (v == bits(drafted[layer][2]).reshape(8, T, Hkv, D)[b, way]).all()


def test_a_step_captured_and_replayed_equals_eager_calls():
    """Release, free list, extension, append with head norms, attention behind the prefix, verification and commit in one graph, replayed with
    other requests, lengths, groups and random numbers."""
    Hq, Hkv, D, n, T, V = 32, 8, 128, 6, 4, 3000
    s = Server(Hq, Hkv, D, n, 14, 120, 5)
    st, room = s.st, 40
    rows, old, new = i32(range(n)), i32([0] * n), i32([0] * n)
    starts, shared = i32([0, 3, n]), i32([0, 0])
    seq, slots, lens = (torch.empty(k, dtype=torch.int32, device="cuda") for k in (room, room, n))
    qkv = torch.empty(room, Hq + 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    q_out, one, out, lse = (torch.zeros(x, dtype=t, device="cuda") for x, t in (((room, Hq, D), torch.bfloat16), ((n, Hq, D), torch.bfloat16),
                                                                             ((n, Hq, D), torch.bfloat16), ((n, Hq), torch.float32)))
    p, d = (torch.empty(n, T, V, device="cuda") for _ in range(2))
    u, tokens = torch.empty(n, T, device="cuda"), torch.zeros(n, T, dtype=torch.int32, device="cuda")
    parents, sizes = i32([[-1, 0, 0, 2]] * n), i32([T] * n)
    path, took, follows, after = torch.empty_like(tokens), torch.empty_like(lens), torch.empty_like(lens), torch.empty_like(lens)
    start_pool = s.pools[0].clone()

    def one_step():
        st.kv_release(rows, old, s.table, s.counts)
        st.kv_free_pages(s.counts, s.free, s.n_free)
        st.kv_extend(rows, old, new, s.table, s.counts, s.free, s.n_free, new_lens=lens, seq=seq, slots=slots)
        st.norm_rope_append(0, s.rope, q, k, v, s.wq, None, seq, slots, slots, s.table, q_out)
        one.copy_(q_out[:n])
        s.prefix.attention(0, one, lens, starts, shared, s.table, out, lse)
        st.tree_verify(p, d, tokens, parents, sizes, u, path, took, follows)
        st.kv_commit([0], path, took, old, s.table, after)

    state = lambda: [x.clone() for x in (s.pools[0], s.table, s.counts, s.free, seq, slots, lens, q_out, out, lse, path, took, follows, after)]  # noqa: E731

    def reset(tab, counts):
        s.pools[0].copy_(start_pool), s.table.copy_(tab), s.counts.copy_(counts), s.free.fill_(-1)
        for x in (q_out, out, lse, path, took, follows, after, seq, slots, lens):
            x.zero_()

    rng = np.random.default_rng(11)
    graph = None
    for turn in range(4):
        have = rng.integers(0, 90, size=n)
        pre = [int(have[:3].min()), int(have[3:].min())]
        tab, counts, free = np.full((n, 14), -1, np.int32), np.zeros(120, np.int32), list(rng.permutation(120))
        for g in range(2):
            whole = [free.pop() for _ in range(pre[g] // P)]
            for b in range(3 * g, 3 * g + 3):
                tab[b, :len(whole)] = whole
                for i in range(len(whole), -(-int(have[b]) // P)):
                    tab[b, i] = free.pop()
        np.add.at(counts, tab[tab >= 0], 1)
        old.copy_(i32(have)), new.copy_(i32(rng.permutation([1, 1, 7, 2, 1, 20]))), shared.copy_(i32(pre))
        qkv.copy_(torch.randn(qkv.shape, generator=s.g, device="cuda"))
        p.copy_(torch.softmax(2 * torch.randn(p.shape, generator=s.g, device="cuda"), -1))
        d.copy_(torch.softmax(2 * torch.randn(p.shape, generator=s.g, device="cuda"), -1))
        tokens.copy_(torch.randint(0, V, tokens.shape, generator=s.g, device="cuda"))
        u.copy_(torch.rand(u.shape, generator=s.g, device="cuda"))
        tab, counts = torch.from_numpy(tab).cuda(), torch.from_numpy(counts).cuda()
        if graph is None:
            reset(tab, counts), one_step()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            reset(tab, counts)
            with torch.cuda.graph(graph):
                one_step()
        reset(tab, counts), one_step()
        eager = state()
        reset(tab, counts), graph.replay()
        for a, b in zip(eager, state()):
            assert torch.equal(a, b)
        assert (lens == old + new).all() and torch.isfinite(lse).all()
    assert st.poll_error() in (B.OPW_OK, B.OPW_ERR_BAD_PAGE)      # (paths may reach beyond the rows that got pages)
