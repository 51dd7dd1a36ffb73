"""The module-level calls of the operators around a step's attention: each reaches its entry point and raises what that refuses."""
import numpy as np
import pytest
import torch

from paper_2609_14237_b200 import binding as B


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()


@pytest.mark.parametrize("call", [
    lambda: B.opw_norm_rope_append(None, 0, 1, 64, 0, 16, 16, 64, 16, 64, 16, 64, None, None, 0, 1e-6, 16, 16, 16, 1, 16, 16),
    lambda: B.opw_tree_verify(None, 1, 4, 8, B.OPW_PROBS_F32, B.OPW_DRAW_AGAIN, 16, 8, 16, 8, *[16] * 7),
    lambda: B.opw_kv_extend(None, 1, 16, 16, 16, 1, 16, 16, 1, 16, 1, 16),
    lambda: B.opw_prefix_attention(None, 0, 1, 1, *[16] * 6),
])
def test_null_handles_raise(call):
    with pytest.raises(B.OpwError) as e:
        call()
    assert e.value.status == B.OPW_ERR_INVALID_ARG


@pytest.mark.gpu
def test_they_do_what_the_methods_do():
    """On addresses instead of tensors: the same bits as through Stage and PrefixAttention."""
    g = torch.Generator(device="cuda")
    g.manual_seed(31)
    Hq, Hkv, D, n, width, pages, T, V = 8, 2, 64, 3, 4, 12, 3, 50
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rope, wq = B.Rope(D), torch.rand(D, generator=g, device="cuda")
    x = torch.randn(n, Hq + 2 * Hkv, D, generator=g, device="cuda", dtype=torch.bfloat16)
    q, k, v = (t.contiguous() for t in (x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]))
    p, d = (torch.softmax(torch.randn(n, T, V, generator=g, device="cuda"), -1) for _ in range(2))
    tokens, parents, sizes, u = i32([[0, 3, 7]] * n), i32([[-1, 0, 0]] * n), i32([T] * n), torch.rand(n, T, generator=g, device="cuda")
    rows, old, new = i32([0, 1, 2]), i32([20, 3, 16]), i32([1, 1, 1])
    start = torch.randn(pages * Hkv * 2 * 16 * D, generator=g, device="cuda", dtype=torch.bfloat16)
    seen = []
    for direct in (False, True):
        pool = start.clone()
        st = B.Stage(pools=[pool], layer_window=[0], num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, max_batch=n, max_pages_per_seq=width)
        pre = B.PrefixAttention(st)
        tab, refs = i32([[0, 1, -1, -1], [2, -1, -1, -1], [3, -1, -1, -1]]), i32([1] * 4 + [0] * 8)
        free, count, end = i32(list(range(4, 12))), i32([8]), i32([0])
        starts, lens, seq, slots = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in (n + 1, n, 5, 5))
        q_out, out, lse = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(n, Hq, device="cuda")
        path, took, follows = torch.zeros_like(tokens), torch.zeros_like(rows), torch.zeros_like(rows)
        groups, shared = i32([0, n]), i32([0])
        if direct:
            a = lambda t: t.data_ptr()  # noqa: E731
            s = torch.cuda.current_stream().cuda_stream
            B.opw_kv_extend(st.handle, n, a(rows), a(old), a(new), n, a(tab), a(refs), pages, a(free), 8, a(count), None, a(end), a(starts), a(lens), 5,
                            a(seq), a(slots), s)
            B.opw_norm_rope_append(st.handle, 0, n, D, 0, a(rope.table), a(q), Hq * D, a(k), Hkv * D, a(v), Hkv * D, a(wq), None, 0, 1e-5, a(seq),
                                   a(slots), a(slots), n, a(tab), a(q_out), s)
            B.opw_prefix_attention(pre.handle, 0, n, 1, a(q_out), a(lens), a(groups), a(shared), a(tab), a(out), a(lse), s)
            B.opw_tree_verify(st.handle, n, T, V, B.OPW_PROBS_F32, B.OPW_DRAW_DISTINCT, a(p), V, a(d), V, a(tokens), a(parents), a(sizes), a(u), a(path),
                              a(took), a(follows), s)
        else:
            st.kv_extend(rows, old, new, tab, refs, free, count, row_starts=starts, new_lens=lens, seq=seq, slots=slots, free_end=end)
            st.norm_rope_append(0, rope, q, k, v, wq, None, seq[:n].contiguous(), slots[:n].contiguous(), slots[:n].contiguous(), tab, q_out, eps=1e-5)
            pre.attention(0, q_out, lens, groups, shared, tab, out, lse)
            st.tree_verify(p, d, tokens, parents, sizes, u, path, took, follows, distinct=True)
        assert st.poll_error() == B.OPW_OK and end.item() == 1 and lens.tolist() == [21, 4, 17]
        assert seq.tolist() == [0, 1, 2, -1, -1] and np.isfinite(lse.cpu().numpy()).all()
        seen.append([pool, tab, refs, starts, slots, q_out, out, lse, path, took, follows])
    assert all(torch.equal(a, b) for a, b in zip(*seen))
