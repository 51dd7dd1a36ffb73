"""GPU parity of the operators around a step's attention (head norms with rotary append, verification of drafted tokens, pages
for ragged requests) against the 64-bit oracle, and their refusals."""
import math

import numpy as np
import pytest
import torch

import oracle
from helpers import P, out_to_f64, rand_bits
from oracle import draft, step
from paper_2609_14237_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()
    assert torch.cuda.is_available()


def dev(a, bf16=False):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t.view(torch.int16).view(torch.bfloat16) if bf16 else t).cuda()


def i32(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()


def host_bits(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


def make_stage(pools, Hq, Hkv, D, rows, width, window=0, **kw):
    return B.Stage(pools=pools, layer_window=[window] * len(pools), num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, max_batch=rows,
                   max_pages_per_seq=width, **kw)


def small_stage(rows=4, width=4, **kw):
    return make_stage([torch.zeros(2 * 16 * 64, dtype=torch.bfloat16, device="cuda")], 1, 1, 64, rows, width, **kw)


# ---------------------------------------------------------------------------- head norms ---

def norm_reference(x, weight, eps, pos, f, layout, amp):
    """The normalised and rotated heads in 64 bits and, per element, the sizes of what is added up."""
    y = step.head_norm(x, weight, eps)
    z = draft.rotate(y, pos, f, layout, amp)
    r = len(f)
    size = np.abs(y)
    a, b = (np.arange(r), np.arange(r) + r) if layout == "half" else (2 * np.arange(r), 2 * np.arange(r) + 1)
    pair = amp * (size[..., a] + size[..., b])
    size[..., a], size[..., b] = pair, pair
    return z, size


def check_norm(got, want, size, D, pos):
    """Half a step of bf16 of the value.  In fp32: a sum of D squares and its mean (D / 2 + 2 roundings of at most 2^-24 each, as the sums run
    side by side; D + 4 is safe) under a square root (halved), 2^-22 for the reciprocal root, 4 products; cosine and sine 2^-22, their
    product with the amplitude and two operations of the rotation: together below ((D + 4) / 2 + 24) 2^-24 of |a| + |b|.  The angle: turns
    in 64 bits (pos 2^-52), rounded to fp32 below half a turn: 2^-25 turns, 2^-22 radians."""
    tol = 2.0 ** -8 * np.abs(want) + (((D + 4) / 2 + 24) * 2.0 ** -24 + 2.0 ** -22 + pos.max() * 2.0 ** -49) * size
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / (tol + 1e-30)).max()


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (32, 8, 128), (5, 1, 64), (6, 2, 256), (16, 1, 128)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("part", ["full", "half", "odd", "two"])
@pytest.mark.parametrize("weights", ["shared", "per head", "none"])
def test_norm_rope_append_matches_the_oracle(Hq, Hkv, D, layout, part, weights):
    rng = np.random.default_rng(6000 + D + Hq)
    rot = {"full": D, "half": D // 2, "odd": D // 4 + 2, "two": 2}[part]
    rows, eps = 23, 1e-5
    tab = rng.permutation(8).astype(np.int32).reshape(4, 2)
    seq = np.array([0] * 7 + [-1] + [3] * 9 + [1] * 5 + [2], np.int32)
    slots = np.concatenate([np.arange(12, 19), [0], np.arange(9), np.arange(27, 32), [16]]).astype(np.int32)
    pos = rng.integers(0, 1 << 20, size=rows).astype(np.int32)
    pos[0] = 0
    gain = np.exp2(rng.integers(-12, 13, size=(rows, 1, 1)))               # rows of very different size, down to where eps counts
    qkv = oracle.f32_to_bf16_bits((rng.standard_normal((rows, Hq + 2 * Hkv, D)) * gain).astype(np.float32))
    qkv[2] = 0                                                             # a row of zeros stays one
    pool = rand_bits(rng, oracle.pool_elems(8, Hkv, P, D))
    shape = lambda h: (h, D) if weights == "per head" else (D,)  # noqa: E731
    wq, wk = (None if weights == "none" else (1 + 0.3 * rng.standard_normal(shape(h))).astype(np.float32) for h in (Hq, Hkv))
    rope = B.Rope(rot, layout=layout, theta=10000.0, scaling="yarn", factor=8.0, original_context=8192.0)
    f, amp = draft.frequencies(rot, 10000.0, "yarn", 8.0, 8192.0), 1 + 0.1 * math.log(8.0)
    d_pool = dev(pool, True)
    st = make_stage([d_pool], Hq, Hkv, D, 4, 2)
    x = dev(qkv, True)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    q_out = torch.full((rows, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    g = [None if w is None else dev(w) for w in (wq, wk)]
    args = (dev(seq), dev(slots), dev(pos), dev(tab))
    st.norm_rope_append(0, rope, q, k, v, *g, *args, q_out, eps=eps)
    assert st.poll_error() == B.OPW_OK and st.launch_count() == 1
    xf, live = oracle.bf16_bits_to_f64(qkv), seq >= 0
    want, size = norm_reference(xf[:, :Hq], wq, eps, pos.astype(np.float64), f, layout, amp)
    got = out_to_f64(q_out)
    check_norm(got[live], want[live], size[live], D, pos)
    assert (got[~live] == 7.0).all() and (got[2] == 0).all()
    want, size = norm_reference(xf[:, Hq:Hq + Hkv], wk, eps, pos.astype(np.float64), f, layout, amp)
    want_pool, got_pool = pool.copy(), host_bits(d_pool)
    gk = np.zeros((rows, Hkv, D))
    for r in np.nonzero(live)[0]:
        a, b = oracle.gather_logical(got_pool, Hkv, P, D, tab[seq[r]], slots[r], slots[r] + 1)
        gk[r] = oracle.bf16_bits_to_f64(a[0])
        assert (b[0] == qkv[r, Hq + Hkv:]).all()
        draft._put_row(want_pool, Hkv, D, tab[seq[r], slots[r] // P], slots[r] % P, a[0], b[0])
    check_norm(gk[live], want[live], size[live], D, pos)
    assert (got_pool == want_pool).all()                                   # nothing else in the cache moved
    # from rows of their own, in place, and without queries
    d2, q2 = dev(pool, True), q.contiguous()
    st2 = make_stage([d2], Hq, Hkv, D, 4, 2)
    st2.norm_rope_append(0, rope, q2, k.contiguous(), v.contiguous(), *g, *args, q2, eps=eps)
    assert torch.equal(q2[dev(live)], q_out[dev(live)]) and torch.equal(q2[dev(~live)], q[dev(~live)]) and torch.equal(d2, d_pool)
    d3 = dev(pool, True)
    st3 = make_stage([d3], Hq, Hkv, D, 4, 2)
    st3.norm_rope_append(0, rope, None, k, v, *g, *args, None, eps=eps)
    assert torch.equal(d3, d_pool) and st3.poll_error() == B.OPW_OK


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (32, 8, 128), (6, 2, 256)])
@pytest.mark.parametrize("layout,rot", [("half", 64), ("interleaved", 64), ("half", 18), ("interleaved", 18)])
@pytest.mark.parametrize("per_head", [False, True])
def test_norm_rope_append_of_many_rows_equals_that_of_few(Hq, Hkv, D, layout, rot, per_head):
    """Many rows take another form of the kernel: the same bits as the same rows in small calls."""
    g = torch.Generator(device="cuda")
    g.manual_seed(61)
    rows, width = 2503, 40
    x = torch.randn(rows, Hq + 2 * Hkv, D, generator=g, device="cuda", dtype=torch.bfloat16)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    seq = torch.arange(rows, device="cuda", dtype=torch.int32) % 5
    slots = torch.arange(rows, device="cuda", dtype=torch.int32) // 5
    tab = torch.randperm(5 * width, generator=g, device="cuda").int().view(5, width)
    w = [torch.randn(*((h, D) if per_head else (D,)), generator=g, device="cuda") for h in (Hq, Hkv)]
    rope, outs, pools = B.Rope(rot, layout=layout), [], []
    for step_rows in (rows, 97):
        pool = torch.zeros(5 * width * Hkv * 2 * 16 * D, dtype=torch.bfloat16, device="cuda")
        st = make_stage([pool], Hq, Hkv, D, 5, width)
        out = torch.empty(rows, Hq, D, dtype=torch.bfloat16, device="cuda")
        for r in range(0, rows, step_rows):
            s = slice(r, min(r + step_rows, rows))
            st.norm_rope_append(0, rope, q[s], k[s], v[s], *w, seq[s], slots[s], slots[s], tab, out[s])
        assert st.poll_error() == B.OPW_OK
        outs.append(out), pools.append(pool)
    assert torch.equal(outs[0], outs[1]) and torch.equal(pools[0], pools[1])


def test_norm_rope_append_skips_and_records_what_it_cannot_place():
    rng = np.random.default_rng(6100)
    Hq, Hkv, D, rows = 8, 2, 64, 5
    tab = np.array([[0, 1], [2, -1], [3, 99]], np.int32)
    seq, slots = np.array([0, 1, 2, 0, 3], np.int32), np.array([0, 16, 20, 32, 0], np.int32)
    pool = rand_bits(rng, oracle.pool_elems(4, Hkv, P, D))
    q, k, v = (dev(rand_bits(rng, (rows, h, D)), True) for h in (Hq, Hkv, Hkv))
    pos = torch.zeros(rows, dtype=torch.int32, device="cuda")
    for layout, rot in (("half", 64), ("interleaved", 64), ("half", 10)):
        d_pool, out = dev(pool, True), torch.zeros_like(q)
        st = make_stage([d_pool], Hq, Hkv, D, 8, 2)
        st.norm_rope_append(0, B.Rope(rot, layout=layout), q, k, v, None, None, dev(seq), dev(slots), pos, dev(tab), out)
        assert st.poll_error() == B.OPW_ERR_BAD_PAGE
        want = step.head_norm(out_to_f64(q), None, 1e-6)                  # position 0 turns by nothing
        check_norm(out_to_f64(out), want, np.abs(want), D, np.zeros(1))
        same = host_bits(d_pool) == pool
        one = np.ones_like(same)
        draft._put_row(one, Hkv, D, 0, 0, np.zeros((Hkv, D)), np.zeros((Hkv, D)))
        assert same[one].all() and not same[~one].all()


def test_norm_rope_append_of_values_that_are_not_finite_stays_in_its_head():
    """Infinities and NaN reach the head they are in, none of the others."""
    Hq, Hkv, D, rows = 8, 2, 128, 4
    x = torch.randn(rows, Hq + 2 * Hkv, D, device="cuda", dtype=torch.bfloat16)
    x[1, 3, 5], x[2, 9, 100], x[3, 0, 64] = float("inf"), float("nan"), float("-inf")
    tab, r = i32([[0]]), torch.arange(rows, device="cuda", dtype=torch.int32)
    for layout, rot in (("half", 128), ("interleaved", 64), ("half", 34)):
        pool = torch.zeros(Hkv * 2 * 16 * D, dtype=torch.bfloat16, device="cuda")
        st, out = make_stage([pool], Hq, Hkv, D, 1, 1), torch.empty(rows, Hq, D, dtype=torch.bfloat16, device="cuda")
        st.norm_rope_append(0, B.Rope(rot, layout=layout), x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], None, None, r * 0, r, r, tab, out)
        fine = torch.isfinite(out).all(-1)
        want = torch.ones_like(fine)
        want[1, 3] = want[3, 0] = False
        assert torch.equal(fine, want)
        k, v = oracle.gather_logical(host_bits(pool), Hkv, P, D, np.array([0]), 0, rows)
        bad = ~np.isfinite(oracle.bf16_bits_to_f64(k)).all(-1)
        assert bad.sum() == 1 and bad[2, 1]


def test_norm_rope_append_refuses():
    Hq, Hkv, D, rows = 8, 2, 64, 3
    pool = torch.zeros(4 * Hkv * 2 * 16 * D, dtype=torch.bfloat16, device="cuda")
    st = make_stage([pool], Hq, Hkv, D, 2, 2)
    rope = B.Rope(64)
    q, k, v = (torch.zeros(rows, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    i = torch.zeros(rows, dtype=torch.int32, device="cuda")
    w = torch.ones(Hq, D, device="cuda")
    tab, out = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.zeros_like(q)
    good = dict(layer=0, rows=rows, rot=64, layout=0, table=rope.table.data_ptr(), q=q.data_ptr(), qs=Hq * D, k=k.data_ptr(), ks=Hkv * D,
                v=v.data_ptr(), vs=Hkv * D, wq=w.data_ptr(), wk=w.data_ptr(), per=0, eps=1e-6, seq=i.data_ptr(), slots=i.data_ptr(),
                pos=i.data_ptr(), num_rows=2, tab=tab.data_ptr(), out=out.data_ptr())
    call = lambda **kw: B.lib().opw_norm_rope_append(st.handle, *{**good, **kw}.values(), None)  # noqa: E731
    for kw in (dict(layer=1), dict(rows=-1), dict(rot=0), dict(rot=63), dict(rot=66), dict(layout=2), dict(table=None), dict(table=good["table"] + 4),
               dict(q=None), dict(out=None), dict(k=None), dict(v=good["v"] + 2), dict(qs=Hq * D - 8), dict(qs=Hq * D + 4), dict(ks=Hkv * D - 8),
               dict(vs=Hkv * D + 1), dict(seq=None), dict(slots=good["slots"] + 2), dict(pos=None), dict(num_rows=0), dict(tab=None),
               dict(out=good["q"], qs=Hq * D + 8), dict(wq=good["wq"] + 4), dict(wk=good["wk"] + 8), dict(per=2), dict(per=-1), dict(eps=0.0),
               dict(eps=-1.0), dict(eps=math.inf), dict(eps=math.nan), dict(out=good["wq"]), dict(out=good["wk"] - 16), dict(out=good["k"])):
        assert call(**kw) == B.OPW_ERR_INVALID_ARG, kw
    assert st.launch_count() == 0 and call(rows=0) == B.OPW_OK and st.launch_count() == 0
    args = (i, i, i, tab, out)
    for bad in ((w[0].half(), None), (w[0, :32], None), (w, w[0]), (w[:2], w[:2]), (None, w), (w[0].cpu(), None)):
        with pytest.raises(ValueError):
            st.norm_rope_append(0, rope, q, k, v, *bad, *args)
    with pytest.raises(ValueError):
        st.norm_rope_append(0, rope, q.float(), k, v, None, None, *args)
    st.norm_rope_append(0, rope, q, k, v, w, w[:Hkv], *args)
    st.norm_rope_append(0, rope, q, k, v, w[0], None, *args)
    assert st.launch_count() == 2


# ---------------------------------------------------------------------------- verification ---

def run_verify(st, target, draft_p, tokens, parents, size, u, distinct=False):
    B_, T = np.asarray(tokens).shape
    path = torch.full((B_, T), 99, dtype=torch.int32, device="cuda")
    took, follows = (torch.full((B_,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
    st.tree_verify(target, draft_p, i32(tokens), i32(parents), i32(size), torch.as_tensor(np.asarray(u, np.float32)).cuda(), path, took, follows,
                   distinct=distinct)
    return path, took, follows


def same_as_oracle(got, target, draft_p, tokens, parents, size, u, draw):
    f = lambda x: None if x is None else x.double().cpu().numpy()  # noqa: E731
    want = step.verify(f(target), f(draft_p), tokens, parents, size, np.asarray(u, np.float32).astype(np.float64), draw)
    for g, w in zip(got, want):
        assert (g.cpu().numpy() == w).all(), (g, w)
    return want


def random_verify(rng, B_, T, V, kind, draw, sharp=3.0):
    x = sharp * rng.standard_normal((B_, T, V))
    y = x + rng.standard_normal((B_, T, V))
    soft = lambda z: np.exp(z - z.max(-1, keepdims=True)) / np.exp(z - z.max(-1, keepdims=True)).sum(-1, keepdims=True)  # noqa: E731
    target, q = (torch.from_numpy(soft(z)).to(kind).cuda() for z in (x, y))
    qn = q.double().cpu().numpy()
    parents, tokens = np.zeros((B_, T), np.int64), np.zeros((B_, T), np.int64)
    for b in range(B_):
        parents[b, 0] = -1
        left = {}
        for i in range(1, T):
            parents[b, i] = up = int(i - 1 - min(i - 1, rng.geometric(0.4) - 1))
            w = left.get(up, qn[b, up])
            if w.sum() <= 0:
                w = np.ones(V)
            tokens[b, i] = x_ = int(rng.choice(V, p=w / w.sum()))
            if draw == "distinct":
                w = w.copy()
                w[x_] = 0.0
                left[up] = w
    size = rng.integers(1, T + 1, size=B_)
    size[0] = T
    return target, None if draw == "certain" else q, tokens, parents, size, rng.random((B_, T))


@pytest.mark.parametrize("V", [1, 2, 7, 33, 128, 1000, 4099, 32000])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("draw", ["again", "distinct", "certain"])
def test_verify_matches_the_oracle(V, kind, draw):
    rng = np.random.default_rng(7000 + V)
    st = small_stage()
    for B_, T in ((1, 1), (1, 64), (37, 5), (5, 17)):
        args = random_verify(rng, B_, T, V, kind, draw)
        got = run_verify(st, *args, distinct=draw == "distinct")
        path, took, _ = same_as_oracle(got, *args, draw)
    assert st.poll_error() == B.OPW_OK and st.launch_count() == 4


@pytest.mark.parametrize("draw", ["again", "distinct", "certain"])
def test_verify_of_many_siblings_that_are_refused(draw):
    """A root with 63 children and a target that the drafter misses: one pass over the vocabulary after the other."""
    rng = np.random.default_rng(7100)
    st = small_stage()
    for kind, V in ((torch.float32, 5003), (torch.bfloat16, 700)):
        target, q, tokens, parents, size, u = random_verify(rng, 6, 64, V, kind, draw, sharp=1.0)
        parents[:, 1:] = 0
        if draw == "distinct":
            for b in range(6):
                w = q[b, 0].double().cpu().numpy()
                tokens[b, 1:] = rng.choice(V, size=63, replace=False, p=w / w.sum())
        u[:, 1:] = 0.9999
        size[:] = [64, 64, 40, 10, 3, 2]
        got = run_verify(st, target, q, tokens, parents, size, u, distinct=draw == "distinct")
        same_as_oracle(got, target, q, tokens, parents, size, u, draw)
    assert st.poll_error() == B.OPW_OK


def test_verify_takes_padded_and_misaligned_rows():
    rng = np.random.default_rng(7200)
    st = small_stage()
    for kind in (torch.float32, torch.bfloat16):
        for V, pad, off, off_q in ((501, 0, 0, 0), (501, 3, 1, 1), (501, 11, 3, 0), (2048, 0, 1, 2), (33, 7, 5, 5), (9000, 1, 0, 0)):
            target, q, tokens, parents, size, u = random_verify(rng, 7, 6, V, kind, "again")
            views = []
            for x, o in ((target, off), (q, off_q)):
                flat = torch.full((7 * 6 * (V + pad) + o + 64,), float("nan"), dtype=kind, device="cuda")   # NaN behind every row
                view = flat[o:o + 7 * 6 * (V + pad)].view(7, 6, V + pad)[..., :V]
                view.copy_(x)
                views.append(view)
            got = run_verify(st, *views, tokens, parents, size, u)
            same_as_oracle(got, target, q, tokens, parents, size, u, "again")
    # a single sequence, node or token: its stride says nothing
    t = torch.rand(3, 1, 5, device="cuda")[::2]
    got = run_verify(st, t, None, [[0], [0]], [[-1], [-1]], [1, 1], [[0.5], [0.2]])
    same_as_oracle(got, t, None, np.zeros((2, 1), int), np.full((2, 1), -1), [1, 1], [[0.5], [0.2]], "certain")
    assert st.poll_error() == B.OPW_OK


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_verify_at_the_ends(kind):
    """Uniforms of 0 and just below 1, distributions of one token, of none, equal ones, negative and NaN entries."""
    st, V, T = small_stage(), 37, 4
    one = torch.zeros(V)
    one[11] = 1.0
    flat = torch.full((V,), 1 / 64)
    tail = torch.zeros(V)
    tail[[3, 36]] = 0.5
    odd = flat.clone()
    odd[[0, 5, 36]] = torch.tensor([float("nan"), -1.0, float("nan")])
    none = torch.zeros(V)
    kinds = [one, flat, tail, odd, none]
    for a in kinds:
        for c in kinds:
            for u in (0.0, 0.5, 1 - 2.0 ** -24):
                target, q = (torch.stack([x] * T).to(kind).cuda()[None].contiguous() for x in (a, c))
                for tokens in ([0, 11, 3, 36], [0, 3, 3, 3], [0, 0, 5, 11]):
                    for parents in ([-1, 0, 0, 0], [-1, 0, 1, 2]):
                        args = (np.array([tokens]), np.array([parents]), [T], [[u] * T])
                        for draw in ("again", "distinct", "certain"):
                            got = run_verify(st, target, None if draw == "certain" else q, *args, distinct=draw == "distinct")
                            same_as_oracle(got, target, None if draw == "certain" else q, *args, draw)
    assert st.poll_error() == B.OPW_OK


def test_verify_inactive_cut_and_bad_nodes():
    rng = np.random.default_rng(7300)
    st, V, T = small_stage(), 100, 5
    target, q, tokens, parents, size, u = random_verify(rng, 6, T, V, torch.float32, "again")
    size[:] = [0, -3, T, T, T, T]
    got = run_verify(st, target, q, tokens, parents, size, u)
    want = same_as_oracle(got, target, q, tokens, parents, size, u, "again")
    assert (want[0][:2] == -1).all() and (want[1][:2] == 0).all() and (want[2][:2] == -1).all() and st.poll_error() == B.OPW_OK
    got2 = run_verify(st, target, q, tokens, parents, np.where(size == T, T + 3, size), u)          # longer than the call: cut, recorded
    assert all(torch.equal(a, b) for a, b in zip(got, got2)) and st.poll_error() == B.OPW_ERR_BAD_PAGE
    for where, value in (("tokens", V), ("tokens", -1), ("tokens", 2 ** 31 - 1), ("parents", 3), ("parents", 4), ("parents", -1), ("parents", 7)):
        tk, pr = tokens.copy(), parents.copy()
        (tk if where == "tokens" else pr)[3, 3] = value
        got = run_verify(st, target, q, tk, pr, size, u)
        pr[3, 3] = 99                                                     # passed over
        same_as_oracle(got, target, q, tk, pr, size, u, "again")
        assert st.poll_error() == B.OPW_ERR_BAD_PAGE
    tokens[:, 0], parents[:, 0] = -5, 77                                  # entries of node 0 are not read
    run_verify(st, target, q, tokens, parents, size, u)
    assert st.poll_error() == B.OPW_OK


@pytest.mark.parametrize("draw", ["again", "distinct", "certain"])
def test_the_first_new_token_is_distributed_as_the_targets(draw):
    """60000 sequences draft two siblings each from the drafter's distribution and verify them: the first new token's counts are those of the
    target, within six standard deviations (a false alarm once in 5e8 per token)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(72)
    n, V, T = 60000, 9, 3
    p = torch.tensor([0.02, 0.3, 0.08, 0.15, 0.2, 0.01, 0.04, 0.1, 0.1], device="cuda")
    q = torch.tensor([0.2, 0.1, 0.1, 0.3, 0.05, 0.05, 0.1, 0.06, 0.04], device="cuda")
    target, drafted = p.expand(n, T, V).contiguous(), q.expand(n, T, V).contiguous()
    tokens = torch.zeros(n, T, dtype=torch.int32, device="cuda")
    if draw == "certain":
        tokens[:, 1:] = torch.tensor([3, 0], device="cuda", dtype=torch.int32)
    else:
        tokens[:, 1:] = torch.multinomial(drafted[:, 0], 2, replacement=draw == "again", generator=g).int()
    parents = torch.tensor([-1, 0, 0], device="cuda", dtype=torch.int32).expand(n, T).contiguous()
    u = torch.rand(n, T, generator=g, device="cuda")
    path, took, follows = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((n, T), n, n))
    st = small_stage()
    st.tree_verify(target, None if draw == "certain" else drafted, tokens, parents, torch.full((n,), T, dtype=torch.int32, device="cuda"), u, path,
                   took, follows, distinct=draw == "distinct")
    first = torch.where(took > 1, tokens.gather(1, path[:, 1:2].clamp(min=0).long())[:, 0], follows)
    counts = torch.bincount(first.long(), minlength=V).double()
    assert ((counts - n * p.double()).abs() <= 6 * (n * p * (1 - p)).double().sqrt()).all()
    assert st.poll_error() == B.OPW_OK and (took > 1).any() and (took == 1).any()


@pytest.mark.parametrize("batch,vocab,kind", [(1, 150001, torch.float32), (9, 70000, torch.bfloat16), (40, 33000, torch.float32)])
@pytest.mark.parametrize("draw", ["again", "distinct", "certain"])
def test_verify_over_many_blocks_a_sequence_captured(batch, vocab, kind, draw):
    rng = np.random.default_rng(7500 + batch)
    st, T = small_stage(), 5
    target, q, tokens, parents, size, u = random_verify(rng, batch, T, vocab, kind, draw, sharp=2.0)
    ints, du = [i32(x) for x in (tokens, parents, size)], torch.zeros(batch, T, device="cuda")
    path, took, follows = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((batch, T), batch, batch))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.tree_verify(target, q, *ints, du, path, took, follows, distinct=draw == "distinct")
    for k in range(3):
        u = rng.random((batch, T)) if k else np.full((batch, T), 0.99999)
        du.copy_(torch.from_numpy(u.astype(np.float32)))
        graph.replay()
        same_as_oracle((path, took, follows), target, q, tokens, parents, size, u, draw)
    assert st.poll_error() == B.OPW_OK


def test_verify_of_the_largest_batch_and_vocabulary():
    rng = np.random.default_rng(7400)
    st = small_stage()
    n = 65535
    p = torch.zeros(n, 1, 3, device="cuda")
    last = torch.from_numpy(rng.integers(0, 3, size=n)).cuda()
    p.scatter_(2, last[:, None, None], 1.0)
    path, took, follows = run_verify(st, p, None, np.zeros((n, 1)), np.full((n, 1), -1), np.ones(n), rng.random((n, 1)))
    assert torch.equal(follows.long(), last) and (took == 1).all() and (path == 0).all()
    V = 1 << 24
    p, q = torch.zeros(1, 2, V, device="cuda"), torch.zeros(1, 2, V, device="cuda")
    p[0, 0, V - 2:], p[0, 1, V - 1], q[0, 0, 5] = 0.5, 1.0, 1.0
    for token, u, want in ((5, (0.4, 0.9), (1, V - 2)), (5, (0.6, 0.0), (1, V - 1)), (V - 1, (0.1, 0.9), (2, V - 1))):
        path, took, follows = run_verify(st, p, q, [[0, token]], [[-1, 0]], [2], [u])
        assert (took.item(), follows.item()) == want
    assert st.poll_error() == B.OPW_OK


def test_verify_refuses():
    st, V, T, n = small_stage(), 64, 4, 3
    target, q = torch.rand(n, T, V, device="cuda"), torch.rand(n, T, V, device="cuda")
    i = torch.zeros(16, n * T, dtype=torch.int32, device="cuda")
    u = torch.zeros(n, T, device="cuda")
    a = [i[k].data_ptr() for k in range(16)]
    good = dict(batch=n, nodes=T, vocab=V, dtype=0, draw=0, target=target.data_ptr(), ts=V, q=q.data_ptr(), qs=V, tokens=a[0], parents=a[1],
                size=a[2], u=u.data_ptr(), path=a[3], took=a[4], follows=a[5])
    call = lambda **kw: B.lib().opw_tree_verify(st.handle, *{**good, **kw}.values(), None)  # noqa: E731
    for kw in (dict(batch=-1), dict(nodes=0), dict(nodes=65), dict(vocab=0), dict(dtype=2), dict(dtype=-1), dict(draw=3), dict(draw=-1), dict(draw=2),
               dict(q=None), dict(q=None, draw=1), dict(target=None), dict(target=good["target"] + 2), dict(q=good["q"] + 1, dtype=1), dict(ts=V - 1),
               dict(qs=V - 1), dict(tokens=None), dict(parents=a[1] + 2), dict(size=None), dict(u=None), dict(path=None), dict(took=a[4] + 1),
               dict(follows=None), dict(path=a[0]), dict(path=a[1] + 4), dict(took=a[2]), dict(follows=a[4]), dict(took=a[3] + 8),
               dict(path=good["target"]), dict(follows=good["q"] + 4 * (V * n * T - 1)), dict(took=good["u"])):
        assert call(**kw) == B.OPW_ERR_INVALID_ARG, kw
    assert call(batch=65536) == B.OPW_ERR_CAPACITY and call(vocab=(1 << 24) + 1, ts=1 << 25, qs=1 << 25) == B.OPW_ERR_CAPACITY
    assert st.launch_count() == 0 and call(batch=0) == B.OPW_OK and st.launch_count() == 0
    ints = (i[0].view(n, T), i[1].view(n, T), i[2, :n].contiguous(), u, i[3].view(n, T), i[4, :n].contiguous(), i[5, :n].contiguous())
    for t, d, kw in ((target.half(), q.half(), {}), (target, q.bfloat16(), {}), (target, q[:, :, :8], {}), (target, None, dict(distinct=True)),
                     (target.transpose(0, 1), q, {}), (target.cpu(), q, {}), (target[0], q[0], {}), (target[:, ::2], q[:, ::2], {})):
        with pytest.raises(ValueError):
            st.tree_verify(t, d, *ints, **kw)
    with pytest.raises(ValueError):
        st.tree_verify(target, q, ints[0].long(), *ints[1:])
    st.tree_verify(target, q, *ints)
    assert st.launch_count() == 1


# ---------------------------------------------------------------------------- pages for requests ---

def run_extend(rows, old, new, table, counts, lst, count, begin=None, room=None, want_starts=True, st=None):
    """The call on copies; returns everything it may write."""
    st = st or small_stage(rows=4, width=table.shape[1])
    tab, refs = i32(table), i32(counts)
    n = len(rows)
    starts, lens, end = (torch.full((k,), -77, dtype=torch.int32, device="cuda") for k in (n + 1, n, 1))
    seq, slots = (None, None) if room is None else (torch.full((room,), -77, dtype=torch.int32, device="cuda") for _ in range(2))
    st.kv_extend(i32(rows), i32(old), i32(new), tab, refs, i32(lst), i32([count]), row_starts=starts if want_starts else None, new_lens=lens, seq=seq,
                 slots=slots, free_begin=None if begin is None else i32([begin]), free_end=end)
    return starts, lens, seq, slots, end, tab, refs, st.poll_error()


def check_extend(rows, old, new, table, counts, lst, count, begin=None, room=None):
    got = run_extend(rows, old, new, table, counts, lst, count, begin, room)
    t, c = np.array(table, np.int64), np.array(counts, np.int64)
    starts, lens, seq, slots, end, recorded = step.extend(rows, old, new, t, c, lst, count, begin or 0, room)
    np_ = lambda x: x.cpu().numpy()  # noqa: E731
    assert (np_(got[0]) == starts).all() and (np_(got[1]) == lens).all() and got[4].item() == end
    if room is not None:
        assert (np_(got[2]) == seq).all() and (np_(got[3]) == slots).all()
    assert (np_(got[5]) == t).all() and (np_(got[6]) == c).all()
    assert got[7] == (B.OPW_ERR_BAD_PAGE if recorded else B.OPW_OK)
    return lens, recorded


def request_state(rng, n, have, width, spare, rows=None):
    rows = rows or n + 3
    row = rng.permutation(rows)[:n]
    pages = [-(-h // P) for h in have]
    total = sum(pages) + spare
    order = rng.permutation(total)
    table, counts, at = np.full((rows, width), -1, np.int64), np.zeros(total, np.int64), 0
    for f in range(n):
        table[row[f], :pages[f]] = order[at:at + pages[f]]
        counts[order[at:at + pages[f]]] = 1
        at += pages[f]
    return row, table, counts, np.sort(order[at:])


@pytest.mark.parametrize("n,longest,spare", [(1, 1, 1), (1, 5000, 400), (3, 40, 2), (31, 100, 60), (32, 1, 32), (33, 17, 5), (257, 80, 700),
                                             (1024, 30, 900), (1100, 3, 5000), (3000, 2, 2000), (8192, 40, 9000)])
@pytest.mark.parametrize("tight", [False, True])
def test_extend_matches_the_oracle(n, longest, spare, tight):
    rng = np.random.default_rng(8000 + n + spare)
    have = rng.integers(0, 90, size=n)
    new = np.where(rng.random(n) < 0.6, 1, rng.integers(0, longest + 1, size=n))
    width = (90 + longest) // P + 2
    row, table, counts, free = request_state(rng, n, have, width, spare + (0 if tight else n * (longest // P + 1)))
    lens, recorded = check_extend(row, have, new, table, counts, free, len(free), room=int(new.sum()) + 37)
    assert not recorded and (tight or (lens == have + new).all())


def test_extend_without_maps_a_cursor_and_lists_longer_than_they_are_given():
    rng = np.random.default_rng(8100)
    have, new = [5, 16, 0, 31, 0], [20, 16, 100, 1, 0]
    row, table, counts, free = request_state(rng, 5, have, 12, 40)
    for begin, count, cut in ((None, 40, 40), (0, 40, 40), (-3, 40, 40), (25, 40, 40), (31, 40, 40), (36, 40, 40), (40, 40, 40), (99, 40, 40),
                              (0, 9, 40), (0, 40, 6), (0, 0, 40), (0, -5, 40)):
        check_extend(row, have, new, table, counts, free[:cut], count, begin=begin)
        check_extend(row, have, new, table, counts, free[:cut], count, begin=begin, room=150)
    # the cursor runs through one list: two calls share it
    st = small_stage(width=12)
    tab, refs, lst, cnt, cur = i32(table), i32(counts), i32(free), i32([40]), i32([0])
    for f in (slice(0, 2), slice(2, 5)):
        st.kv_extend(i32(row[f]), i32(have[f]), i32(new[f]), tab, refs, lst, cnt, free_begin=cur, free_end=cur)
    t, c = table.copy(), counts.copy()
    step.extend(row, have, new, t, c, free, 40)
    assert (tab.cpu().numpy() == t).all() and (refs.cpu().numpy() == c).all() and cur.item() == 9 and st.poll_error() == B.OPW_OK
    # a second time they hold what they need: nothing is dealt
    st.kv_extend(i32(row), i32(have), i32(new), tab, refs, lst, cnt, free_begin=cur, free_end=cur)
    assert (tab.cpu().numpy() == t).all() and cur.item() == 9 and st.poll_error() == B.OPW_OK


def test_extend_refuses_bad_requests_one_by_one():
    rng = np.random.default_rng(8200)
    have, new = [20, 33, 5, 64, 0, 7], [30, 2, 60, 16, 33, 1]
    row, table, counts, free = request_state(rng, 6, have, 10, 30, rows=9)
    base = dict(rows=row, old=np.array(have), new=np.array(new), table=table, counts=counts, lst=free, count=30, room=200)
    lens, bad = check_extend(**base)
    assert not bad and (lens == base["old"] + base["new"]).all()

    def change(key, at, value):
        x = base[key].copy()
        x[at] = value
        return {**base, key: x}

    shared = counts.copy()
    shared[table[row[2], 0]] = 2
    for kw in (change("rows", 1, 9), change("rows", 1, 2 ** 31 - 1), change("rows", 4, row[1]), change("old", 2, -1), change("new", 2, -7),
               change("new", 3, 97), change("new", 3, 2 ** 31 - 1), change("old", 4, 16 * 10), change("table", (row[2], 0), -1),
               change("table", (row[2], 0), 1 << 20), change("table", (row[2], 0), len(counts)), {**base, "counts": shared}, {**base, "room": 141},
               {**base, "room": 60}, {**base, "room": 0}):
        _, bad = check_extend(**kw)
        assert bad, kw
    _, bad = check_extend(**change("rows", 3, -1))                        # idle: not recorded, its rows are padding
    assert not bad
    t = table.copy()
    t[row[0], 3] = free[7]                                                # a page in hand already: kept if it is the request's own
    c = counts.copy()
    c[free[7]] = 1
    check_extend(**{**base, "table": t, "counts": c, "lst": np.delete(free, 7), "count": 29})
    _, bad = check_extend(**{**base, "table": t})                         # (its count says it is free)
    assert bad
    for lst in (np.full(30, free[0]), np.r_[free[:3], -1, 1 << 20, len(counts), free[3:27]]):       # a list that is out of date
        got = run_extend(**{**base, "lst": lst}, want_starts=False)
        assert got[7] == B.OPW_ERR_BAD_PAGE and got[6].max().item() == 1
        held = got[5][got[5] >= 0]
        assert held.unique().numel() == held.numel() and (got[0] == -77).all()


def test_extend_refuses():
    st = small_stage(rows=4, width=3)
    i = torch.zeros(16, 64, dtype=torch.int32, device="cuda")
    a = [i[k].data_ptr() for k in range(16)]
    good = dict(n=4, rows=a[0], old=a[1], new=a[2], num_rows=4, table=a[3], refs=a[4], pages=8, lst=a[5], most=8, count=a[6], begin=a[7], end=a[8],
                starts=a[9], lens=a[10], room=16, seq=a[11], slots=a[12])
    call = lambda **kw: B.lib().opw_kv_extend(st.handle, *{**good, **kw}.values(), None)  # noqa: E731
    for kw in (dict(n=-1), dict(rows=None), dict(old=None), dict(new=a[2] + 2), dict(num_rows=0), dict(table=None), dict(refs=None), dict(pages=0),
               dict(pages=1 << 31), dict(lst=None), dict(most=-1), dict(count=None), dict(begin=a[7] + 1), dict(room=-1), dict(seq=None), dict(slots=None),
               dict(lens=a[1]), dict(starts=a[2]), dict(end=a[6]), dict(seq=a[0]), dict(slots=a[11]), dict(seq=a[3] + 4), dict(starts=a[10]),
               dict(lens=a[4]), dict(begin=a[9]), dict(begin=a[9] + 4), dict(begin=a[3]), dict(table=a[5]), dict(refs=a[5]), dict(end=a[10])):
        assert call(**kw) == B.OPW_ERR_INVALID_ARG, kw
    assert call(n=8193) == B.OPW_ERR_CAPACITY and call(num_rows=(1 << 18) + 1) == B.OPW_ERR_CAPACITY and st.launch_count() == 0
    tab = i[3, :12].view(4, 3)
    ints = [i[k, :4].contiguous() for k in range(3)]
    for kw in (dict(seq=i[11]), dict(row_starts=i[9, :4]), dict(new_lens=i[10, :5]), dict(free_end=i[8, :2]), dict(new_lens=i[10, :4].long())):
        with pytest.raises(ValueError):
            st.kv_extend(*ints, tab, i[4, :8], i[5, :8], i[6, :1], **kw)
    with pytest.raises(ValueError):
        st.kv_extend(ints[0], ints[1][:3], ints[2], tab, i[4, :8], i[5, :8], i[6, :1])
    # no request at all: the maps are all padding
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    seq, slots, starts = (torch.full((k,), 5, dtype=torch.int32, device="cuda") for k in (70, 70, 1))
    st.kv_extend(e, e, e, tab, i[4, :8], i[5, :8], i[6, :1], seq=seq, slots=slots, row_starts=starts)
    assert (seq == -1).all() and (slots == -1).all() and starts.item() == 0 and st.poll_error() == B.OPW_OK


def test_extend_in_a_large_table_of_long_rows():
    """Requests at the ends of a table of 262144 rows, and a prompt of 130000 tokens."""
    width, rows = 8200, 1 << 18
    st = small_stage(width=width)
    tab = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
    refs, lst = torch.zeros(9000, dtype=torch.int32, device="cuda"), torch.randperm(9000, device="cuda").int()
    row, new = i32([rows - 1, 0, rows - 1 - 32]), i32([130001, 1, 17])
    seq, slots = (torch.empty(130030, dtype=torch.int32, device="cuda") for _ in range(2))
    starts = torch.empty(4, dtype=torch.int32, device="cuda")
    st.kv_extend(row, i32([0, 0, 0]), new, tab, refs, lst, i32([9000]), seq=seq, slots=slots, row_starts=starts)
    assert st.poll_error() == B.OPW_OK and starts.tolist() == [0, 130001, 130002, 130019]
    need = [8126, 1, 2]
    assert torch.equal(tab[rows - 1, :8126], lst[:8126]) and (tab[rows - 1, 8126:] == -1).all() and tab[0, 0] == lst[8126]
    assert torch.equal(tab[rows - 33, :2], lst[8127:8129]) and (tab >= 0).sum().item() == sum(need) and refs.sum().item() == sum(need)
    assert torch.equal(slots[:130001], torch.arange(130001, device="cuda").int()) and (seq[:130001] == rows - 1).all()
    assert seq[130001].item() == 0 and (seq[130002:130019] == rows - 33).all() and (seq[130019:] == -1).all()


# ---------------------------------------------------------------------------- streams and graphs ---

def test_the_calls_on_a_side_stream_without_early_launches_and_captured():
    rng = np.random.default_rng(8300)
    st = small_stage(flags=B.OPW_FLAG_NO_PDL)
    side = torch.cuda.Stream()
    target, q, tokens, parents, size, u = random_verify(rng, 5, 6, 777, torch.float32, "again")
    ints = [i32(x) for x in (tokens, parents, size)]
    du = torch.from_numpy(u.astype(np.float32)).cuda()
    path, took, follows = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((5, 6), 5, 5))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        st.tree_verify(target, q, *ints, du, path, took, follows)
    side.synchronize()
    same_as_oracle((path, took, follows), target, q, tokens, parents, size, u, "again")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        st.tree_verify(target, q, *ints, du, path, took, follows)
    for _ in range(3):
        u = rng.random(u.shape)
        du.copy_(torch.from_numpy(u.astype(np.float32)))
        g.replay()
        same_as_oracle((path, took, follows), target, q, tokens, parents, size, u, "again")
    assert st.poll_error() == B.OPW_OK
