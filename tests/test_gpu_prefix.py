"""GPU parity of decode attention behind shared prefixes against the 64-bit oracle, row by row over each row's own page table."""
import numpy as np
import pytest
import torch

import oracle
from helpers import P, out_to_f64, rand_bits
from oracle import draft, step
from paper_2609_14237_b200 import binding as B

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 64), (32, 8, 128), (64, 8, 128), (5, 1, 64), (16, 1, 128), (4, 4, 64), (16, 2, 256), (6, 2, 256)]


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()
    assert torch.cuda.is_available()


def dev(a, bf16=False):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t.view(torch.int16).view(torch.bfloat16) if bf16 else t).cuda()


def i32(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()


def make_stage(pools, Hq, Hkv, D, rows, width, window=0, **kw):
    windows = window if isinstance(window, list) else [window] * len(pools)
    return B.Stage(pools=pools, layer_window=windows, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, max_batch=rows, max_pages_per_seq=width, **kw)


def shared_batch(rng, sizes, prefix, lens, Hq, Hkv, D, spare=2, width=None):
    """A cache of random rows: each group's first whole pages of its prefix held by all of its members."""
    starts = np.concatenate([[0], np.cumsum(sizes)])
    n = int(starts[-1])
    pages = [max(-(-x // P), 0) for x in lens]
    width = width or max(max(pages), 1) + 1
    total = sum(pages) + sum(x // P for x in prefix) + spare
    order = rng.permutation(total)
    tab, at = np.full((n, width), -1, np.int32), 0
    for g, pre in enumerate(prefix):
        members = range(starts[g], starts[g + 1])
        whole = pre // P
        mine = order[at:at + whole]
        at += whole
        for b in members:
            k = min(whole, pages[b])
            tab[b, :k] = mine[:k]
            tab[b, k:pages[b]] = order[at:at + pages[b] - k]
            at += pages[b] - k
    pool = rand_bits(rng, oracle.pool_elems(total, Hkv, P, D))
    q = rand_bits(rng, (n, Hq, D))
    return pool, tab, q, starts


def run(pool, tab, q, lens, starts, prefix, Hq, Hkv, D, window=0, scale=0.0, **kw):
    st = make_stage([dev(pool, True)], Hq, Hkv, D, len(lens), tab.shape[1], window, softmax_scale=scale, **kw)
    pre = B.PrefixAttention(st)
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:2], float("nan"), dtype=torch.float32, device="cuda")
    pre.attention(0, dev(q, True), i32(lens), i32(starts), i32(prefix), dev(tab), out, lse)
    rc = st.poll_error()
    assert st.launch_count() == 2
    pre.close()
    st.close()
    return out, lse, rc


def check(out, lse, ref, n):
    """Counted in roundings (half a step of bf16 is 2^-8 of the value, of fp32 2^-24):
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


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("sizes", [[1], [2, 1, 0, 3, 1], [4, 4], [13], [40, 1, 3]])
@pytest.mark.parametrize("window", [0, 37, 300])
def test_matches_the_oracle(Hq, Hkv, D, sizes, window):
    """Groups of any size; members longer than the prefix, just as long, shorter, empty and inactive; prefixes of no page, inside a
    page, and over several tiles."""
    rng = np.random.default_rng(9000 + Hq + D + len(sizes) + window)
    prefix = [int(rng.choice([0, 5, 16, 33, 64, 200, 337])) if len(sizes) > 2 else 337 for _ in sizes]
    lens = []
    for s, pre in zip(sizes, prefix):
        choice = [pre + 1, pre + 40, pre, pre // P * P, max(pre - 3, 0), pre // 2, 1, 0, -2, pre + 130, pre + 16]
        lens += [pre + 70] + [int(rng.choice(choice)) for _ in range(s - 1)] if s else []
    pool, tab, q, starts = shared_batch(rng, sizes, prefix, lens, Hq, Hkv, D)
    out, lse, rc = run(pool, tab, q, lens, starts, prefix, Hq, Hkv, D, window)
    assert rc == B.OPW_OK
    check(out, lse, step.decode_attention(pool, Hq, Hkv, D, q, lens, tab, window), 500)
    gone = np.array(lens) <= 0
    assert (out_to_f64(out)[gone] == 0).all()


@pytest.mark.parametrize("Hq,Hkv,D,members", [(32, 8, 128, 5), (32, 8, 128, 40), (64, 8, 128, 37), (8, 2, 64, 70), (8, 2, 64, 9), (6, 2, 256, 11),
                                              (16, 1, 128, 33)])
@pytest.mark.parametrize("window", [0, 90, 1500])
def test_long_prefixes_split_over_workers(Hq, Hkv, D, members, window):
    rng = np.random.default_rng(9100 + D + members + window)
    sizes, prefix = [members, 2, members // 2], [2085, 700, 1300]
    lens = [int(prefix[g] + rng.integers(1, 400)) for g, s in enumerate(sizes) for _ in range(s)]
    lens[1] = 1000                                            # one row ends inside the shared part
    pool, tab, q, starts = shared_batch(rng, sizes, prefix, lens, Hq, Hkv, D)
    out, lse, rc = run(pool, tab, q, lens, starts, prefix, Hq, Hkv, D, window)
    assert rc == B.OPW_OK
    check(out, lse, step.decode_attention(pool, Hq, Hkv, D, q, lens, tab, window), 2600)
    # the same again, and with other physical pages: the same bits
    out2, lse2, _ = run(pool, tab, q, lens, starts, prefix, Hq, Hkv, D, window)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    total = pool.size // (Hkv * 2 * P * D)
    moved = rng.permutation(total).astype(np.int32)
    pool3, tab3 = np.empty_like(pool).reshape(total, -1), np.where(tab >= 0, moved[np.maximum(tab, 0)], tab)
    pool3[moved] = pool.reshape(total, -1)
    out3, lse3, _ = run(pool3.reshape(-1), tab3, q, lens, starts, prefix, Hq, Hkv, D, window)
    assert torch.equal(out, out3) and torch.equal(lse, lse3)


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (32, 8, 128), (6, 2, 256)])
@pytest.mark.parametrize("members", [2, 9, 45])
@pytest.mark.parametrize("window", [0, 50])
def test_what_a_row_does_not_see_may_hold_anything(Hq, Hkv, D, members, window):
    """NaN and infinities behind the rows' ends, before their windows, and in shared keys that only the longer rows see."""
    rng = np.random.default_rng(9200 + D + members)
    prefix = [150]
    lens = [150 + int(x) for x in rng.integers(1, 30, size=members)]
    lens[0], lens[-1] = 101, 170                              # the first row sees shared keys 0 .. 100
    pool, tab, q, starts = shared_batch(rng, [members], prefix, lens, Hq, Hkv, D)
    tab[0] = np.where(np.arange(tab.shape[1]) < 7, tab[1], -1)
    clean = step.decode_attention(pool, Hq, Hkv, D, q, lens, tab, window)
    junk = np.array([0x7FC0, 0x7F80, 0xFF80, 0xFFFF], np.uint16)
    row = lambda: (junk[rng.integers(0, 4, size=(Hkv, D))], junk[rng.integers(0, 4, size=(Hkv, D))])  # noqa: E731
    for b in range(members):
        for s in range(lens[b], (tab[b] >= 0).sum() * P):
            if s >= 144:                                      # its own last page
                draft._put_row(pool, Hkv, D, tab[b, s // P], s % P, *row())
    if window:
        for s in range(0, 101 - window):                      # before every row's window
            draft._put_row(pool, Hkv, D, tab[1, s // P], s % P, *row())
    out, lse, rc = run(pool, tab, q, lens, [0, members], prefix, Hq, Hkv, D, window)
    assert rc == B.OPW_OK
    check(out, lse, clean, 300)
    # an infinity and a NaN among the values of shared key 130, which all rows but the first see (unless their windows begin behind it)
    k, v = oracle.gather_logical(pool, Hkv, P, D, tab[1], 130, 131)
    v[0, 0, 3], v[0, Hkv - 1, D - 1] = 0x7F80, 0x7FC0
    draft._put_row(pool, Hkv, D, tab[1, 130 // P], 130 % P, k[0], v[0])
    ref = step.decode_attention(pool, Hq, Hkv, D, q, lens, tab, window)
    assert np.isnan(ref[0]).any() and np.isfinite(ref[0][0]).all()
    out, lse, rc = run(pool, tab, q, lens, [0, members], prefix, Hq, Hkv, D, window)
    check(out, lse, ref, 300)
    # and a key of NaN
    draft._put_row(pool, Hkv, D, tab[1, 130 // P], 130 % P, np.full((Hkv, D), 0x7FC0, np.uint16), rand_bits(rng, (Hkv, D)))
    out, lse, rc = run(pool, tab, q, lens, [0, members], prefix, Hq, Hkv, D, window)
    got, got_lse = out_to_f64(out), lse.cpu().numpy()
    for b in range(members):
        hit = lens[b] > 130 and (not window or 130 >= lens[b] - window)
        assert np.isnan(got[b]).all() == hit and np.isnan(got_lse[b]).all() == hit and (hit or np.isfinite(got[b]).all())


@pytest.mark.parametrize("Hq,Hkv,D,members", [(32, 8, 128, 3), (32, 8, 128, 12), (8, 2, 64, 50), (6, 2, 256, 7)])
def test_only_the_longest_rows_entries_are_read_for_the_prefix(Hq, Hkv, D, members):
    rng = np.random.default_rng(9300 + D)
    lens = [200 + 3 * b for b in range(members)]
    pool, tab, q, starts = shared_batch(rng, [members], [190], lens, Hq, Hkv, D)
    good = run(pool, tab, q, lens, starts, [190], Hq, Hkv, D)
    tab[:-1, :190 // P] = -1                                  # (a server that keeps the prefix's pages with one row)
    out, lse, rc = run(pool, tab, q, lens, starts, [190], Hq, Hkv, D)
    assert rc == B.OPW_OK and torch.equal(out, good[0]) and torch.equal(lse, good[1])
    out, lse, rc = run(pool, tab, q, lens, starts, [0], Hq, Hkv, D)          # without the prefix they count, and are recorded
    assert rc == B.OPW_ERR_BAD_PAGE and torch.isfinite(out).all()


@pytest.mark.parametrize("Hq,Hkv,D,members", [(32, 8, 128, 2), (32, 8, 128, 12), (8, 2, 64, 70)])
def test_bad_pages_starts_and_lengths_are_masked_and_recorded(Hq, Hkv, D, members):
    rng = np.random.default_rng(9400 + D)
    lens = [180 + b % 20 for b in range(2 * members)]
    pool, tab, q, starts = shared_batch(rng, [members, members], [150, 170], lens, Hq, Hkv, D)
    ref = step.decode_attention(pool, Hq, Hkv, D, q, lens, tab)
    good, good_lse, rc = run(pool, tab, q, lens, starts, [150, 170], Hq, Hkv, D)
    assert rc == B.OPW_OK
    n = 2 * members
    for wrong in ([0, members, n - 1], [1, members, n], [0, n, members], [0, -5, n], [0, n + 9, n], [0, members, n + 1], [0, members, 1 << 30]):
        out, lse, rc = run(pool, tab, q, lens, wrong, [150, 170], Hq, Hkv, D)
        assert rc == B.OPW_ERR_BAD_PAGE
        check(out, lse, ref, 300)
    for pre in ([-7, 170], [150, 1 << 30], [-(1 << 31), (1 << 31) - 1]):     # shared as far as the rows go; nothing is
        tab2 = tab.copy()
        lens2 = lens[:members] + [170 // P * P] * members if pre[1] > 1000 else lens
        out, lse, rc = run(pool, tab2, q, lens2, starts, pre, Hq, Hkv, D)
        assert rc == B.OPW_OK
        check(out, lse, step.decode_attention(pool, Hq, Hkv, D, q, lens2, tab2), 300)
    bad = tab.copy()
    bad[:members, 3] = 1 << 20                                               # a shared page of the first group
    bad[n - 1, 11] = -1                                                      # one of the last row's own
    out, lse, rc = run(pool, bad, q, lens, starts, [150, 170], Hq, Hkv, D)
    assert rc == B.OPW_ERR_BAD_PAGE and torch.equal(out[members:n - 1], good[members:n - 1]) and torch.isfinite(out).all()
    for b in (0, members - 1, n - 1):                                        # as if those sixteen keys were not there
        hole = 3 if b < members else 11
        keep = [s for s in range(lens[b]) if s // P != hole]
        k, v = oracle.gather_logical(pool, Hkv, P, D, tab[b], 0, lens[b])
        pool2 = rand_bits(rng, oracle.pool_elems(16, Hkv, P, D))
        tab2 = np.arange(16, dtype=np.int32)[None]
        draft.append_rows(pool2, Hkv, D, [0] * len(keep), np.arange(len(keep)), tab2, k[keep], v[keep])
        check(out[b:b + 1], lse[b:b + 1], step.decode_attention(pool2, Hq, Hkv, D, q[b:b + 1], [len(keep)], tab2), 300)
    cut = lens.copy()
    cut[0], cut[n - 1] = tab.shape[1] * P + 5, (1 << 31) - 1                 # beyond the table
    full = np.where(tab < 0, 0, tab)
    out, lse, rc = run(pool, full, q, cut, starts, [150, 170], Hq, Hkv, D)
    assert rc == B.OPW_ERR_BAD_PAGE
    at = [min(x, tab.shape[1] * P) for x in cut]
    check(out, lse, step.decode_attention(pool, Hq, Hkv, D, q, at, full), 300)


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (32, 8, 128), (4, 1, 256)])
def test_the_largest_batch_and_number_of_groups(Hq, Hkv, D):
    rng = np.random.default_rng(9500 + D)
    n, groups = B.OPW_PREFIX_MAX_BATCH, B.OPW_PREFIX_MAX_GROUPS
    for sizes in ([2] * groups, [n - groups + 1] + [1] * (groups - 1), [n], [1000, 1048]):
        pages = 200
        prefix = [int(x) for x in rng.integers(0, 60, size=len(sizes))]
        lens = np.concatenate([np.full(s, pre) for s, pre in zip(sizes, prefix)]) + rng.integers(0, 40, size=n)
        starts = np.concatenate([[0], np.cumsum(sizes)])
        tab = rng.integers(0, pages, size=(n, 8)).astype(np.int32)
        for g, pre in enumerate(prefix):
            tab[starts[g]:starts[g + 1], :pre // P] = tab[starts[g], :pre // P]
        pool = rand_bits(rng, oracle.pool_elems(pages, Hkv, P, D))
        q = rand_bits(rng, (n, Hq, D))
        out, lse, rc = run(pool, tab, q, lens, starts, prefix, Hq, Hkv, D)
        assert rc == B.OPW_OK
        pick = np.unique(np.concatenate([[0, 1, n - 1], rng.integers(0, n, size=40)]))
        ref = step.decode_attention(pool, Hq, Hkv, D, q[pick], lens[pick], tab[pick])
        check(out[dev(pick)], lse[dev(pick)], ref, 120)


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (32, 8, 128), (6, 2, 256), (16, 1, 128)])
def test_one_large_group_among_single_rows(Hq, Hkv, D):
    rng = np.random.default_rng(9550 + D)
    sizes = [1] * 9 + [70] + [1] * 12
    prefix = [int(x) for x in rng.integers(0, 200, size=len(sizes))]
    prefix[9] = 777
    lens = [int(prefix[g] + rng.integers(1, 90)) for g, s in enumerate(sizes) for _ in range(s)]
    pool, tab, q, starts = shared_batch(rng, sizes, prefix, lens, Hq, Hkv, D)
    for window in (0, 300):
        out, lse, rc = run(pool, tab, q, lens, starts, prefix, Hq, Hkv, D, window)
        assert rc == B.OPW_OK
        check(out, lse, step.decode_attention(pool, Hq, Hkv, D, q, lens, tab, window), 900)


@pytest.mark.parametrize("Hq,Hkv,D,members", [(32, 8, 128, 33), (8, 2, 64, 20), (16, 2, 256, 4)])
@pytest.mark.parametrize("shape", ["rise", "fall", "alternate"])
def test_scores_that_rise_and_fall_along_the_keys(Hq, Hkv, D, members, shape):
    """Maxima that move within the prefix and behind it: keys along the first dimension, a query that looks there."""
    rng = np.random.default_rng(9600 + D + members)
    pre, lens = 1024, [1024 + 9 * b + 1 for b in range(members)]
    pool, tab, q, starts = shared_batch(rng, [members], [pre], lens, Hq, Hkv, D)
    n = max(lens)
    ramp = {"rise": np.linspace(-60, 60, n), "fall": np.linspace(60, -60, n), "alternate": 50 * (-1.0) ** (np.arange(n) // 64)}[shape]
    for b in range(members):
        lo = 0 if b == 0 else pre
        k, v = oracle.gather_logical(pool, Hkv, P, D, tab[b], lo, lens[b])
        k = k.copy()
        k[:, :, 0] = oracle.f32_to_bf16_bits(ramp[lo:lens[b], None].astype(np.float32))
        draft.append_rows(pool, Hkv, D, [b] * (lens[b] - lo), np.arange(lo, lens[b]), tab, k, v)
    q[:, :, 0] = oracle.f32_to_bf16_bits(np.full(1, 2.0 * np.sqrt(D) / 4, np.float32))[0]
    for scale in (0.0, 0.7):
        out, lse, rc = run(pool, tab, q, lens, starts, [pre], Hq, Hkv, D, scale=scale)
        assert rc == B.OPW_OK
        check(out, lse, step.decode_attention(pool, Hq, Hkv, D, q, lens, tab, scale=scale or None), 1400)


def test_layers_of_their_own_and_the_decode_step_agree():
    """Two layers with windows and pools of their own in one handle; without groups the call is decode attention."""
    rng = np.random.default_rng(9700)
    Hq, Hkv, D, sizes, prefix = 32, 8, 128, [6, 5, 9], [300, 40, 100]
    lens = [int(prefix[g] + rng.integers(1, 90)) for g, s in enumerate(sizes) for _ in range(s)]
    pool, tab, q, starts = shared_batch(rng, sizes, prefix, lens, Hq, Hkv, D)
    pool2 = rand_bits(rng, pool.shape)
    st = make_stage([dev(pool, True), dev(pool2, True)], Hq, Hkv, D, len(lens), tab.shape[1], [0, 64])
    pre = B.PrefixAttention(st)
    dq, dl, dt = dev(q, True), i32(lens), dev(tab)
    for layer, (x, w) in enumerate(((pool, 0), (pool2, 64))):
        ref = step.decode_attention(x, Hq, Hkv, D, q, lens, tab, w)
        out, lse, o2, l2 = (torch.empty(s, dtype=t, device="cuda") for s, t in ((q.shape, torch.bfloat16), (q.shape[:2], torch.float32)) * 2)
        for s, p in ((starts, prefix), (list(range(len(lens) + 1)), [999] * len(lens)), ([0, len(lens)], [0])):
            pre.attention(layer, dq, dl, i32(s), i32(p), dt, out, lse)
            check(out, lse, ref, 400)
            pre.attention(layer, dq, dl, i32(s), i32(p), dt, o2)             # no lse asked for
            assert torch.equal(out, o2)
        st.decode_attention(layer, dq, dl, dt, o2, l2)
        check(o2, l2, ref, 400)
    assert st.poll_error() == B.OPW_OK


@pytest.mark.parametrize("flags", [0, B.OPW_FLAG_NO_PDL])
@pytest.mark.parametrize("Hq,Hkv,D", [(32, 8, 128), (8, 2, 64), (6, 2, 256)])
def test_in_a_graph_on_another_stream_with_lengths_and_groups_changed(Hq, Hkv, D, flags):
    rng = np.random.default_rng(9800 + D)
    n, width, pages = 24, 30, 400
    pool = rand_bits(rng, oracle.pool_elems(pages, Hkv, P, D))
    st = make_stage([dev(pool, True)], Hq, Hkv, D, n, width, flags=flags)
    pre = B.PrefixAttention(st)
    q, lens, starts, prefix = dev(rand_bits(rng, (n, Hq, D)), True), i32([0] * n), i32([0, 8, 16, n]), i32([0] * 3)
    tab = torch.zeros(n, width, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(n, Hq, device="cuda")
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        pre.attention(0, q, lens, starts, prefix, tab, out, lse)
        pre.attention(0, q, lens, starts, prefix, tab, out, lse)             # one after the other in one workspace
    for sizes in ([8, 8, 8], [24, 0, 0], [1, 20, 3], [0, 2, 22]):
        s = np.concatenate([[0], np.cumsum(sizes)])
        pr = rng.integers(0, 350, size=3)
        ln = np.concatenate([np.full(k, x) for k, x in zip(sizes, pr)]) + rng.integers(-20, 100, size=n)
        t = rng.integers(0, pages, size=(n, width)).astype(np.int32)
        for k in range(3):
            t[s[k]:s[k + 1], :pr[k] // P] = t[min(s[k], n - 1), :pr[k] // P]
        lens.copy_(i32(ln)), starts.copy_(i32(s)), prefix.copy_(i32(pr)), tab.copy_(dev(t))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        side.synchronize()
        bits = q.cpu().view(torch.int16).numpy().view(np.uint16)
        check(out, lse, step.decode_attention(pool, Hq, Hkv, D, bits, ln, t), 500)
        o2, l2 = torch.empty_like(out), torch.empty_like(lse)
        pre.attention(0, q, lens, starts, prefix, tab, o2, l2)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
    assert st.poll_error() == B.OPW_OK


def test_handles_of_their_own_run_side_by_side():
    rng = np.random.default_rng(9900)
    Hq, Hkv, D = 32, 8, 128
    lens = [2000 + 10 * b for b in range(20)]
    pool, tab, q, starts = shared_batch(rng, [20], [1900], lens, Hq, Hkv, D)
    st = make_stage([dev(pool, True)], Hq, Hkv, D, 20, tab.shape[1])
    args = (dev(q, True), i32(lens), i32(starts), i32([1900]), dev(tab))
    want, want_lse = torch.empty_like(args[0]), torch.empty(20, Hq, device="cuda")
    first = B.PrefixAttention(st)
    first.attention(0, *args, want, want_lse)
    handles, streams = [first, B.PrefixAttention(st)], [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [[torch.empty_like(want) for _ in range(20)] for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        for h, s, o in zip(handles, streams, outs):
            with torch.cuda.stream(s):
                h.attention(0, *args, o[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for os in outs for o in os) and st.poll_error() == B.OPW_OK


def test_refuses():
    Hq, Hkv, D, n, groups = 8, 2, 64, 4, 2
    pool = torch.zeros(4 * Hkv * 2 * 16 * D, dtype=torch.bfloat16, device="cuda")
    st = make_stage([pool], Hq, Hkv, D, n, 3)
    pre = B.PrefixAttention(st)
    q, out, lse = torch.zeros(n, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, Hq, device="cuda")
    i = torch.zeros(8, 16, dtype=torch.int32, device="cuda")
    a = [i[k].data_ptr() for k in range(8)]
    good = dict(layer=0, batch=n, groups=groups, q=q.data_ptr(), lens=a[0], starts=a[1], prefix=a[2], tab=a[3], out=out.data_ptr(), lse=lse.data_ptr())
    call = lambda **kw: B.lib().opw_prefix_attention(pre.handle, *{**good, **kw}.values(), None)  # noqa: E731
    for kw in (dict(layer=1), dict(layer=-1), dict(batch=-1), dict(groups=0), dict(q=None), dict(q=good["q"] + 8), dict(lens=None), dict(lens=a[0] + 2),
               dict(starts=None), dict(prefix=None), dict(prefix=a[2] + 1), dict(tab=None), dict(out=None), dict(out=good["out"] + 2), dict(lse=good["lse"] + 1),
               dict(out=good["q"]), dict(out=good["q"] + 16), dict(lse=good["q"] + 64), dict(lse=good["out"]), dict(lse=a[0]), dict(lse=a[1]),
               dict(lse=a[2] - 4), dict(lse=a[3] + 4)):
        assert call(**kw) == B.OPW_ERR_INVALID_ARG, kw
    assert call(batch=n + 1) == B.OPW_ERR_CAPACITY and call(groups=B.OPW_PREFIX_MAX_GROUPS + 1) == B.OPW_ERR_CAPACITY
    assert st.launch_count() == 0 and call(batch=0) == B.OPW_OK and st.launch_count() == 0
    L, h = B.lib(), B.ctypes.c_void_p()
    size = B.opw_prefix_attn_workspace_bytes(st.handle)
    for ws, nbytes, flags, want in ((0, size, 0, B.OPW_ERR_INVALID_ARG), (256, size - 1, 0, B.OPW_ERR_CAPACITY), (260, size, 0, B.OPW_ERR_INVALID_ARG),
                                    (256, size, 1, B.OPW_ERR_INVALID_ARG)):
        assert L.opw_prefix_attn_create(st.handle, flags, ws, nbytes, B.ctypes.byref(h)) == want and h.value is None
    starts, prefix, tab = i[1, :3], i[2, :2], i[3, :12].view(4, 3)
    args = (i[0, :4], starts, prefix, tab, out, lse)
    for k, bad in ((0, i[0, :3]), (0, i[0, :4].long()), (1, i[1, :2]), (3, tab[:3]), (3, tab[:, :2]), (4, out[:2]), (4, out.float()), (5, lse[:2]), (0, i[0, :4].cpu())):
        with pytest.raises(ValueError):
            pre.attention(0, q, *[bad if j == k else x for j, x in enumerate(args)])
    for bad in (q[:, :4], q.float(), q.transpose(0, 1), q.view(n, Hq * D)):
        with pytest.raises(ValueError):
            pre.attention(0, bad, *args)
    assert st.launch_count() == 0
    wide = make_stage([pool], Hq, Hkv, D, 1, 2 ** 27 - 1)
    assert B.opw_prefix_attn_workspace_bytes(wide.handle) == 0
    with pytest.raises(B.OpwError):
        B.PrefixAttention(wide)
    st.close()
    with pytest.raises(ValueError):
        pre.attention(0, q, *args)


def test_contexts_at_the_end_of_32_bits():
    """A table of 2^27 - 16 pages a row, almost all of them before the window: the last keys of two rows that share a prefix of 2^31 - 336
    tokens (their window reaches into it)."""
    Hq, Hkv, D, width, window = 8, 2, 64, (1 << 27) - 16, 100
    rng = np.random.default_rng(9950)
    pool = rand_bits(rng, oracle.pool_elems(40, Hkv, P, D))
    tab = torch.full((2, width), -1, dtype=torch.int32, device="cuda")
    end = width * P
    pre_pages = width - 5
    ids = rng.permutation(40).astype(np.int32)
    tab[:, pre_pages - 8:pre_pages] = dev(ids[:8])
    tab[0, pre_pages:], tab[1, pre_pages:] = dev(ids[8:13]), dev(ids[13:18])
    lens = [end, end - 37]
    q = rand_bits(rng, (2, Hq, D))
    st = make_stage([dev(pool, True)], Hq, Hkv, D, 2, width, window)
    pre = B.PrefixAttention(st)
    out, lse = torch.empty(2, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(2, Hq, device="cuda")
    pre.attention(0, dev(q, True), i32(lens), i32([0, 2]), i32([pre_pages * P]), tab, out, lse)
    assert st.poll_error() == B.OPW_OK
    small = np.stack([np.r_[ids[:8], ids[8:13]], np.r_[ids[:8], ids[13:18]]])
    cut = (pre_pages - 8) * P
    check(out, lse, step.decode_attention(pool, Hq, Hkv, D, q, [x - cut for x in lens], small, window), 200)
