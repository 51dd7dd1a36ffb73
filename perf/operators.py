"""Cases of the operators that verify drafted tokens on the stage and keep the pages of its cache.

tree     attention of a tree of drafted tokens over the paged cache (one pass of one layer)
rope     rotary encoding of new tokens' queries and keys, keys and values appended to the paged cache
commit   the accepted path's cached rows moved together behind the committed context
fork     a sequence's cached prefix handed to another row of the page table: whole pages shared, the tokens of a last partial one copied
release  rows forked at a page boundary and dropped again, then the list of the pages that nobody holds
"""
import math

import numpy as np
import torch

own = False

PAGE = 16


# ---------------------------------------------------------------------------------- cases ---

def listed():
    return [
        # a chain of four drafted tokens of one sequence: the smallest call a server makes, latency only
        dict(name="tree chain of 4, 1 seq", op="tree", batch=1, nodes=4, shape="chain", ctx_lo=1000, ctx_hi=1000,
             heads=32, kv_heads=8, dim=128, window=0),
        # the middle: 64 sequences of 1k to 4k tokens with small ragged trees
        dict(name="tree of 8, 64 seqs", op="tree", batch=64, nodes=8, shape="tree", ctx_lo=1024, ctx_hi=4096,
             heads=32, kv_heads=8, dim=128, window=0),
        # the largest: full trees of 64 over long contexts
        dict(name="tree of 64, 16 x 32k", op="tree", batch=16, nodes=64, shape="full", ctx_lo=32768, ctx_hi=32768,
             heads=32, kv_heads=8, dim=128, window=0),
        # a sliding-window layer of a hybrid stack, odd tree sizes, contexts far longer than the window
        dict(name="tree of 26, window 4096", op="tree", batch=32, nodes=26, shape="tree", ctx_lo=8192, ctx_hi=65536,
             heads=32, kv_heads=8, dim=128, window=4096),
        # the drafted tokens of 16 trees before their attention
        dict(name="rope 16 trees of 8", op="rope", rows=128, seqs=16, packed=False, layout="half", rotary=128,
             scaling="plain", far=4096, heads=32, kv_heads=8, dim=128),
        # prompts of together 8192 tokens entering the cache, straight from the packed projection, long-context scaling
        dict(name="rope prompts, 8192 tokens", op="rope", rows=8192, seqs=7, packed=True, layout="interleaved", rotary=64,
             scaling="yarn", far=1000000, heads=32, kv_heads=8, dim=128),
        # one sequence accepts a part of its chain
        dict(name="commit 1 seq", op="commit", batch=1, nodes=4, ctx_lo=1000, ctx_hi=1000, layers=1, kv_heads=8, dim=128),
        # every sequence of a batch after a step with full trees, the whole hybrid stack in one call
        dict(name="commit 64 seqs, 8 layers", op="commit", batch=64, nodes=64, ctx_lo=100, ctx_hi=1000, layers=8, kv_heads=8,
             dim=128),
        # a prompt sampled four times
        dict(name="fork 1 to 4", op="fork", parents=1, children=4, len_lo=1000, len_hi=1000, layers=1, kv_heads=8, dim=128),
        # beams of a batch, the whole stack
        dict(name="fork 32 to 256, 8 layers", op="fork", parents=32, children=256, len_lo=100, len_hi=1000, layers=8, kv_heads=8,
             dim=128),
        # a few short branches dropped
        dict(name="release 8 rows", op="release", parents=2, children=8, len_lo=256, len_hi=1024, layers=1, kv_heads=2, dim=64),
        # a batch of long branches dropped
        dict(name="release 128 long rows", op="release", parents=16, children=128, len_lo=16384, len_hi=32768, layers=1,
             kv_heads=2, dim=64),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "rope", "commit", "fork", "release"])
    heads, kv_heads, dim = rng.choice([(32, 8, 128), (32, 8, 128), (64, 8, 128), (8, 2, 64), (32, 16, 128), (16, 1, 128), (5, 1, 64),
                                       (24, 2, 64), (16, 2, 256)])
    if op == "tree":
        window = rng.choice([0, 0, 0, 40, 1024, 4096])
        batch, nodes = _log(rng, 1, 64), _log(rng, 1, 64)
        hi = _log(rng, 1, 65536)
        # keys that a pass reads, and scores that it computes: no more than the largest listed case
        span = (min(hi, window) if window else hi) + nodes
        while batch > 1 and (batch * span * kv_heads * dim > 16 * 32832 * 1024 or batch * span * nodes * heads > 16 * 32832 * 64 * 32):
            batch = batch // 2
        if span * nodes * heads * batch > 16 * 32832 * 64 * 32:
            nodes = max(1, nodes // 4)
        return dict(op=op, batch=batch, nodes=nodes, shape=rng.choice(["tree", "chain", "full"]), ctx_lo=rng.randint(0, hi), ctx_hi=hi,
                    heads=heads, kv_heads=kv_heads, dim=dim, window=window)
    if op == "rope":
        rows = _log(rng, 1, 8192 * 32 * 128 // max(heads * dim, 4096))
        rotary = rng.choice([dim, dim, dim // 2, dim // 4, dim // 4 + 2])
        return dict(op=op, rows=rows, seqs=rng.randint(1, min(rows, 64)), packed=rng.random() < 0.5,
                    layout=rng.choice(["half", "interleaved"]), rotary=rotary,
                    scaling=rng.choice(["plain", "linear", "ntk", "bands", "yarn"]), far=_log(rng, 8192, 1000000),
                    heads=heads, kv_heads=kv_heads, dim=dim)
    if op == "commit":
        hi = _log(rng, 1, 1000)
        return dict(op=op, batch=_log(rng, 1, 64), nodes=_log(rng, 1, 64), ctx_lo=rng.randint(0, hi), ctx_hi=hi,
                    layers=rng.randint(1, 8), kv_heads=min(kv_heads, 8), dim=dim)
    children = _log(rng, 1, 256 if op == "fork" else 128)
    hi = _log(rng, 17, 1000 if op == "fork" else 32768)
    return dict(op=op, parents=rng.randint(1, min(32, children)), children=children, len_lo=rng.randint(1, hi), len_hi=hi,
                layers=rng.randint(1, 8) if op == "fork" else 1, kv_heads=min(kv_heads, 8) if op == "fork" else 2,
                dim=dim if op == "fork" else 64)


# --------------------------------------------------------------------------------- inputs ---

def _lens(rng, lo, hi, n):
    lens = rng.integers(lo, hi + 1, size=n)
    lens[0] = hi
    return lens.astype(np.int64)


def _tables(rng, pages_of, width, total):
    """A random page table with pages_of[b] of `total` physical pages in row b, -1 behind them; and the pages left over."""
    order = rng.permutation(total).astype(np.int32)
    table = np.full((len(pages_of), width), -1, dtype=np.int32)
    at = 0
    for b, c in enumerate(pages_of):
        table[b, :c] = order[at:at + c]
        at += int(c)
    return table, order[at:]


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _tree(rng, kind, nodes):
    """Parents of one sequence's drafted tokens, each before its children; -1: the last committed token."""
    if kind == "chain":
        return [i - 1 for i in range(nodes)]
    # drafters extend a few likely branches: recent nodes get most of the children
    return [-1] + [int(i - 1 - min(i, rng.geometric(0.3))) if i > 2 else -1 + int(rng.integers(0, i)) for i in range(1, nodes)]


def _frequencies(case):
    """Radians per position of each rotated pair (64 bits) and the factor on the rotated values."""
    rot, theta, factor, original = case["rotary"], 10000.0, 8.0, 8192.0
    kind = case["scaling"]
    if kind == "ntk":
        theta = theta * factor ** (rot / (rot - 2))
    f = theta ** (-2.0 * np.arange(rot // 2, dtype=np.float64) / rot)
    amplitude = 1.0
    if kind == "linear":
        f = f / factor
    elif kind == "bands":
        turns = original * f / (2 * np.pi)
        smooth = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        f = (1 - smooth) * f / factor + smooth * f
    elif kind == "yarn":
        border = lambda beta: rot * math.log(original / (beta * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
        low, high = max(math.floor(border(32.0)), 0), min(math.ceil(border(1.0)), rot - 1)
        ramp = np.clip((np.arange(rot // 2) - low) / max(high - low, 0.001), 0.0, 1.0)
        f = ramp * f / factor + (1 - ramp) * f
        amplitude = 0.1 * math.log(factor) + 1.0
    return f, amplitude


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"case": case}
    Hkv, D, op = case["kv_heads"], case["dim"], case["op"]
    page = Hkv * 2 * PAGE * D
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    if op == "tree":
        B, T, Hq, W = case["batch"], case["nodes"], case["heads"], case["window"]
        ctx = _lens(rng, case["ctx_lo"], case["ctx_hi"], B)
        size = np.full(B, T) if case["shape"] == "full" else rng.integers(max(1, T // 2), T + 1, size=B)
        size[0] = T
        mask, depth = np.zeros((B, T), dtype=np.uint64), np.zeros((B, T), dtype=np.int64)
        for b in range(B):
            for i, p in enumerate(_tree(rng, case["shape"], int(size[b]))):
                mask[b, i] = (int(mask[b, p]) if p >= 0 else 0) | 1 << i
                depth[b, i] = depth[b, p] + 1 if p >= 0 else 0
        pages = (ctx + size + PAGE - 1) // PAGE
        first = np.maximum(0, ctx + 1 - W) // PAGE if W else np.zeros(B, dtype=np.int64)
        width = int(pages.max())
        table = np.full((B, width), -1, dtype=np.int32)       # pages that no query can see any more are unmapped
        total = int((pages - first).sum()) + 3
        held, _ = _tables(rng, pages - first, width, total)
        for b in range(B):
            table[b, first[b]:pages[b]] = held[b, :pages[b] - first[b]]
        s.update(pool=_normal(gen, total * page), q=_normal(gen, B, T, Hq, D), mask=cuda(mask.view(np.int64)),
                 positions=cuda((ctx[:, None] + depth).astype(np.int32)), ctx=cuda(ctx.astype(np.int32)),
                 size=cuda(size.astype(np.int32)), table=cuda(table), first=cuda(first), span=int((pages - first).max()),
                 out=torch.empty(B, T, Hq, D, dtype=torch.bfloat16, device="cuda"),
                 lse=torch.empty(B, T, Hq, dtype=torch.float32, device="cuda"))
        pools, windows, rows = [s["pool"]], [W], B
    elif op == "rope":
        R, Hq, n = case["rows"], case["heads"], case["seqs"]
        seq = np.sort(np.concatenate([np.arange(n), rng.integers(0, n, size=R - n)]))
        count = np.bincount(seq, minlength=n)
        start = rng.integers(0, 40, size=n)                   # tokens already cached: the new ones begin inside a page
        slot = start[seq] + np.arange(R) - (np.cumsum(count) - count)[seq]
        pages = (start + count + PAGE - 1) // PAGE
        total = (R + 54 * n) // PAGE + 2                      # whatever the seed
        table, _ = _tables(rng, pages, int(pages.max()), total)
        shift = rng.integers(0, case["far"], size=n)          # what the positions are ahead of the slots
        qkv = _normal(gen, R, Hq + 2 * Hkv, D)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        if not case["packed"]:
            q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        f, amplitude = _frequencies(case)
        s.update(pool=_normal(gen, total * page), q=q, k=k, v=v, seq=cuda(seq.astype(np.int32)), slot=cuda(slot.astype(np.int32)),
                 positions=cuda((slot + shift[seq]).astype(np.int32)), table=cuda(table), f=cuda(f), amplitude=amplitude,
                 out=torch.empty(R, Hq, D, dtype=torch.bfloat16, device="cuda"))
        pools, windows, rows = [s["pool"]], [0], n
    elif op == "commit":
        B, T, L = case["batch"], case["nodes"], case["layers"]
        ctx = _lens(rng, case["ctx_lo"], case["ctx_hi"], B)
        took = rng.integers(0, T + 1, size=B)
        took[0] = max(1, T // 2)
        path = np.zeros((B, T), dtype=np.int32)
        for b in range(B):                                    # a path through the tree: ascending nodes
            path[b, :took[b]] = np.sort(rng.permutation(T)[:took[b]])
        pages = (ctx + T + PAGE - 1) // PAGE
        total = B * int(pages.max())
        table, _ = _tables(rng, pages, int(pages.max()), total)
        s.update(pools=[_normal(gen, total * page) for _ in range(L)], path=cuda(path), took=cuda(took.astype(np.int32)),
                 ctx=cuda(ctx.astype(np.int32)), table=cuda(table), lens=torch.empty(B, dtype=torch.int32, device="cuda"))
        pools, windows, rows = s["pools"], [0] * L, B
    else:
        P, C, L = case["parents"], case["children"], case["layers"]
        have = _lens(rng, case["len_lo"], case["len_hi"], P)
        src = rng.integers(0, P, size=C)
        lens = have[src]
        if op == "release":
            lens = lens // PAGE * PAGE
        pages = (have + PAGE - 1) // PAGE
        total = P * int(pages.max()) + C + 5
        held, spare = _tables(rng, pages, int(pages.max()), total)
        table = np.full((P + C, held.shape[1]), -1, dtype=np.int32)
        table[:P] = held
        counts = np.zeros(total, dtype=np.int32)
        counts[held[held >= 0]] = 1
        s.update(pools=[_normal(gen, total * page) for _ in range(L)] if op == "fork" else
                 [torch.zeros(total * page, dtype=torch.bfloat16, device="cuda")],
                 src=cuda(src.astype(np.int32)), dst=cuda(P + rng.permutation(C).astype(np.int32)), lens=cuda(lens.astype(np.int32)),
                 new=cuda(spare[:C].astype(np.int32)), table=cuda(table), counts=cuda(counts),
                 free=torch.full((total,), -1, dtype=torch.int32, device="cuda"),
                 n_free=torch.zeros(1, dtype=torch.int32, device="cuda"))
        pools, windows, rows = s["pools"], [0] * L, P + C
    if own:
        from paper_2609_14237_b200 import binding as B_
        s["stage"] = B_.Stage(pools=pools, layer_window=windows, num_q_heads=case.get("heads", Hkv), num_kv_heads=Hkv, head_dim=D,
                              max_batch=rows, max_pages_per_seq=s["table"].shape[1])
        s["layers"] = list(range(len(pools)))
        if op == "tree":
            s["tree"] = B_.TreeAttention(s["stage"], case["nodes"])
        if op == "rope":
            s["rope"] = B_.Rope(case["rotary"], layout=case["layout"], theta=10000.0, scaling=case["scaling"], factor=8.0,
                                original_context=8192.0, device=s["pool"].device)
    return s


# ------------------------------------------------------------------------------ plain forms ---

def _order(D, device):
    """Where element (slot t, dim d) stands in a page's tile of one head: groups of eight permuted by the slot."""
    t, d = torch.arange(PAGE, device=device)[:, None], torch.arange(D, device=device)[None]
    return t * D + ((d // 8) ^ (t & 7)) * 8 + d % 8


def _places(pool, table, seq, slot, Hkv, D):
    """Element offsets [rows, Hkv, 2, D] of the cached rows at (sequence, slot)."""
    pid = table[seq.long(), slot.long() // PAGE].long()
    t = slot.long() % PAGE
    heads = torch.arange(Hkv, device=pool.device)
    tile = ((pid[:, None] * Hkv + heads)[:, :, None] * 2 + torch.arange(2, device=pool.device)) * (PAGE * D)
    return tile[..., None] + _order(D, pool.device)[t][:, None, None]


def _plain_tree(s):
    c = s["case"]
    B, T, Hq, Hkv, D, W = c["batch"], c["nodes"], c["heads"], c["kv_heads"], c["dim"], c["window"]
    dev, S = s["pool"].device, s["span"] * PAGE
    page = s["first"][:, None] + torch.arange(s["span"], device=dev)
    pid = torch.gather(s["table"], 1, page.clamp(max=s["table"].shape[1] - 1)).clamp(min=0).long()
    kv = s["pool"].view(-1, Hkv, 2, PAGE * D)[pid][..., _order(D, dev).reshape(-1)]
    kv = kv.view(B, s["span"], Hkv, 2, PAGE, D).permute(3, 0, 2, 1, 4, 5).reshape(2, B, Hkv, S, D)
    q = s["q"].view(B, T, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    x = torch.matmul(q.float(), kv[0].float().transpose(-1, -2)) * (1.0 / math.sqrt(D))
    key = (s["first"] * PAGE)[:, None] + torch.arange(S, device=dev)                       # [B, S]
    node = key - s["ctx"][:, None]
    drafted = (s["mask"][:, :, None] >> node.clamp(0, 63)[:, None]) & 1
    sees = torch.where(node[:, None] < 0, True, (drafted != 0) & (node < s["size"][:, None])[:, None])
    if W:                                                                                  # the window counts positions
        at = torch.where(node < 0, key, torch.gather(s["positions"].long(), 1, node.clamp(0, T - 1)))
        sees = sees & (at[:, None] > s["positions"].long()[:, :, None] - W)
    sees = sees & (torch.arange(T, device=dev) < s["size"][:, None])[:, :, None]           # [B, T, S]
    hides = ~sees[:, None, :, None].expand(B, Hkv, T, Hq // Hkv, S).reshape(B, Hkv, -1, S)
    x = x.masked_fill_(hides, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, kv[1].float()) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total)).view(B, Hkv, T, -1).permute(0, 2, 1, 3).reshape(B, T, Hq)
    return out.view(B, Hkv, T, -1, D).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D).to(torch.bfloat16), lse


def _plain_rope(s):
    c = s["case"]
    rot = c["rotary"]
    angle = s["positions"].double()[:, None] * s["f"]
    cos, sin = ((g(angle) * s["amplitude"]).float()[:, None] for g in (torch.cos, torch.sin))

    def turn(x):
        x = x.float()
        if c["layout"] == "half":
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        return torch.cat([y, x[..., rot:]], -1).to(torch.bfloat16)

    at = _places(s["pool"], s["table"], s["seq"], s["slot"], c["kv_heads"], c["dim"])
    s["pool"][at] = torch.stack([turn(s["k"]), s["v"]], 2)
    return turn(s["q"]), s["pool"]


def _plain_commit(s):
    c = s["case"]
    B, T = c["batch"], c["nodes"]
    dev = s["path"].device
    row = torch.arange(B, device=dev)[:, None].expand(B, T).reshape(-1)
    i = torch.arange(T, device=dev)[None]
    taken = i < s["took"][:, None]
    src = (s["ctx"][:, None] + torch.where(taken, s["path"], i)).reshape(-1)               # rows behind the path stay
    dst = (s["ctx"][:, None] + i).reshape(-1)
    for pool in s["pools"]:
        a = _places(pool, s["table"], row, src, c["kv_heads"], c["dim"])
        pool[_places(pool, s["table"], row, dst, c["kv_heads"], c["dim"])] = pool[a]
    return s["pools"], s["ctx"] + s["took"]


def _plain_fork(s):
    C, width = s["case"]["children"], s["table"].shape[1]
    src, dst, lens = s["src"].long(), s["dst"].long(), s["lens"].long()
    full, i = (lens // PAGE)[:, None], torch.arange(width, device=src.device)[None]
    old = s["table"][src]
    rest = (lens % PAGE)[:, None]
    s["table"][dst] = torch.where(i < full, old, torch.where((i == full) & (rest > 0), s["new"][:, None], -1))
    shared = torch.where(i < full, old, 0).reshape(-1).long()
    s["counts"].index_add_(0, shared, (i < full).expand(C, width).reshape(-1).int())
    partial = torch.gather(old, 1, full.clamp(max=width - 1)).squeeze(1).long()
    new = s["new"].long()
    s["counts"][new] = torch.where(rest.squeeze(1) > 0, 1, s["counts"][new])
    if s["case"]["op"] == "fork":
        for pool in s["pools"]:
            pages = pool.view(s["counts"].shape[0], -1, PAGE, s["case"]["dim"])
            held = torch.arange(PAGE, device=src.device)[None, :] < rest                   # the slots that hold a token
            pages[new] = torch.where(held[:, None, :, None], pages[partial.clamp(min=0)], pages[new])
    return s["pools"], s["table"], s["counts"]


def _plain_release(s):
    _plain_fork(s)
    dst = s["dst"].long()
    drop = s["table"][dst].reshape(-1)
    s["counts"].index_add_(0, drop.clamp(min=0).long(), -(drop >= 0).int())
    s["table"][dst] = -1
    idle = s["counts"] == 0
    n = s["counts"].shape[0]
    place = torch.where(idle, torch.cumsum(idle, 0) - 1, n)
    lst = torch.cat([s["free"], s["free"][:1]])
    lst[place] = torch.arange(n, device=dst.device, dtype=torch.int32)
    s["free"] = lst[:n]
    return s["table"], s["counts"], s["free"], idle.sum().int().reshape(1)


# -------------------------------------------------------------------------------------- run ---

def run(s):
    op = s["case"]["op"]
    if own:
        stage = s["stage"]
        if op == "tree":
            s["tree"].attention(0, s["q"], s["mask"], s["positions"], s["ctx"], s["size"], s["table"], s["out"], s["lse"])
            return s["out"], s["lse"]
        if op == "rope":
            stage.rope_append(0, s["rope"], s["q"], s["k"], s["v"], s["seq"], s["slot"], s["positions"], s["table"], s["out"])
            return s["out"], s["pool"]
        if op == "commit":
            stage.kv_commit(s["layers"], s["path"], s["took"], s["ctx"], s["table"], s["lens"])
            return s["pools"], s["lens"]
        stage.kv_fork(s["layers"], s["src"], s["dst"], s["lens"], s["new"], s["table"], s["counts"])
        if op == "fork":
            return s["pools"], s["table"], s["counts"]
        stage.kv_release(s["dst"], None, s["table"], s["counts"])
        stage.kv_free_pages(s["counts"], s["free"], s["n_free"])
        return s["table"], s["counts"], s["free"], s["n_free"]
    return {"tree": _plain_tree, "rope": _plain_rope, "commit": _plain_commit, "fork": _plain_fork, "release": _plain_release}[op](s)


# ------------------------------------------------------------------------------------- work ---

def work(case):
    op, Hkv, D = case["op"], case["kv_heads"], case["dim"]
    row = Hkv * 2 * D * 2                                     # bytes of one token's key and value rows
    if op == "tree":
        B, T, Hq, W = case["batch"], case["nodes"], case["heads"], case["window"]
        ctx = (case["ctx_lo"] + case["ctx_hi"]) / 2 + (case["ctx_hi"] - case["ctx_lo"]) / 2 / B
        size = T if case["shape"] == "full" else (max(1, T // 2) + T) / 2
        keys = min(ctx, W) if W else ctx
        return {"bytes": B * ((keys + size) * row + 2 * T * Hq * D * 2 + T * Hq * 4), "flops": 4 * B * size * Hq * D * (keys + size / 2)}
    if op == "rope":
        return {"bytes": case["rows"] * (2 * (case["heads"] * D * 2 + row) + 12), "flops": case["rows"] * (case["heads"] + Hkv) * case["rotary"] * 3}
    if op == "commit":
        return {"bytes": case["batch"] * (case["nodes"] / 2) * (2 * row * case["layers"] + 4) + case["batch"] * 12, "flops": 0}
    C, P = case["children"], case["parents"]
    pages = (case["len_lo"] + case["len_hi"]) / 2 / PAGE
    if op == "fork":
        return {"bytes": C * (7.5 * 2 * row * case["layers"] + 20 + 16 * pages), "flops": 0}
    total = P * ((case["len_hi"] + PAGE - 1) // PAGE) + C + 5
    return {"bytes": C * pages * 16 + C * 16 + total * 4 + (C + 5) * 4, "flops": 0}


# ------------------------------------------------------------------------------------ exact ---

def _rows_of(pool, table_row, lo, n, Hkv, D):
    """Cached rows [lo, n) of one sequence from their definition: [n - lo, Hkv, 2, D]."""
    j = np.arange(lo, n)
    d = np.arange(D)
    chunk = ((d[None] >> 3) ^ (j[:, None] & 7)) * 8 + (d[None] & 7)                        # [keys, D]
    tile = table_row[j // PAGE].astype(np.int64)[:, None, None] * Hkv + np.arange(Hkv)[None, :, None]
    at = ((tile * 2 + np.arange(2)[None, None]) * PAGE + (j % PAGE)[:, None, None])[..., None] * D + chunk[:, None, None]
    return torch.from_numpy(at).to(pool.device)


def exact(case, seed):
    s = prepare(case, seed)
    op, Hkv, D = case["op"], case["kv_heads"], case["dim"]
    table = s["table"].cpu().numpy()
    if op == "tree":
        B, T, Hq, W = case["batch"], case["nodes"], case["heads"], case["window"]
        G = Hq // Hkv
        ctx, size = s["ctx"].tolist(), s["size"].tolist()
        mask, pos = s["mask"].cpu().numpy().view(np.uint64), s["positions"].cpu().numpy().astype(np.int64)
        out = torch.zeros(B, T, Hq, D, dtype=torch.float64, device="cuda")
        lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64, device="cuda")
        for b in range(B):
            lo = max(0, ctx[b] + 1 - W) if W else 0
            n = ctx[b] + size[b]
            rows = s["pool"][_rows_of(s["pool"], table[b], lo, n, Hkv, D)].double()       # [keys, Hkv, 2, D]
            where = np.concatenate([np.arange(lo, ctx[b]), pos[b, :size[b]]])
            for i in range(size[b]):
                seen = np.array([True] * (ctx[b] - lo) + [bool(int(mask[b, i]) >> m & 1) for m in range(size[b])])
                if W:
                    seen &= where >= pos[b, i] - W + 1
                if not seen.any():
                    continue
                hidden = torch.from_numpy(np.where(seen, 0.0, -math.inf)).cuda()
                q = s["q"][b, i].double().view(Hkv, G, D)
                x = torch.einsum("hgd,khd->hgk", q, rows[:, :, 0]) / math.sqrt(D) + hidden
                lse[b, i] = torch.logsumexp(x, -1).view(Hq)
                out[b, i] = torch.einsum("hgk,khd->hgd", torch.softmax(x, -1), rows[:, :, 1]).reshape(Hq, D)
        return out, lse
    if op == "rope":
        rot = case["rotary"]
        z = torch.polar(torch.tensor(s["amplitude"], dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["f"])

        def turn(x):
            y = x.double().contiguous()
            if case["layout"] == "half":
                w = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * z[:, None]
                y[..., :rot // 2], y[..., rot // 2:rot] = w.real, w.imag
            else:
                w = torch.view_as_complex(y[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * z[:, None]
                y[..., :rot] = torch.view_as_real(w).flatten(-2)
            return y

        pool, k = s["pool"].double(), turn(s["k"])
        slot, seq = s["slot"].cpu().numpy(), s["seq"].cpu().numpy()
        for b in range(case["seqs"]):
            mine = np.nonzero(seq == b)[0]
            at = _rows_of(pool, table[b], int(slot[mine[0]]), int(slot[mine[-1]]) + 1, Hkv, D)
            r = torch.from_numpy(mine).cuda()
            pool[at] = torch.stack([k[r], s["v"][r].double()], 2)
        return turn(s["q"]), pool
    if op == "commit":
        path, took, ctx = s["path"].tolist(), s["took"].tolist(), s["ctx"].tolist()
        pools = [p.double() for p in s["pools"]]
        for b in range(case["batch"]):
            at = _rows_of(pools[0], table[b], ctx[b], ctx[b] + case["nodes"], Hkv, D)
            m = took[b]
            for p in pools:
                p[at[:m]] = p[at[path[b][:m]]]
        return pools, None
    if op == "fork":
        src, lens, new = s["src"].tolist(), s["lens"].tolist(), s["new"].tolist()
        pools = [p.double().view(s["counts"].shape[0], -1, PAGE, D) for p in s["pools"]]
        for p in pools:
            for c in range(case["children"]):
                if lens[c] % PAGE:
                    p[new[c], :, :lens[c] % PAGE] = p[int(table[src[c], lens[c] // PAGE]), :, :lens[c] % PAGE]
        return [p.view(-1) for p in pools], None, None
    return None
