"""Cases of the operators that a step of a server makes around the attention of shared and drafted tokens.

prefix   decode attention of sequences that share the first pages of their cache, the shared keys taken once for all of a group
verify   which drafted tokens of a tree the target's probabilities accept, by given random numbers, and the token that follows
norm     queries and keys normalised head by head, rotated and appended to the paged cache in one pass
extend   pages for the new tokens of ragged requests, dealt from the list of free ones, and the rows' places in the cache
"""
import math

import numpy as np
import torch

own = False

PAGE = 16


# ---------------------------------------------------------------------------------- cases ---

def listed():
    return [
        # four samples of one short prompt: the smallest call, latency only
        dict(name="prefix 4 samples of 1000", op="prefix", groups=1, batch=4, even=True, pre_lo=1000, pre_hi=1000, own_lo=40, own_hi=40,
             heads=32, kv_heads=8, dim=128, window=0),
        # a batch behind one kept system prompt
        dict(name="prefix 64 behind 8k", op="prefix", groups=1, batch=64, even=True, pre_lo=8192, pre_hi=8192, own_lo=1, own_hi=1024,
             heads=32, kv_heads=8, dim=128, window=0),
        # the largest: many prompts, each sampled sixteen times
        dict(name="prefix 16 x 16 behind 16k", op="prefix", groups=16, batch=256, even=True, pre_lo=16384, pre_hi=16384, own_lo=16,
             own_hi=2048, heads=32, kv_heads=8, dim=128, window=0),
        # groups of uneven sizes on a sliding-window layer: the window ends inside the shared part for some rows
        dict(name="prefix 5 ragged, window 4096", op="prefix", groups=5, batch=33, even=False, pre_lo=2000, pre_hi=7000, own_lo=1,
             own_hi=3000, heads=32, kv_heads=8, dim=128, window=4096),
        # one sequence's chain of four: the smallest call
        dict(name="verify chain of 4, 1 seq", op="verify", batch=1, nodes=4, shape="chain", vocab=32000, dtype="f32", draw="again"),
        # the middle of a batch with a large vocabulary, branches drawn independently
        dict(name="verify trees of 8, 64 seqs", op="verify", batch=64, nodes=8, shape="tree", vocab=131072, dtype="f32", draw="again"),
        # half-width probabilities, an odd vocabulary, distinct branches
        dict(name="verify trees of 13, 128 seqs", op="verify", batch=128, nodes=13, shape="tree", vocab=50001, dtype="bf16",
             draw="distinct"),
        # the drafted tokens of 16 trees before their attention
        dict(name="norm 16 trees of 8", op="norm", rows=128, seqs=16, packed=False, layout="half", rotary=128, per_head=False,
             heads=32, kv_heads=8, dim=128),
        # prompts of together 8192 tokens entering the cache, straight from the packed projection
        dict(name="norm prompts, 8192 tokens", op="norm", rows=8192, seqs=7, packed=True, layout="half", rotary=128, per_head=False,
             heads=32, kv_heads=8, dim=128),
        # a decode step: a token for each of 64 sequences, a page for every sixteenth
        dict(name="extend 64 decodes", op="extend", requests=64, prompts=0, tokens=1, have=4096),
        # a step that takes in prompts beside a large batch of decodes
        dict(name="extend 1000 and 24 prompts", op="extend", requests=1024, prompts=24, tokens=2600, have=8192),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["prefix", "prefix", "verify", "verify", "norm", "extend"])
    heads, kv_heads, dim = rng.choice([(32, 8, 128), (32, 8, 128), (64, 8, 128), (8, 2, 64), (32, 16, 128), (16, 1, 128), (5, 1, 64),
                                       (24, 2, 64), (16, 2, 256)])
    if op == "prefix":
        batch = _log(rng, 2, 256)
        groups = _log(rng, 1, min(16, batch))
        pre, mine = _log(rng, 1, 16384), _log(rng, 1, 2048)
        # keys that a pass reads, and scores that it computes: no more than the largest listed case
        while (groups * pre + batch * mine) * kv_heads * dim > 16 * 32768 * 1024 or batch * (pre + mine) * heads * dim > 256 * 18432 * 4096:
            pre, mine = max(1, pre // 2), max(1, mine // 2)
        return dict(op=op, groups=groups, batch=batch, even=rng.random() < 0.5, pre_lo=rng.randint(0, pre), pre_hi=pre,
                    own_lo=rng.randint(1, mine), own_hi=mine, heads=heads, kv_heads=kv_heads, dim=dim,
                    window=rng.choice([0, 0, 0, 40, 1024, 4096]))
    if op == "verify":
        vocab = _log(rng, 1000, 151000)
        batch, nodes = _log(rng, 1, 256), _log(rng, 1, 64)
        while batch * nodes * vocab > 64 * 8 * 131072:
            batch, nodes = max(1, batch // 2), max(1, nodes * 2 // 3)
        return dict(op=op, batch=batch, nodes=nodes, shape=rng.choice(["tree", "chain"]), vocab=vocab, dtype=rng.choice(["f32", "f32", "bf16"]),
                    draw=rng.choice(["again", "distinct", "certain"]))
    if op == "norm":
        rows = _log(rng, 1, 8192 * 32 * 128 // max(heads * dim, 4096))
        return dict(op=op, rows=rows, seqs=rng.randint(1, min(rows, 64)), packed=rng.random() < 0.5, layout=rng.choice(["half", "interleaved"]),
                    rotary=rng.choice([dim, dim, dim // 2, dim // 4, dim // 4 + 2]), per_head=rng.random() < 0.25,
                    heads=heads, kv_heads=kv_heads, dim=dim)
    requests = _log(rng, 1, 1024)
    prompts = rng.randint(0, min(requests, 24))
    return dict(op=op, requests=requests, prompts=prompts, tokens=_log(rng, 1, 2600), have=_log(rng, 1, 8192))


# --------------------------------------------------------------------------------- inputs ---

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _spread(rng, lo, hi, n):
    x = rng.integers(lo, hi + 1, size=n)
    x[0] = hi
    return x.astype(np.int64)


def _parents(rng, kind, nodes):
    """The drafted tree of one sequence: node 0 is the last token that was decided, the others follow an earlier node."""
    if kind == "chain":
        return [i - 1 for i in range(nodes)]
    return [-1] + [int(i - 1 - min(i - 1, rng.geometric(0.3) - 1)) for i in range(1, nodes)]


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"case": case}
    op = case["op"]
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    i32 = lambda a: cuda(np.asarray(a).astype(np.int32))  # noqa: E731
    Hkv, D = case.get("kv_heads", 1), case.get("dim", 64)
    Hq, page = case.get("heads", Hkv), Hkv * 2 * PAGE * D
    if op == "prefix":
        G, B = case["groups"], case["batch"]
        if case["even"]:
            start = np.arange(G + 1) * B // G
        else:
            start = np.concatenate([[0], np.sort(rng.permutation(B - 1)[:G - 1]) + 1, [B]])
        group = np.repeat(np.arange(G), np.diff(start))
        pre = _spread(rng, case["pre_lo"], case["pre_hi"], G)
        shared = pre // PAGE                                  # a fork shares whole pages and copies the last partial one
        lens = pre[group] + _spread(rng, case["own_lo"], case["own_hi"], B)
        pages = (lens + PAGE - 1) // PAGE
        width, total = int(pages.max()), int(shared.sum() + (pages - shared[group]).sum()) + 3
        order = rng.permutation(total).astype(np.int32)
        table, at = np.full((B, width), -1, dtype=np.int32), 0
        for g in range(G):
            table[start[g]:start[g + 1], :shared[g]] = order[at:at + shared[g]]
            at += int(shared[g])
        for b in range(B):
            mine = int(pages[b] - shared[group[b]])
            table[b, shared[group[b]]:pages[b]] = order[at:at + mine]
            at += mine
        s.update(pool=_normal(gen, total * page), q=_normal(gen, B, Hq, D), lens=i32(lens), starts=i32(start), pre=i32(pre), table=cuda(table),
                 group=cuda(group), member=cuda(np.arange(B) - start[group]), most=int(np.diff(start).max()), span=int(shared.max()),
                 rest=int((pages - shared[group]).max()), out=torch.empty(B, Hq, D, dtype=torch.bfloat16, device="cuda"),
                 lse=torch.empty(B, Hq, dtype=torch.float32, device="cuda"))
        pools, windows, rows = [s["pool"]], [case["window"]], B
    elif op == "verify":
        B, T, V = case["batch"], case["nodes"], case["vocab"]
        kind = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        parents = np.array([_parents(rng, case["shape"], T) for _ in range(B)])
        size = np.where(rng.random(B) < 0.3, rng.integers(1, T + 1, size=B), T)
        size[0] = T
        # a language model's distributions: a few likely tokens, a long tail; the drafter's are near the target's
        target, draft = (torch.empty(B, T, V, dtype=kind, device="cuda") for _ in range(2))
        part = max(1, (1 << 27) // (T * V))
        drawn = torch.empty(B, T, T, dtype=torch.int64, device="cuda")
        for b in range(0, B, part):
            x = 3.0 * torch.randn(min(part, B - b), T, V, generator=gen, device="cuda")
            y = x + 0.7 * torch.randn(x.shape, generator=gen, device="cuda")
            target[b:b + part] = torch.softmax(x, -1).to(kind)
            p = torch.softmax(y, -1).to(kind)
            draft[b:b + part] = p
            if case["draw"] == "certain":
                drawn[b:b + part] = torch.topk(y, T, -1).indices
            else:
                drawn[b:b + part] = torch.multinomial(p.float().view(-1, V), T, replacement=case["draw"] == "again",
                                                      generator=gen).view(-1, T, T)
        rank = np.array([[(parents[b, :i] == parents[b, i]).sum() for i in range(T)] for b in range(B)])
        tokens = drawn[torch.arange(B, device="cuda")[:, None], cuda(parents).clamp(min=0), cuda(rank)].int().contiguous()
        s.update(target=target, draft=None if case["draw"] == "certain" else draft, tokens=tokens, parents=i32(parents), size=i32(size),
                 u=torch.rand(B, T, generator=gen, device="cuda"), path=torch.empty(B, T, dtype=torch.int32, device="cuda"),
                 took=torch.empty(B, dtype=torch.int32, device="cuda"), follows=torch.empty(B, dtype=torch.int32, device="cuda"),
                 pool=torch.zeros(page, dtype=torch.bfloat16, device="cuda"), table=i32(np.zeros((B, 1))))
        pools, windows, rows = [s["pool"]], [0], B
    elif op == "norm":
        R, n = case["rows"], case["seqs"]
        seq = np.sort(np.concatenate([np.arange(n), rng.integers(0, n, size=R - n)]))
        count = np.bincount(seq, minlength=n)
        start = rng.integers(0, 40, size=n)                   # tokens already cached: the new ones begin inside a page
        slot = start[seq] + np.arange(R) - (np.cumsum(count) - count)[seq]
        pages = (start + count + PAGE - 1) // PAGE
        total = (R + 54 * n) // PAGE + 2                      # whatever the seed
        order, table, at = rng.permutation(total).astype(np.int32), np.full((n, int(pages.max())), -1, dtype=np.int32), 0
        for b in range(n):
            table[b, :pages[b]] = order[at:at + pages[b]]
            at += int(pages[b])
        qkv = _normal(gen, R, Hq + 2 * Hkv, D)
        qkv *= torch.exp(torch.randn(R, 1, 1, generator=gen, device="cuda"))                # rows of different size
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        if not case["packed"]:
            q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        weight = lambda heads: 1 + 0.2 * torch.randn(*((heads, D) if case["per_head"] else (D,)), generator=gen, device="cuda")  # noqa: E731
        s.update(pool=_normal(gen, total * page), q=q, k=k, v=v, wq=weight(Hq), wk=weight(Hkv), seq=i32(seq), slot=i32(slot),
                 positions=i32(slot + rng.integers(0, 4096, size=n)[seq]), table=cuda(table),
                 f=cuda(10000.0 ** (-2.0 * np.arange(case["rotary"] // 2) / case["rotary"])),
                 out=torch.empty(R, Hq, D, dtype=torch.bfloat16, device="cuda"))
        pools, windows, rows = [s["pool"]], [0], n
    else:
        n = case["requests"]
        have = _spread(rng, 1, case["have"], n)
        new = np.ones(n, dtype=np.int64)
        first = rng.permutation(n)[:case["prompts"]]
        have[first] = 0
        new[first] = _spread(rng, 1, case["tokens"], len(first)) if len(first) else 0
        # all but a few rows of the table are in use, and the requests come in no order
        B = n + n // 8 + 1
        row = rng.permutation(B)[:n]
        width = (max(case["have"], case["tokens"]) + PAGE) // PAGE + 1
        pages = (have + PAGE - 1) // PAGE
        total = n * ((case["have"] + PAGE) // PAGE + 1) + case["prompts"] * (case["tokens"] // PAGE + 1) + 7
        order, table, at = rng.permutation(total).astype(np.int32), np.full((B, width), -1, dtype=np.int32), 0
        counts = np.zeros(total, dtype=np.int32)
        for f in range(n):
            table[row[f], :pages[f]] = order[at:at + pages[f]]
            at += int(pages[f])
        counts[order[:at]] = 1
        room = n + case["prompts"] * case["tokens"]           # a captured step has room for its largest number of rows
        ints = lambda k: torch.empty(k, dtype=torch.int32, device="cuda")  # noqa: E731
        s.update(pool=torch.zeros(page, dtype=torch.bfloat16, device="cuda"), rows=i32(row), have=i32(have), new=i32(new),
                 table=cuda(table), counts=cuda(counts), free=i32(np.nonzero(counts == 0)[0]), n_free=i32([int((counts == 0).sum())]),
                 room=room, begins=ints(n + 1), lens=ints(n), seq=ints(room), slot=ints(room), used=ints(1))
        pools, windows, rows = [s["pool"]], [0], B
    if own:
        from paper_2609_14237_b200 import binding as B_
        s["stage"] = B_.Stage(pools=pools, layer_window=windows, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, max_batch=rows,
                              max_pages_per_seq=s["table"].shape[1])
        if op == "prefix":
            s["prefix"] = B_.PrefixAttention(s["stage"])
        if op == "norm":
            s["rope"] = B_.Rope(case["rotary"], layout=case["layout"], theta=10000.0, device=s["pool"].device)
    return s


# ------------------------------------------------------------------------------ plain forms ---

def _order(D, device):
    """Where element (slot t, dim d) stands in a page's tile of one head: groups of eight permuted by the slot."""
    t, d = torch.arange(PAGE, device=device)[:, None], torch.arange(D, device=device)[None]
    return t * D + ((d // 8) ^ (t & 7)) * 8 + d % 8


def _keys_values(pool, pid, Hkv, D):
    """fp32 keys and values of the pages pid [n, m]: 2 x [n, Hkv, m * 16, D]."""
    n, m = pid.shape
    kv = pool.view(-1, Hkv, 2, PAGE * D)[pid.clamp(min=0).long()][..., _order(D, pool.device).reshape(-1)]
    kv = kv.view(n, m, Hkv, 2, PAGE, D).permute(3, 0, 2, 1, 4, 5).reshape(2, n, Hkv, m * PAGE, D)
    return kv[0].float(), kv[1].float()


def _plain_prefix(s):
    c = s["case"]
    G, B, Hq, Hkv, D, W, M = c["groups"], c["batch"], c["heads"], c["kv_heads"], c["dim"], c["window"], s["most"]
    dev, lens, start, shared = s["q"].device, s["lens"].long(), s["starts"].long(), s["pre"].long() // PAGE
    lo = (lens - W).clamp(min=0) if W else torch.zeros_like(lens)
    q = s["q"].view(B, Hkv, Hq // Hkv, D).float() * (1.0 / math.sqrt(D))
    # the shared keys against all rows of a group at a time
    rows = (start[:-1, None] + torch.arange(M, device=dev)).clamp(max=B - 1)               # [G, M]
    k, v = _keys_values(s["pool"], s["table"][start[:-1], :s["span"]], Hkv, D)
    x = torch.matmul(q[rows].permute(0, 2, 1, 3, 4).reshape(G, Hkv, M * Hq // Hkv, D), k.transpose(-1, -2))
    P = s["span"] * PAGE
    x = x.view(G, Hkv, M, Hq // Hkv, P).permute(0, 2, 1, 3, 4)[s["group"], s["member"]]    # [B, Hkv, Hq / Hkv, P]
    key = torch.arange(P, device=dev)[None]
    sees = (key < torch.minimum(lens, shared[s["group"]] * PAGE)[:, None]) & (key >= lo[:, None])
    x = x.masked_fill_(~sees[:, None, None], -math.inf)
    # each row's own keys
    page = shared[s["group"]][:, None] + torch.arange(s["rest"], device=dev)
    k2, v2 = _keys_values(s["pool"], torch.gather(s["table"], 1, page.clamp(max=s["table"].shape[1] - 1)), Hkv, D)
    y = torch.matmul(q, k2.transpose(-1, -2))
    key = (page[:, :, None] * PAGE + torch.arange(PAGE, device=dev)).view(B, -1)
    y = y.masked_fill_(~((key < lens[:, None]) & (key >= lo[:, None]))[:, None, None], -math.inf)
    top = y.amax(-1, keepdim=True)
    if P:
        top = torch.maximum(top, x.amax(-1, keepdim=True))
    x, y = torch.exp(x - top), torch.exp(y - top)
    total = x.sum(-1, keepdim=True) + y.sum(-1, keepdim=True)
    out = torch.matmul(y, v2)
    back = torch.zeros(G, M, *x.shape[1:], device=dev)
    back[s["group"], s["member"]] = x
    back = torch.matmul(back.permute(0, 2, 1, 3, 4).reshape(G, Hkv, M * Hq // Hkv, P), v)
    out += back.view(G, Hkv, M, Hq // Hkv, D).permute(0, 2, 1, 3, 4)[s["group"], s["member"]]
    return (out / total).reshape(B, Hq, D).to(torch.bfloat16), (top + torch.log(total)).reshape(B, Hq)


def _plain_verify(s):
    c = s["case"]
    B, T, V = c["batch"], c["nodes"], c["vocab"]
    dev, seqs = s["u"].device, torch.arange(B, device=s["u"].device)
    now = torch.zeros(B, dtype=torch.int64, device=dev)                                    # the last accepted node
    path, took = torch.full((B, T), -1, dtype=torch.int32, device=dev), torch.ones(B, dtype=torch.int64, device=dev)
    path[:, 0] = 0
    token, u = s["tokens"].long(), s["u"].double()
    r = s["target"][:, 0].double()                                                         # what is left of its distribution
    q = None if s["draft"] is None else s["draft"][:, 0].double()
    for i in range(1, T):                                                                  # each decision goes by the ones before
        asked = (s["parents"][:, i] == now) & (i < s["size"])
        x = token[:, i, None]
        if s["draft"] is None:
            q = torch.zeros_like(r).scatter_(1, x, 1.0)
        takes = asked & (u[:, i] * q.gather(1, x)[:, 0] < r.gather(1, x)[:, 0])
        left = (r - q).clamp(min=0)
        total = left.sum(1, keepdim=True)
        drops = (asked & ~takes)[:, None]
        r = torch.where(drops & (total > 0), left / total, r)
        if c["draw"] == "distinct":                                                        # the next branch is another token
            fewer = q.scatter(1, x, 0.0)
            q = torch.where(drops, fewer / fewer.sum(1, keepdim=True).clamp(min=1e-300), q)
        r = torch.where(takes[:, None], s["target"][:, i].double(), r)
        if s["draft"] is not None:
            q = torch.where(takes[:, None], s["draft"][:, i].double(), q)
        path.scatter_(1, torch.where(takes, took, 0)[:, None], torch.where(takes, i, 0)[:, None].int())
        now, took = torch.where(takes, i, now), took + takes
    sums = torch.cumsum(r, 1)
    over = sums > u[:, :1] * sums[:, -1:]
    ids = torch.arange(V, device=dev)
    last = torch.where(r > 0, ids, -1).amax(1)                                             # where the sums round to nothing above
    follows = torch.where(over.any(1), torch.where(over, ids, V).amin(1), last)
    return path, took.int(), follows.int()


def _plain_norm(s):
    c = s["case"]
    rot, Hkv, D = c["rotary"], c["kv_heads"], c["dim"]
    angle = s["positions"].double()[:, None] * s["f"]
    cos, sin = (g(angle).float()[:, None] for g in (torch.cos, torch.sin))

    def turn(x, w):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
        if c["layout"] == "half":
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        return torch.cat([y, x[..., rot:]], -1).to(torch.bfloat16)

    slot = s["slot"].long()
    pid = s["table"][s["seq"].long(), slot // PAGE].long()
    tile = ((pid[:, None] * Hkv + torch.arange(Hkv, device=pid.device))[:, :, None] * 2 + torch.arange(2, device=pid.device)) * (PAGE * D)
    s["pool"][tile[..., None] + _order(D, pid.device)[slot % PAGE][:, None, None]] = torch.stack([turn(s["k"], s["wk"]), s["v"]], 2)
    return turn(s["q"], s["wq"]), s["pool"]


def _plain_extend(s):
    n, width, dev = s["rows"].shape[0], s["table"].shape[1], s["rows"].device
    row, have, new = s["rows"].long(), s["have"].long(), s["new"].long()
    begins = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), torch.cumsum(new, 0)])
    page = torch.arange(width, device=dev)[None]
    drop = torch.where(page >= ((have + PAGE - 1) // PAGE)[:, None], s["table"][row], -1)  # what the tokens taken back held
    s["counts"].index_add_(0, drop.clamp(min=0).view(-1).long(), -(drop >= 0).view(-1).int())
    s["table"][row] = torch.where(drop >= 0, -1, s["table"][row])
    wants = (page >= (have // PAGE)[:, None]) & (page < ((have + new + PAGE - 1) // PAGE)[:, None]) & (s["table"][row] < 0)
    need = wants.sum(1)
    fits = (torch.cumsum(need, 0) <= s["n_free"]) | (need == 0)
    wants = wants & fits[:, None]
    place = (torch.cumsum(wants.view(-1), 0) - 1).view(n, width)
    given = torch.where(wants, s["free"][place.clamp(0, s["free"].shape[0] - 1)], s["table"][row])
    s["table"][row] = given
    s["counts"].index_add_(0, torch.where(wants, given, 0).view(-1).long(), wants.view(-1).int())
    r = torch.arange(s["room"], device=dev)
    f = torch.searchsorted(begins, r, right=True) - 1
    live = (r < begins[-1]) & fits[f.clamp(max=n - 1)]
    f = f.clamp(max=n - 1)
    seq = torch.where(live, row[f], -1).int()
    slot = torch.where(live, have[f] + r - begins[f], -1).int()
    lens = torch.where(fits, have + new, have).int()
    return begins.int(), seq, slot, lens, wants.sum().int().reshape(1), s["table"], s["counts"]


# -------------------------------------------------------------------------------------- run ---

def run(s):
    op = s["case"]["op"]
    if own:
        stage = s["stage"]
        if op == "prefix":
            s["prefix"].attention(0, s["q"], s["lens"], s["starts"], s["pre"], s["table"], s["out"], s["lse"])
            return s["out"], s["lse"]
        if op == "verify":
            stage.tree_verify(s["target"], s["draft"], s["tokens"], s["parents"], s["size"], s["u"], s["path"], s["took"], s["follows"],
                              distinct=s["case"]["draw"] == "distinct")
            return s["path"], s["took"], s["follows"]
        if op == "norm":
            stage.norm_rope_append(0, s["rope"], s["q"], s["k"], s["v"], s["wq"], s["wk"], s["seq"], s["slot"], s["positions"], s["table"],
                                   s["out"], eps=1e-6)
            return s["out"], s["pool"]
        # a step whose tokens were not kept gives its pages back first, so that every pass has the same to do
        stage.kv_release(s["rows"], s["have"], s["table"], s["counts"])
        stage.kv_extend(s["rows"], s["have"], s["new"], s["table"], s["counts"], s["free"], s["n_free"], row_starts=s["begins"],
                        new_lens=s["lens"], seq=s["seq"], slots=s["slot"], free_end=s["used"])
        return s["begins"], s["seq"], s["slot"], s["lens"], s["used"], s["table"], s["counts"]
    return {"prefix": _plain_prefix, "verify": _plain_verify, "norm": _plain_norm, "extend": _plain_extend}[op](s)


# ------------------------------------------------------------------------------------- work ---

def work(case):
    op = case["op"]
    if op == "prefix":
        Hq, Hkv, D, B, G, W = (case[k] for k in ("heads", "kv_heads", "dim", "batch", "groups", "window"))
        pre = (case["pre_lo"] + case["pre_hi"]) / 2 + (case["pre_hi"] - case["pre_lo"]) / 2 / G
        mine = (case["own_lo"] + case["own_hi"]) / 2 + (case["own_hi"] - case["own_lo"]) / 2 / B
        if W:
            mine, pre = min(mine, W), min(pre, max(0.0, W - mine))
        return {"bytes": (G * pre + B * mine) * Hkv * D * 4 + B * Hq * (D * 4 + 4), "flops": 4 * B * (pre + mine) * Hq * D}
    if op == "verify":
        B, T, V, width = case["batch"], case["nodes"], case["vocab"], 4 if case["dtype"] == "f32" else 2
        # the row that the next token is drawn from; where a branch was refused there, the drafter's too: about every second time
        rows = 1.0 if case["draw"] == "certain" else 1.5
        return {"bytes": B * (rows * V * width + T * (3 * 4 + 2 * width + 4) + 12), "flops": B * V * 3}
    if op == "norm":
        Hq, Hkv, D = case["heads"], case["kv_heads"], case["dim"]
        return {"bytes": case["rows"] * (2 * (Hq + 2 * Hkv) * D * 2 + 12), "flops": case["rows"] * (Hq + Hkv) * (case["rotary"] * 3 + 4 * D)}
    n, m = case["requests"], case["prompts"]
    new = (n - m) + m * (1 + case["tokens"]) / 2
    pages = (n - m) / PAGE + m * (1 + case["tokens"]) / 2 / PAGE
    # requests, lengths, places of all rows, new entries with their counts, taken back and given
    return {"bytes": n * 20 + (n + m * case["tokens"]) * 8 + pages * 28 + n * 4, "flops": new}


# ------------------------------------------------------------------------------------ exact ---

def _rows_of(table_row, lo, n, Hkv, D):
    """Element offsets of cached rows [lo, n) of one sequence, from the layout's definition: [n - lo, Hkv, 2, D]."""
    j = np.arange(lo, n)
    d = np.arange(D)
    chunk = ((d[None] >> 3) ^ (j[:, None] & 7)) * 8 + (d[None] & 7)
    tile = table_row[j // PAGE].astype(np.int64)[:, None, None] * Hkv + np.arange(Hkv)[None, :, None]
    at = ((tile * 2 + np.arange(2)[None, None]) * PAGE + (j % PAGE)[:, None, None])[..., None] * D + chunk[:, None, None]
    return torch.from_numpy(at).cuda()


def exact(case, seed):
    op = case["op"]
    if op not in ("prefix", "norm"):
        return None
    s = prepare(case, seed)
    Hkv, D, table = case["kv_heads"], case["dim"], s["table"].cpu().numpy()
    if op == "prefix":                                        # every row by itself, over all of its keys
        B, Hq, W, lens = case["batch"], case["heads"], case["window"], s["lens"].tolist()
        out = torch.zeros(B, Hq, D, dtype=torch.float64, device="cuda")
        lse = torch.zeros(B, Hq, dtype=torch.float64, device="cuda")
        for b in range(B):
            rows = s["pool"][_rows_of(table[b], max(0, lens[b] - W) if W else 0, lens[b], Hkv, D)].double()
            x = torch.einsum("hgd,khd->hgk", s["q"][b].double().view(Hkv, -1, D), rows[:, :, 0]) / math.sqrt(D)
            lse[b] = torch.logsumexp(x, -1).view(Hq)
            out[b] = torch.einsum("hgk,khd->hgd", torch.softmax(x, -1), rows[:, :, 1]).reshape(Hq, D)
        return out, lse
    rot = case["rotary"]
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["f"])

    def turn(x, w):
        y = x.double()
        y = (w.double() * y / torch.sqrt(y.square().sum(-1, keepdim=True) / D + 1e-6)).contiguous()
        if case["layout"] == "half":
            t = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * z[:, None]
            y[..., :rot // 2], y[..., rot // 2:rot] = t.real, t.imag
        else:
            t = torch.view_as_complex(y[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * z[:, None]
            y[..., :rot] = torch.view_as_real(t).flatten(-2)
        return y

    pool, k = s["pool"].double(), turn(s["k"], s["wk"])
    slot, seq = s["slot"].cpu().numpy(), s["seq"].cpu().numpy()
    for b in range(case["seqs"]):
        mine = np.nonzero(seq == b)[0]
        r = torch.from_numpy(mine).cuda()
        pool[_rows_of(table[b], int(slot[mine[0]]), int(slot[mine[-1]]) + 1, Hkv, D)] = torch.stack([k[r], s["v"][r].double()], 2)
    return turn(s["q"], s["wq"]), pool
