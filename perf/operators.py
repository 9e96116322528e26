"""Cases and plain forms of the operators that run around a verification call: attention of a drafted block over a
paged cache, rotary positions, and the cache's pages (reserve, append, commit, fork, truncate).

Layouts are the library's: K and V pages [layers, pages, kv_heads, page_size, head_dim]; page_table [seqs, max_pages]
(-1: no page); seq_len, held [seqs]; refs [pages] owners of a page; free_bits [ceil(pages / 32)] bit set = page free.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token of one conversation, the call of a plain decoding step: latency alone
        dict(name="attend one token", op="attend", B=1, T=1, q_heads=32, kv_heads=8, D=128, ctx_lo=701, ctx_hi=701, page=16, dtype="bf16", tree="chain"),
        # a batch of chains of 8 drafted tokens behind the last context token, narrow heads, ragged contexts
        dict(name="attend chains, narrow heads", op="attend", B=16, T=9, q_heads=32, kv_heads=8, D=64, ctx_lo=90, ctx_hi=6000, page=32, dtype="bf16", tree="chain"),
        # trees of 25 drafted tokens, a few long conversations
        dict(name="attend trees", op="attend", B=4, T=26, q_heads=64, kv_heads=8, D=128, ctx_lo=9000, ctx_hi=40000, page=64, dtype="bf16", tree="per_seq"),
        # one tree at the end of a very long context, 128 query heads: the largest call
        dict(name="attend long context", op="attend", B=1, T=26, q_heads=128, kv_heads=8, D=128, ctx_lo=131046, ctx_hi=131046, page=16, dtype="bf16", tree="shared"),
        # single precision, odd sizes
        dict(name="attend f32, odd sizes", op="attend", B=3, T=5, q_heads=6, kv_heads=2, D=80, ctx_lo=0, ctx_hi=1500, page=8, dtype="f32", tree="shared"),
        # a long prompt's queries and keys, scaled frequencies, positions up to the end of the context window
        dict(name="rotate prompt", op="rotate", N=16384, heads=40, D=128, rot=128, layout="half", dtype="bf16", inverse=False, far=131072),
        # gradient of a partial, interleaved rotation in single precision
        dict(name="rotate gradient f32", op="rotate", N=1001, heads=12, D=80, rot=64, layout="interleaved", dtype="f32", inverse=True, far=20000),
        # one token's key and value into the cache
        dict(name="append one token", op="append", B=1, T=1, q_heads=32, kv_heads=8, D=128, rot=128, layout="half", ctx_lo=1000, ctx_hi=1000, page=16, dtype="bf16"),
        # a batch of drafted trees into the cache
        dict(name="append batch", op="append", B=64, T=26, q_heads=64, kv_heads=8, D=128, rot=128, layout="half", ctx_lo=20, ctx_hi=900, page=64, dtype="bf16"),
        # rewind, reserve, commit of one conversation's chain in all layers
        dict(name="step one chain", op="step", L=32, B=1, T=9, paths=1, kv_heads=8, D=128, ctx_lo=300, ctx_hi=300, page=16, dtype="bf16"),
        # the same for a batch of trees, the longest accepted path of four kept
        dict(name="step trees", op="step", L=32, B=64, T=26, paths=4, kv_heads=8, D=128, ctx_lo=50, ctx_hi=250, page=32, dtype="bf16"),
        # every conversation forked into several, whose last pages are copied before they are written
        dict(name="fork", op="fork", L=32, B=3, copies=8, T=17, kv_heads=8, D=128, ctx_lo=1000, ctx_hi=5000, page=64, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "rotate", "append", "step", "fork"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    page = rng.choice([8, 16, 32, 64, 128])
    kv = rng.choice([1, 2, 4, 8])
    D = rng.choice([64, 128]) if dtype == "bf16" else rng.choice([40, 64, 80, 128])
    layout = rng.choice(["half", "interleaved"])
    if op == "rotate":
        heads = _log(rng, 1, 80)
        return dict(op=op, N=_log(rng, 1, 16384 * 40 // heads // 2), heads=heads, D=D, rot=rng.choice([D, D // 2]), layout=layout, dtype=dtype,
                    inverse=rng.random() < 0.5, far=_log(rng, 100, 1000000))
    T = rng.choice([1, 5, 9, 17, 26, _log(rng, 1, 64), _log(rng, 1, 128)])
    if op == "attend":
        group = rng.choice([1, 2, 4, 5, 8, 16])
        most = (1 << 28) // (T * group * kv) // (1 if dtype == "bf16" else 16)     # scores: no more than the longest listed call has
        hi = _log(rng, 16, min(100000, most))
        B = _log(rng, 1, max(1, min(64, most // hi, (1 << 31) // (hi * kv * D * 8))))
        return dict(op=op, B=B, T=T, q_heads=kv * group, kv_heads=kv, D=D, ctx_lo=rng.choice([0, hi // 3, hi]), ctx_hi=hi, page=page, dtype=dtype,
                    tree=rng.choice(["chain", "shared", "per_seq"]))
    hi = _log(rng, 1, 600)
    if op == "append":
        return dict(op=op, B=_log(rng, 1, 64), T=T, q_heads=kv * rng.choice([1, 4, 8]), kv_heads=kv, D=D, rot=rng.choice([D, D // 2]), layout=layout,
                    ctx_lo=hi // 4, ctx_hi=hi, page=page, dtype=dtype)
    if op == "step":
        return dict(op=op, L=_log(rng, 1, 32), B=_log(rng, 1, 40), T=T, paths=1 if T == 1 else rng.choice([1, 2, 4]), kv_heads=kv, D=D, ctx_lo=hi // 4, ctx_hi=hi, page=page, dtype=dtype)
    return dict(op=op, L=_log(rng, 1, 32), B=_log(rng, 1, 4), copies=_log(rng, 1, 8), T=T, kv_heads=kv, D=D, ctx_lo=hi // 4, ctx_hi=hi, page=page, dtype=dtype)


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(c):
    """Context lengths of the case's sequences: spread evenly over the range, the same for every seed."""
    return [c["ctx_lo"] + (c["ctx_hi"] - c["ctx_lo"]) * (c["B"] - 1 - b) // max(1, c["B"] - 1) for b in range(c["B"])]


def _pages(n, page):
    return -(-n // page)


def _cache(c, gen, lens, room, layers, extra_seqs=0, spare=0):
    """A cache that holds lens[b] tokens and room for `room` more of each sequence, its pages scattered over the pool."""
    S, page = len(lens) + extra_seqs, c["page"]
    want = [_pages(n + room, page) if room else _pages(n, page) for n in lens]
    P = sum(want) + spare + 1
    most = max([_pages(n + c["T"], page) for n in lens] + [1])
    order = torch.randperm(P, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((S, most), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(want):
        table[b, :n] = order[at:at + n]
        at += n
    refs = torch.zeros(P, dtype=torch.int32, device=DEV)
    refs[order[:at].long()] = 1
    shape = (layers, P, c["kv_heads"], page, c["D"])
    s = dict(table=table, refs=refs, k=torch.randn(shape, generator=gen, device=DEV, dtype=DT[c["dtype"]]), v=torch.randn(shape, generator=gen, device=DEV, dtype=DT[c["dtype"]]))
    s["len"] = torch.tensor(lens + [0] * extra_seqs, dtype=torch.int32, device=DEV)
    s["held"] = torch.tensor(want + [0] * extra_seqs, dtype=torch.int32, device=DEV)
    bits = torch.zeros(-(-P // 32) * 32, dtype=torch.int64, device=DEV)
    bits[:P] = refs == 0
    words = (bits.view(-1, 32) << torch.arange(32, device=DEV)).sum(1)
    s["free"] = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
    return s


def _parents(T, gen, n):
    """Random trees: the parent of node i is one of the nodes before it, most often a near one."""
    i = torch.arange(T)
    back = torch.rand(n, T, generator=gen).mul(4).floor().long() + 1
    return torch.clamp(i[None, :] - back, min=0) * (i > 0) - (i == 0).long()


def _visible(parents):
    """[n, T, T] truth values (node i sees its ancestors and itself) and depths [n, T]."""
    n, T = parents.shape
    see = torch.zeros(n, T, T, dtype=torch.bool)
    for i in range(T):
        if i:
            see[:, i] = see[torch.arange(n), parents[:, i]]
        see[:, i, i] = True
    return see, (see.sum(2) - 1).to(torch.int32)


def _words(see):
    n, T, _ = see.shape
    W = -(-T // 32)
    b = torch.zeros(n, T, W * 32, dtype=torch.int64)
    b[:, :, :T] = see
    w = (b.view(n, T, W, 32) << torch.arange(32)).sum(3)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _freqs(rot, scaled):
    f = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if scaled:       # long wavelengths stretched eightfold, short ones kept, a linear blend between
        turns = 8192 * f / (2 * math.pi)
        keep = ((turns - 1) / 3).clamp(0, 1)
        f = f * (keep + (1 - keep) / 8)
    return f.to(torch.float32).to(DEV)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    host = torch.Generator()
    host.manual_seed(seed)
    op, dt = c["op"], DT[c["dtype"]]
    s = dict(c=c)
    if op == "rotate":
        s["freq"] = _freqs(c["rot"], c["far"] > 8192)
        s["x"] = torch.randn(c["N"], c["heads"], c["D"], generator=gen, device=DEV, dtype=dt)
        s["pos"] = torch.randint(0, c["far"], (c["N"],), generator=gen, device=DEV, dtype=torch.int32)
        if own:
            from paper_2501_19309_b200 import jd
            s["rotary"] = jd.Rotary(s["freq"], layout=c["layout"], amplitude=1.0)
            s["out"] = torch.empty_like(s["x"])
        return s
    lens = _lengths(c)
    B, T, page = c["B"], c["T"], c["page"]
    if op == "attend":
        s |= _cache(c, gen, lens, T, 1)
        s["q"] = torch.randn(B, T, c["q_heads"], c["D"], generator=gen, device=DEV, dtype=dt)
        n = {"chain": 0, "shared": 1, "per_seq": B}[c["tree"]]
        s["see"] = s["words"] = None
        if n:
            see, depth = _visible(_parents(T, host, n))
            s["words"] = _words(see).to(DEV) if n > 1 or c["tree"] == "per_seq" else _words(see)[0].to(DEV)
            s["see"], s["depth"] = see.to(DEV), depth.to(DEV)
        else:
            s["see"] = torch.ones(1, T, T, dtype=torch.bool, device=DEV).tril()
        s["most"] = max(_pages(n + T, page) for n in lens)
    elif op == "append":
        s |= _cache(c, gen, lens, T, 2)
        s["freq"] = _freqs(c["rot"], False)
        s["q"] = torch.randn(B, T, c["q_heads"], c["D"], generator=gen, device=DEV, dtype=dt)
        s["nk"] = torch.randn(B, T, c["kv_heads"], c["D"], generator=gen, device=DEV, dtype=dt)
        s["nv"] = torch.randn(B, T, c["kv_heads"], c["D"], generator=gen, device=DEV, dtype=dt)
        see, depth = _visible(_parents(T, host, 1))
        s["words"], s["depth"] = _words(see)[0].to(DEV), depth[0].to(DEV)
    elif op == "step":
        s |= _cache(c, gen, lens, 0, c["L"], spare=sum(_pages(n + T, page) - _pages(n, page) for n in lens) + 2)
        s["base"] = s["len"].clone()
        M = T - 1
        # strictly rising node numbers of every root-to-leaf path, and how many of each were accepted
        picks = torch.rand(B, c["paths"], max(M, 1), generator=host).argsort(2).add(1)
        depth = max(1, min(M, 2 + M // 2)) if c["paths"] > 1 else max(M, 1)
        paths = picks[:, :, :depth].sort(2).values.to(torch.int32)
        s["paths"] = paths.to(DEV) if c["paths"] > 1 else None
        s["accept"] = torch.randint(0, min(M, depth) + 1, (B, c["paths"]), generator=host).to(torch.int32).to(DEV)
    elif op == "fork":
        n = c["copies"]
        s |= _cache(c, gen, lens, 0, c["L"], extra_seqs=B * n, spare=sum(n * (_pages(x + T, page) - x // page) for x in lens) + 2)
        s["src"] = torch.arange(B, dtype=torch.int32, device=DEV).repeat_interleave(n)
        s["dst"] = torch.arange(B, B + B * n, dtype=torch.int32, device=DEV)
    if own:
        from paper_2501_19309_b200 import jd
        s["cache"] = jd.PagedCache(s["k"], s["v"], s["table"], s["len"], s["held"], s["refs"], s["free"], q_heads=c.get("q_heads", c["kv_heads"]), max_nodes=T)
        if op == "attend":
            s["tree"] = jd.Tree(T, mask=s["words"])
            s["out"] = dict(out=torch.empty_like(s["q"]), lse=torch.empty(B, T, c["q_heads"], device=DEV))
        if op == "append":
            s["rotary"] = jd.Rotary(s["freq"], layout=c["layout"], amplitude=1.0)
            s["tree"] = jd.Tree(T, mask=s["words"], depth=s["depth"])
            s["q_out"] = torch.empty_like(s["q"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _rotate(x, angle, layout, inverse):
    """x [..., heads, D] in 32 bits, angle [..., rot / 2] in 64: the first rot elements of every head rotated."""
    half = angle.shape[-1]
    cos, sin = torch.cos(angle).float().unsqueeze(-2), torch.sin(angle).float().unsqueeze(-2)
    if inverse:
        sin = -sin
    x = x.float()
    part, rest = x[..., :2 * half], x[..., 2 * half:]
    if layout == "half":
        a, b = part[..., :half], part[..., half:]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((y, rest), -1)


def _plain_attend(s):
    c = s["c"]
    B, T, H, Hq, D = c["B"], c["T"], c["kv_heads"], c["q_heads"], c["D"]
    pt = s["table"][:, :s["most"]].clamp(min=0).long()
    N = s["most"] * c["page"]
    ctx = s["len"].long()
    at = torch.arange(N, device=DEV)[None, :] - ctx[:, None]                        # node number of a cached row, < 0: context
    there = at < T
    node = at.clamp(0, T - 1)
    see = torch.gather(s["see"].expand(B, T, T), 2, node[:, None, :].expand(B, T, N))
    see = ((at < 0)[:, None, :] | see) & there[:, None, :]
    k = s["k"][0][pt].permute(0, 2, 1, 3, 4).reshape(B, H, N, D).float()
    q = s["q"].float().reshape(B, T, H, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)
    sc = (q @ k.transpose(2, 3)).mul_(D ** -0.5)
    del k
    sc = sc.view(B, H, T, Hq // H, N).masked_fill_(~see[:, None, :, None, :], -math.inf)
    m = sc.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = sc.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    v = s["v"][0][pt].permute(0, 2, 1, 3, 4).reshape(B, H, N, D).float().masked_fill_(~there[:, None, :, None], 0.0)
    o = (p.view(B, H, -1, N) @ v).view(B, H, T, Hq // H, D)
    o = torch.where(l > 0, o / l, torch.zeros_like(o))
    lse = (m + l.log()).squeeze(-1)
    return dict(out=o.permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D).to(s["q"].dtype), lse=lse.permute(0, 2, 1, 3).reshape(B, T, Hq).contiguous())


def _plain_append(s):
    c = s["c"]
    pos = s["len"].long()[:, None] + s["depth"].long()[None, :]
    angle = pos.double()[..., None] * s["freq"].double()
    at = s["len"].long()[:, None] + torch.arange(c["T"], device=DEV)
    page = torch.gather(s["table"].long(), 1, at // c["page"])
    row = at % c["page"]
    s["k"][1][page, :, row] = _rotate(s["nk"], angle, c["layout"], False).to(s["k"].dtype)
    s["v"][1][page, :, row] = s["nv"]
    return _rotate(s["q"], angle, c["layout"], False).to(s["q"].dtype)


def _plain_free_words(refs):
    n = refs.numel()
    b = torch.zeros(-(-n // 32) * 32, dtype=torch.int64, device=refs.device)
    b[:n] = refs == 0
    w = (b.view(-1, 32) << torch.arange(32, device=refs.device)).sum(1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _plain_release(s, rows, keep):
    """Pages keep[i].. of the sequences rows[i] lose an owner and leave the table."""
    col = torch.arange(s["table"].shape[1], device=DEV)[None, :]
    t = s["table"][rows].long()
    gone = (col >= keep[:, None]) & (col < s["held"][rows][:, None])
    s["refs"].index_add_(0, t.clamp(min=0).flatten(), -gone.flatten().to(torch.int32))
    s["table"][rows] = torch.where(gone, -1, t).to(torch.int32)
    s["held"][rows] = torch.minimum(s["held"][rows].long(), keep).to(torch.int32)


def _plain_truncate(s, rows, length):
    page = s["c"]["page"]
    _plain_release(s, rows, (length.long() + page - 1) // page)
    s["len"][rows] = length.to(torch.int32)


def _plain_reserve(s, rows, n):
    """Pages for n more tokens; a page that others own too is copied first where its rest is about to be written. Lowest free pages first."""
    page = s["c"]["page"]
    ln, held = s["len"][rows].long(), s["held"][rows].long()
    want = torch.maximum((ln + n + page - 1) // page, held)
    last, part = ln // page, ln % page
    t = s["table"][rows].long()
    lastp = torch.gather(t, 1, last.clamp(max=t.shape[1] - 1)[:, None])[:, 0]
    shared = (part > 0) & (lastp >= 0)
    before = ((lastp[:, None] == lastp[None, :]) & shared[None, :]).tril(-1).sum(1)
    copy = shared & (s["refs"][lastp.clamp(min=0)].long() - before > 1)
    col = torch.arange(t.shape[1], device=DEV)[None, :]
    new = (copy[:, None] & (col == last[:, None])) | ((col >= held[:, None]) & (col < want[:, None]))
    order = torch.argsort((s["refs"] != 0).to(torch.int8), stable=True)
    rank = (new.flatten().long().cumsum(0) - 1).clamp(min=0).view_as(t)
    got = torch.where(new, order[rank.clamp(max=order.numel() - 1)], t)
    s["refs"].index_add_(0, got.clamp(min=0).flatten(), new.flatten().to(torch.int32))
    s["refs"].index_add_(0, lastp.clamp(min=0), -copy.to(torch.int32))
    s["table"][rows] = got.to(torch.int32)
    s["held"][rows] = want.to(torch.int32)
    to = torch.gather(got, 1, last.clamp(max=t.shape[1] - 1)[:, None])[:, 0].clamp(min=0)
    take = copy[:, None] & (torch.arange(page, device=DEV)[None, :] < part[:, None])
    for x in (s["k"], s["v"]):
        src = x[:, lastp.clamp(min=0)]
        x[:, to] = torch.where(take[None, :, None, :, None], src, x[:, to])


def _plain_commit(s, rows):
    c = s["c"]
    page, n = c["page"], s["accept"].shape[0]
    best = s["accept"].max(1)
    chosen = (s["accept"] == best.values[:, None]).to(torch.int8).argmax(1)
    a = best.values.long()
    ln = s["len"][rows].long()
    if s["paths"] is not None:
        path = s["paths"][torch.arange(n, device=DEV), chosen].long()
        i = torch.arange(path.shape[1], device=DEV)[None, :]
        ok = i < a[:, None]
        src = torch.where(ok, ln[:, None] + path, ln[:, None])
        dst = torch.where(ok, ln[:, None] + 1 + i, ln[:, None])
        t = s["table"][rows].long()
        sp, dp = torch.gather(t, 1, src // page), torch.gather(t, 1, dst // page)
        for x in (s["k"], s["v"]):
            x[:, dp, :, dst % page] = x[:, sp, :, src % page]
    new = ln + a + 1
    s["len"][rows] = new.to(torch.int32)
    _plain_release(s, rows, (new + page - 1) // page)
    return chosen.to(torch.int32)


def _state(s):
    return dict(k=s["k"], v=s["v"], table=s["table"], len=s["len"], held=s["held"], refs=s["refs"], free=s["free"])


def run(state):
    s, c = state, state["c"]
    op = c["op"]
    if op == "rotate":
        if own:
            return s["rotary"].rotate(s["x"], s["pos"], out=s["out"], inverse=c["inverse"])
        return _rotate(s["x"], s["pos"].double()[:, None] * s["freq"].double(), c["layout"], c["inverse"]).to(s["x"].dtype)
    if op == "attend":
        return s["cache"].attend(0, s["q"], s["tree"], out=s["out"]) if own else _plain_attend(s)
    if op == "append":
        q = s["cache"].append(1, s["nk"], s["nv"], s["tree"], rotary=s["rotary"], q=s["q"], q_out=s["q_out"]) if own else _plain_append(s)
        return dict(q=q, k=s["k"][1], v=s["v"][1])
    if op == "step":
        if own:
            s["cache"].truncate(s["base"])
            s["cache"].reserve(c["T"])
            chosen = s["cache"].commit(s["accept"], s["paths"])
        else:
            rows = torch.arange(c["B"], device=DEV)
            _plain_truncate(s, rows, s["base"])
            _plain_reserve(s, rows, c["T"])
            chosen = _plain_commit(s, rows)
            s["free"].copy_(_plain_free_words(s["refs"]))
        return dict(_state(s), chosen=chosen)
    if own:
        s["cache"].free(s["dst"])
        s["cache"].fork(s["src"], s["dst"])
        s["cache"].reserve(c["T"], slots=s["dst"])
    else:
        dst, src = s["dst"].long(), s["src"].long()
        _plain_truncate(s, dst, torch.zeros_like(dst))
        s["table"][dst] = s["table"][src]
        s["len"][dst] = s["len"][src]
        s["held"][dst] = s["held"][src]
        t = s["table"][src].long()
        s["refs"].index_add_(0, t.clamp(min=0).flatten(), (t >= 0).flatten().to(torch.int32))
        _plain_reserve(s, dst, c["T"])
        s["free"].copy_(_plain_free_words(s["refs"]))
    return _state(s)


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The same outputs from the definitions, one sequence and one key head at a time; nothing for outputs that are only moved."""
    c = case
    if c["op"] in ("step", "fork"):
        return None
    s = prepare(c, seed)
    if c["op"] == "rotate":
        return _exact_rotation(s["x"], s["pos"], s["freq"], c["layout"], -1.0 if c["inverse"] else 1.0)
    if c["op"] == "append":
        pos = torch.stack([s["len"] + d for d in s["depth"]], 1)
        kc, vc = s["k"][1].double(), s["v"][1].double()
        rk = _exact_rotation(s["nk"], pos, s["freq"], c["layout"], 1.0)
        for b, n in enumerate(_lengths(c)):
            for t in range(c["T"]):
                p = int(s["table"][b, (n + t) // c["page"]])
                kc[p, :, (n + t) % c["page"]] = rk[b, t]
                vc[p, :, (n + t) % c["page"]] = s["nv"][b, t].double()
        return dict(q=_exact_rotation(s["q"], pos, s["freq"], c["layout"], 1.0), k=kc, v=vc)
    B, T, H, G, D = c["B"], c["T"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["D"]
    out = torch.zeros(B, T, H * G, D, dtype=torch.float64, device=DEV)
    lse = torch.full((B, T, H * G), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(c)):
        pages = s["table"][b, :_pages(n + T, c["page"])].long()
        bias = torch.zeros(T, n + T, dtype=torch.float64, device=DEV)
        bias[:, n:][~s["see"][b if s["see"].shape[0] > 1 else 0]] = -math.inf
        for h in range(H):
            keys = s["k"][0, pages, h].reshape(-1, D)[:n + T].double()
            vals = s["v"][0, pages, h].reshape(-1, D)[:n + T].double()
            z = torch.einsum("tgd,nd->gtn", s["q"][b, :, h * G:(h + 1) * G].double(), keys) / math.sqrt(D) + bias
            lse[b, :, h * G:(h + 1) * G] = torch.logsumexp(z, 2).T
            out[b, :, h * G:(h + 1) * G] = torch.einsum("gtn,nd->tgd", torch.softmax(z, 2), vals)
    return dict(out=out, lse=lse)


def _exact_rotation(x, pos, freq, layout, sign):
    y = x.double().clone()
    turn = torch.exp(1j * sign * pos.double().unsqueeze(-1) * freq.double()).unsqueeze(-2)
    n = freq.numel()
    re, im = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    z = torch.complex(x[..., re].double(), x[..., im].double()) * turn
    y[..., re], y[..., im] = z.real, z.imag
    return y


# ------------------------------------------------------------------------------------------------ floors
def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "rotate":
        n = c["N"] * c["heads"] * c["D"]
        return dict(bytes=2 * n * e + 4 * c["N"], flops=3 * c["N"] * c["heads"] * c["rot"])
    lens, T, H, D, page = _lengths(c), c["T"], c["kv_heads"], c["D"], c["page"]
    if c["op"] == "attend":
        rows = sum(n + T for n in lens)
        q = c["B"] * T * c["q_heads"]
        return dict(bytes=2 * rows * H * D * e + 2 * q * D * e + 4 * q + 4 * sum(_pages(n + T, page) for n in lens), flops=4 * T * c["q_heads"] * D * rows)
    if c["op"] == "append":
        n = c["B"] * T * D
        return dict(bytes=2 * n * (c["q_heads"] + 2 * H) * e, flops=3 * c["B"] * T * c["rot"] * (c["q_heads"] + H))
    if c["op"] == "step":      # half of the longest path's rows, read and written, and the tables
        rows = c["B"] * (min(T - 1, 2 + (T - 1) // 2) / 2 if c["paths"] > 1 else 0)
        return dict(bytes=2 * 2 * rows * c["L"] * H * D * e + 32 * c["B"], flops=0)
    moved = sum(c["copies"] * (n % page) for n in lens)
    return dict(bytes=2 * 2 * moved * c["L"] * H * D * e + 8 * sum(c["copies"] * _pages(n, page) for n in lens) + 32 * c["B"] * c["copies"], flops=0)
