"""Cases and plain forms of operators of a decoding step: norms of query and key heads with their rotation (several position axes
among them) in one pass, alone, on the way into the cache and backwards; attention of sequences that share a long prefix; and the
verification of drafted chains and trees against the target's probabilities from given random numbers.

Layouts are the library's: heads [tokens, heads, head_dim]; K and V pages [layers, pages, kv_heads, page_size, head_dim]; page_table
[seqs, max_pages] (-1: no page); seq_len, held [seqs]; probabilities [seqs, nodes, vocabulary], node 0 the last context token.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a long prompt's queries and keys, out of the projection that holds values too
        dict(name="heads of a prompt", op="heads", N=16384, q_heads=32, kv_heads=8, D=128, rot=128, layout="half", sections="", dtype="bf16", far=131072),
        # an image's tokens in single precision, time, height and width as axes, odd sizes
        dict(name="heads of an image f32", op="heads", N=1373, q_heads=12, kv_heads=3, D=80, rot=64, layout="interleaved", sections="8,12,12", dtype="f32", far=4000),
        # training on video: the same backwards, with the gradients of the norms' weights
        dict(name="heads backward, three axes", op="heads_grad", N=8192, q_heads=32, kv_heads=8, D=128, rot=128, layout="half", sections="16,24,24", dtype="bf16", far=32768),
        # a short training sequence in single precision, partial rotation
        dict(name="heads backward f32, odd sizes", op="heads_grad", N=1001, q_heads=12, kv_heads=3, D=80, rot=64, layout="half", sections="", dtype="f32", far=20000),
        # one token's queries, key and value on their way into the cache
        dict(name="append one token, norms", op="append", B=1, T=1, q_heads=32, kv_heads=8, D=128, rot=128, layout="half", sections="", ctx_lo=1000, ctx_hi=1000, page=16, dtype="bf16"),
        # a batch of drafted trees behind images: positions given on three axes
        dict(name="append trees, three axes", op="append", B=64, T=26, q_heads=64, kv_heads=8, D=128, rot=128, layout="half", sections="16,24,24", ctx_lo=20, ctx_hi=900, page=64, dtype="bf16"),
        # sixteen samples of one prompt, a token each
        dict(name="shared prompt, one token each", op="shared", L=4, B=16, convs=1, T=1, q_heads=32, kv_heads=8, D=128, prefix=1900, own_lo=40, own_hi=300, page=16, dtype="bf16"),
        # requests behind one long system prompt, chains of drafted tokens
        dict(name="shared long prompt, chains", op="shared", L=2, B=32, convs=1, T=9, q_heads=64, kv_heads=8, D=128, prefix=32768, own_lo=90, own_hi=1500, page=64, dtype="bf16"),
        # two conversations forked into three each, in single precision, odd sizes
        dict(name="shared forks f32, odd sizes", op="shared", L=4, B=6, convs=2, T=5, q_heads=6, kv_heads=2, D=80, prefix=1501, own_lo=0, own_hi=77, page=8, dtype="f32"),
        # one conversation's chain of drafted tokens
        dict(name="verify one chain", op="verify", B=1, T=9, V=128256, tree="chain", siblings="independent", mode="standard", dtype="f32"),
        # a batch of chains, accepted by a judge's scores too
        dict(name="verify chains", op="verify", B=64, T=17, V=128256, tree="chain", siblings="independent", mode="judge_or_standard", dtype="f32"),
        # a batch of drafted trees, siblings drawn without replacement
        dict(name="verify trees", op="verify", B=16, T=26, V=128256, tree="per_seq", siblings="distinct", mode="standard", dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _sections(rng, half):
    if rng.random() < 0.5 or half < 4:
        return ""
    a = rng.randint(1, half - 2)
    b = rng.randint(1, half - a - 1) if rng.random() < 0.7 else half - a
    return ",".join(str(x) for x in (a, b, half - a - b) if x)


def draw(rng):
    op = rng.choice(["heads", "heads_grad", "append", "shared", "shared", "verify", "verify"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    page = rng.choice([8, 16, 32, 64, 128])
    kv = rng.choice([1, 2, 3, 4, 8])
    group = rng.choice([1, 2, 4, 5, 8])
    D = rng.choice([64, 128]) if dtype == "bf16" else rng.choice([40, 64, 80, 128])
    rot = rng.choice([D, D, D // 2])
    layout = rng.choice(["half", "interleaved"])
    sections = _sections(rng, rot // 2)
    if op in ("heads", "heads_grad"):
        most = 16384 * 40 * 128 if op == "heads" else 8192 * 40 * 128
        return dict(op=op, N=_log(rng, 1, most // (kv * (group + 1) * D) // (1 if dtype == "bf16" else 2)), q_heads=kv * group, kv_heads=kv, D=D, rot=rot,
                    layout=layout, sections=sections, dtype=dtype, far=_log(rng, 100, 1000000))
    T = rng.choice([1, 1, 5, 9, 17, 26, _log(rng, 1, 64)])
    if op == "append":
        hi = _log(rng, 1, 600)
        return dict(op=op, B=_log(rng, 1, 64), T=T, q_heads=kv * group, kv_heads=kv, D=D, rot=rot, layout=layout, sections=sections, ctx_lo=hi // 4, ctx_hi=hi,
                    page=page, dtype=dtype)
    if op == "shared":
        convs = rng.choice([1, 1, 1, 2, 3])
        B = convs * _log(rng, 2, 32 // convs)
        hi = _log(rng, 1, 1500)
        rows = (1 << 29) // (1 if dtype == "bf16" else 16)          # scores of a layer: no more than the largest listed call has
        prefix = _log(rng, 100, max(128, min(32768, rows // (B * T * kv * group) - hi)))
        return dict(op=op, L=rng.choice([1, 2]), B=B, convs=convs, T=T, q_heads=kv * group, kv_heads=kv, D=D, prefix=prefix, own_lo=rng.choice([0, hi // 3, hi]), own_hi=hi,
                    page=page, dtype=dtype)
    tree = rng.choice(["chain", "chain", "shared", "per_seq"])
    V = _log(rng, 1000, 160000)
    T = _log(rng, 2, 33)
    return dict(op=op, B=_log(rng, 1, max(1, min(64, 64 * 17 * 128256 // (T * V) if tree == "chain" else 16 * 26 * 128256 // (T * V)))), T=T, V=V, tree=tree,
                siblings=rng.choice(["independent", "distinct"]), mode=rng.choice(["standard", "standard", "judge_or_standard", "judge"]), dtype=rng.choice(["f32", "f32", "bf16"]))


# ------------------------------------------------------------------------------------------------ inputs
def _pages(n, page):
    return -(-n // page)


def _lengths(c, lo, hi):
    """Numbers of tokens spread evenly over the range, the same for every seed."""
    return [lo + (hi - lo) * (c["B"] - 1 - b) // max(1, c["B"] - 1) for b in range(c["B"])]


def _axis_of(c):
    """The axis of every frequency; one axis: zeroes."""
    sizes = [int(x) for x in c["sections"].split(",")] if c["sections"] else [c["rot"] // 2]
    return [a for a, n in enumerate(sizes) for _ in range(n)]


def _head_inputs(s, c, gen, lead):
    """Norm weights near 1, frequencies, and queries and keys whose heads differ in size, out of one projection's rows."""
    D, Hq, Hk, dt = c["D"], c["q_heads"], c["kv_heads"], DT[c["dtype"]]
    rnd = lambda *shape: torch.randn(*shape, generator=gen, device=DEV)  # noqa: E731
    s["wq"], s["wk"] = 1 + 0.2 * rnd(D), 1 + 0.2 * rnd(D)
    s["freq"] = (500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])).float().to(DEV)
    s["axis"] = torch.tensor(_axis_of(c), device=DEV)
    size = torch.exp(rnd(Hq + 2 * Hk, 1))
    qkv = torch.randn(*lead, Hq + 2 * Hk, D, generator=gen, device=DEV, dtype=dt).mul_(size.to(dt))
    s["q"], s["nk"], s["nv"] = qkv[..., :Hq, :], qkv[..., Hq:Hq + Hk, :], qkv[..., Hq + Hk:, :]


def _parents(c, host, n):
    """Parents of n trees: most often a near node, so that siblings are few and paths are long; a chain: the node in front."""
    i = torch.arange(c["T"])
    if c.get("tree", "per_seq") == "chain":
        return (i - 1).expand(n, -1)
    back = torch.rand(n, c["T"], generator=host).mul(4).floor().long() + 1
    return torch.clamp(i - back, min=0) * (i > 0) - (i == 0).long()


def _cache(s, c, gen, table, lens, held, P, layers):
    shape = (layers, P, c["kv_heads"], c["page"], c["D"])
    s["k"] = torch.randn(shape, generator=gen, device=DEV, dtype=DT[c["dtype"]])
    s["v"] = torch.randn(shape, generator=gen, device=DEV, dtype=DT[c["dtype"]])
    s["table"] = table
    s["len"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["held"] = torch.tensor(held, dtype=torch.int32, device=DEV)
    s["refs"] = torch.bincount(table[table >= 0].long(), minlength=P).to(torch.int32)
    bits = torch.zeros(_pages(P, 32) * 32, dtype=torch.int64, device=DEV)
    bits[:P] = s["refs"] == 0
    words = (bits.view(-1, 32) << torch.arange(32, device=DEV)).sum(1)
    s["free"] = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def _prepare_append(s, c, gen, host):
    B, T, page = c["B"], c["T"], c["page"]
    lens = _lengths(c, c["ctx_lo"], c["ctx_hi"])
    held = [_pages(n + T, page) for n in lens]
    P = sum(held) + 1
    order = torch.randperm(P, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((B, max(held)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    _cache(s, c, gen, table, lens, held, P, 2)
    _head_inputs(s, c, gen, (B, T))
    depth = torch.zeros(T, dtype=torch.int32)
    for i, p in enumerate(_parents(c, host, 1)[0].tolist()):
        depth[i] = depth[p] + 1 if p >= 0 else 0
    s["depth"] = depth.to(DEV)
    # behind images a text token's position is less than the number of tokens, the same on every axis
    pos = s["len"][:, None] // 2 + s["depth"][None, :] if c["sections"] else s["len"][:, None] + s["depth"][None, :]
    s["pos"] = pos[..., None].expand(B, T, max(_axis_of(c)) + 1).to(torch.int32).contiguous()


def _prepare_shared(s, c, gen):
    B, T, page, pre = c["B"], c["T"], c["page"], c["prefix"]
    lens = [pre + n for n in _lengths(c, c["own_lo"], c["own_hi"])]
    held, common = [_pages(n + T, page) for n in lens], pre // page       # the page that a prefix ends in is a copy of each one's own
    P = c["convs"] * common + sum(n - common for n in held) + 1
    order = torch.randperm(P, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((B, max(held)), -1, dtype=torch.int32, device=DEV)
    at = c["convs"] * common
    for b, n in enumerate(held):
        conv = b % c["convs"]
        table[b, :common] = order[conv * common:(conv + 1) * common]
        table[b, common:n] = order[at:at + n - common]
        at += n - common
    _cache(s, c, gen, table, lens, held, P, c["L"])
    s["q"] = torch.randn(c["L"], B, T, c["q_heads"], c["D"], generator=gen, device=DEV, dtype=DT[c["dtype"]])
    s["most"] = max(held)


def _prepare_verify(s, c, gen, host):
    """Peaked distributions; the draft's is the target's with noise on its logits, and the drafted tokens are drawn from it."""
    B, T, V, dt = c["B"], c["T"], c["V"], DT[c["dtype"]]
    p, q = torch.empty(B, T, V, dtype=dt, device=DEV), torch.empty(B, T - 1, V, dtype=dt, device=DEV)
    n = {"chain": 1, "shared": 1, "per_seq": B}[c["tree"]]
    parents = _parents(c, host, n)
    rank = ((parents[:, :, None] == parents[:, None, :]) & (torch.arange(T)[None, None, :] < torch.arange(T)[None, :, None])).sum(2)     # elder siblings
    most = int(rank.max()) + 1
    parents, rank = parents.expand(B, T).to(DEV), rank.expand(B, T).to(DEV)
    s["tokens"] = torch.empty(B, T - 1, dtype=torch.int32, device=DEV)
    for b in range(B):
        z = torch.randn(T, V, generator=gen, device=DEV) * 3
        p[b] = torch.softmax(z, 1).to(dt)
        z = z[:-1] + torch.randn(T - 1, V, generator=gen, device=DEV) * 0.7
        q[b] = torch.softmax(z, 1).to(dt)
        w = q[b].float()
        if c["siblings"] == "distinct":
            picks = (w.log() - torch.empty_like(w).exponential_(generator=gen).log()).topk(most, 1).indices
        else:
            picks = torch.stack([(w.log() - torch.empty_like(w).exponential_(generator=gen).log()).argmax(1) for _ in range(most)], 1)
        s["tokens"][b] = picks[parents[b, 1:], rank[b, 1:]].to(torch.int32)
    s["p"], s["pd"] = p, q
    s["u"] = torch.rand(B, T - 1, generator=gen, device=DEV)
    s["us"] = torch.rand(B, generator=gen, device=DEV)
    s["judge"] = torch.rand(B, T - 1, generator=gen, device=DEV)
    s["tau"] = 0.5 if c["mode"] == "judge" else 0.8
    s["parents"] = None if c["tree"] == "chain" else (parents[0] if c["tree"] == "shared" else parents).to(torch.int32).contiguous()


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    host = torch.Generator()
    host.manual_seed(seed)
    s = dict(c=c)
    if c["op"] in ("heads", "heads_grad"):
        _head_inputs(s, c, gen, (c["N"],))
        axes, side = max(_axis_of(c)) + 1, max(1, math.isqrt(c["N"]))
        n = torch.arange(c["N"], device=DEV)
        start = torch.randint(0, c["far"], (1,), generator=gen, device=DEV)
        # a sequence's tokens in a row; with axes, of an image: the first axis stands, the others run over rows and columns
        s["pos"] = (start + n if axes == 1 else torch.stack([start + 0 * n, start + n // side, start + n % side][:axes], 1)).to(torch.int32)
        if c["op"] == "heads_grad":
            s["gq"], s["gk"] = (torch.randn(x.shape, generator=gen, device=DEV, dtype=x.dtype) for x in (s["q"], s["nk"]))
    elif c["op"] == "append":
        _prepare_append(s, c, gen, host)
    elif c["op"] == "shared":
        _prepare_shared(s, c, gen)
    else:
        _prepare_verify(s, c, gen, host)
    if own:      # what a program keeps: frequencies and weights as objects, the cache's handle, a plan's buffers
        from paper_2501_19309_b200 import jd
        if "freq" in s:
            s["rotary"] = jd.Rotary(s["freq"], layout=c["layout"], axes=_axis_of(c) if c["sections"] else None)
            s["norm"] = jd.HeadNorm(s["wq"], s["wk"], eps=1e-6)
        if "table" in s:
            s["cache"] = jd.PagedCache(s["k"], s["v"], s["table"], s["len"], s["held"], s["refs"], s["free"], q_heads=c["q_heads"], max_nodes=c["T"])
        if c["op"] == "append":
            s["tree"] = jd.Tree(c["T"], depth=s["depth"])
        if c["op"] == "shared":
            s["plan"] = s["cache"].share(c["T"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
EPS = 1e-6


def _turns(s):
    """Cosines and sines [..., rot / 2] of the tokens' angles, which are formed in 64 bits."""
    pos = s["pos"].double()
    at = pos[..., s["axis"]] if pos.dim() == s["q"].dim() - 1 else pos[..., None]
    angle = at * s["freq"].double()
    return torch.cos(angle).float().unsqueeze(-2), torch.sin(angle).float().unsqueeze(-2)


def _rotate(x, cos, sin, layout):
    half = cos.shape[-1]
    part, rest = x[..., :2 * half], x[..., 2 * half:]
    if layout == "half":
        a, b = part[..., :half], part[..., half:]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((y, rest), -1)


def _plain_heads(x, w, cos, sin, layout):
    x32 = x.float()
    r = torch.rsqrt(x32.square().mean(-1, keepdim=True) + EPS)
    return _rotate(x32 * r * w, cos, sin, layout).to(x.dtype)


def _plain_heads_grad(g, x, w, cos, sin, layout):
    g, x32 = _rotate(g.float(), cos, -sin, layout), x.float()
    r = torch.rsqrt(x32.square().mean(-1, keepdim=True) + EPS)
    n = x32 * r
    gw = g * w
    dx = r * (gw - n * (gw * n).mean(-1, keepdim=True))
    return dx.to(x.dtype), (g * n).sum((0, 1))


def _plain_shared(s, layer):
    c = s["c"]
    B, T, H, Hq, D = c["B"], c["T"], c["kv_heads"], c["q_heads"], c["D"]
    pt = s["table"][:, :s["most"]].clamp(min=0).long()
    N = s["most"] * c["page"]
    node = torch.arange(N, device=DEV)[None, :] - s["len"].long()[:, None]              # node number of a cached row, < 0: context
    see = node[:, None, :] <= torch.arange(T, device=DEV)[None, :, None]
    k = s["k"][layer][pt].permute(0, 2, 1, 3, 4).reshape(B, H, N, D).float()
    q = s["q"][layer].float().reshape(B, T, H, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)
    sc = (q @ k.transpose(2, 3)).mul_(D ** -0.5)
    del k
    sc = sc.view(B, H, T, Hq // H, N).masked_fill_(~see[:, None, :, None, :], -math.inf)
    m = sc.amax(-1, keepdim=True)
    p = sc.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    v = s["v"][layer][pt].permute(0, 2, 1, 3, 4).reshape(B, H, N, D).float()
    o = (p.view(B, H, -1, N) @ v).view(B, H, T, Hq // H, D) / l
    lse = (m + l.log()).squeeze(-1)
    return dict(out=o.permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D).to(s["q"].dtype), lse=lse.permute(0, 2, 1, 3).reshape(B, T, Hq).contiguous())


def _drawn(w, fallback, u):
    """The first token whose running sum of weights exceeds u of the whole; weights that are all zero give way to the fallback's."""
    total = w.sum(1, keepdim=True)
    w = torch.where(total > 0, w, fallback)
    run = w.cumsum(1)
    return (run <= u.double()[:, None] * run[:, -1:]).sum(1).clamp(max=w.shape[1] - 1).to(torch.int32)


def _plain_chain(s):
    c = s["c"]
    M = c["T"] - 1
    x = s["tokens"].long()[..., None]
    px, qx = (t[:, :M].gather(2, x)[..., 0].double() for t in (s["p"], s["pd"]))
    ok = s["u"].double() * qx < px
    if c["mode"] != "standard":
        judged = s["judge"] > s["tau"]
        ok = judged if c["mode"] == "judge" else ok | judged
    n = ok.long().cumprod(1).sum(1)
    b = torch.arange(c["B"], device=DEV)
    p = s["p"][b, n].double()
    q = s["pd"][b, n.clamp(max=M - 1)].double() * (n < M)[:, None]
    i = torch.arange(M, device=DEV)
    path = torch.where(i < n[:, None], i + 1, -1).to(torch.int32)
    return dict(accept_len=n.to(torch.int32), next_token=_drawn((p - q).clamp(min=0), p, s["us"]), path=path)


def _plain_tree(s):
    """Nodes in order. Of every sequence: the node it stands at, w = what is left of the target's weights there after the rejected children, W their
    sum, q and Q the draft's weights that are left and their sum."""
    c = s["c"]
    B, M, V = c["B"], c["T"] - 1, c["V"]
    b = torch.arange(B, device=DEV)
    parents = s["parents"].long().expand(B, M + 1)
    cur, n = torch.zeros(B, dtype=torch.long, device=DEV), torch.zeros(B, dtype=torch.long, device=DEV)
    w, q = s["p"][:, 0].double(), s["pd"][:, 0].double()
    W = torch.ones(B, dtype=torch.float64, device=DEV)
    Q = torch.ones_like(W)
    path = torch.full((B, M + 1), -1, dtype=torch.int32, device=DEV)
    for node in range(1, M + 1):
        at, x = parents[:, node] == cur, s["tokens"][:, node - 1].long()
        ok = s["u"][:, node - 1].double() * W * q[b, x] < w[b, x] * Q
        if c["mode"] != "standard":
            judged = s["judge"][:, node - 1] > s["tau"]
            ok = judged if c["mode"] == "judge" else ok | judged
        ok &= at
        no = at & ~ok
        path[b, torch.where(ok, n, M)] = node
        n, cur = n + ok, torch.where(ok, node, cur)
        left = (w * Q[:, None] - W[:, None] * q).clamp(min=0)
        gone = q[b, x] if c["siblings"] == "distinct" else torch.zeros_like(W)
        q = q.clone()
        q[b, x] -= gone * no
        Q = torch.where(ok, 1.0, Q - gone * no)
        w = torch.where(ok[:, None], s["p"][:, node].double(), torch.where(no[:, None], left, w))
        W = torch.where(ok, 1.0, torch.where(no, w.sum(1), W))
        q = torch.where(ok[:, None], s["pd"][:, min(node, M - 1)].double(), q)
    path[:, M] = -1
    return dict(accept_len=n.to(torch.int32), next_token=_drawn(w, s["p"][b, cur].double(), s["us"]), path=path[:, :M].contiguous())


def run(state):
    s, c = state, state["c"]
    op = c["op"]
    if op == "heads":
        if own:
            q, k = s["rotary"].rotate_qk(s["q"], s["nk"], s["pos"], norm=s["norm"])
        else:
            cos, sin = _turns(s)
            q, k = (_plain_heads(x, w, cos, sin, c["layout"]) for x, w in ((s["q"], s["wq"]), (s["nk"], s["wk"])))
        return dict(q=q, k=k)
    if op == "heads_grad":
        if own:
            return s["rotary"].rotate_qk_grad(s["gq"], s["gk"], s["q"], s["nk"], s["pos"], norm=s["norm"])
        cos, sin = _turns(s)
        dq, wq = _plain_heads_grad(s["gq"], s["q"], s["wq"], cos, sin, c["layout"])
        dk, wk = _plain_heads_grad(s["gk"], s["nk"], s["wk"], cos, sin, c["layout"])
        return dict(q=dq, k=dk, q_weight=wq, k_weight=wk)
    if op == "append":
        if own:
            q = s["cache"].append(1, s["nk"], s["nv"], s["tree"], rotary=s["rotary"], q=s["q"], norm=s["norm"], positions=s["pos"] if c["sections"] else None)
        else:
            cos, sin = _turns(s)
            at = s["len"].long()[:, None] + torch.arange(c["T"], device=DEV)
            page, row = torch.gather(s["table"].long(), 1, at // c["page"]), at % c["page"]
            s["k"][1][page, :, row] = _plain_heads(s["nk"], s["wk"], cos, sin, c["layout"])
            s["v"][1][page, :, row] = s["nv"]
            q = _plain_heads(s["q"], s["wq"], cos, sin, c["layout"])
        return dict(q=q, k=s["k"][1], v=s["v"][1])
    if op == "shared":
        if own:
            plan = s["cache"].share(c["T"], plan=s["plan"])
            return [s["cache"].attend(layer, s["q"][layer], shared=plan) for layer in range(c["L"])]
        return [_plain_shared(s, layer) for layer in range(c["L"])]
    if own:
        from paper_2501_19309_b200 import jd
        return jd.verify_probs(s["p"], s["pd"], s["tokens"], s["u"], s["us"], parents=s["parents"], siblings=c["siblings"], mode=c["mode"],
                               judge_scores=None if c["mode"] == "standard" else s["judge"], tau=s["tau"])
    return _plain_chain(s) if c["tree"] == "chain" else _plain_tree(s)


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The same outputs from the definitions; nothing for outputs that are only moved."""
    c = case
    s = prepare(c, seed)
    if c["op"] == "heads":
        return dict(q=_exact_heads(s["q"].double(), s["wq"].double(), s, c), k=_exact_heads(s["nk"].double(), s["wk"].double(), s, c))
    if c["op"] == "heads_grad":
        got = {}
        for name, x, w, g in (("q", s["q"], s["wq"], s["gq"]), ("k", s["nk"], s["wk"], s["gk"])):
            x, w = x.double().requires_grad_(), w.double().requires_grad_()
            got[name], got[name + "_weight"] = torch.autograd.grad(_exact_heads(x, w, s, c), (x, w), g.double())
        return got
    if c["op"] == "append":
        kc = s["k"][1].double()
        rk = _exact_heads(s["nk"].double(), s["wk"].double(), s, c)
        for b, n in enumerate(s["len"].tolist()):
            for t in range(c["T"]):
                kc[int(s["table"][b, (n + t) // c["page"]]), :, (n + t) % c["page"]] = rk[b, t]
        return dict(q=_exact_heads(s["q"].double(), s["wq"].double(), s, c), k=kc, v=None)
    if c["op"] == "shared":
        return [_exact_attend(s, c, layer) for layer in range(c["L"])]
    return _exact_verify(s, c)


def _exact_heads(x, w, s, c):
    """Norm and rotation in 64 bits, pairs as complex numbers."""
    y = x / torch.sqrt(torch.mean(x * x, -1, keepdim=True) + EPS) * w
    pos = s["pos"].double() if s["pos"].dim() == x.dim() - 1 else s["pos"].double().unsqueeze(-1)
    n = c["rot"] // 2
    turn = torch.exp(1j * torch.stack([pos[..., a] * float(f) for a, f in zip(_axis_of(c), s["freq"].tolist())], -1)).unsqueeze(-2)
    if c["layout"] == "half":
        z = torch.complex(y[..., :n], y[..., n:2 * n]) * turn
        return torch.cat((z.real, z.imag, y[..., 2 * n:]), -1)
    z = torch.view_as_complex(y[..., :2 * n].unflatten(-1, (n, 2)).contiguous()) * turn
    return torch.cat((torch.view_as_real(z).flatten(-2), y[..., 2 * n:]), -1)


def _exact_attend(s, c, layer):
    B, T, H, G, D = c["B"], c["T"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["D"]
    out = torch.zeros(B, T, H * G, D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(B, T, H * G, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["len"].tolist()):
        pages = s["table"][b, :_pages(n + T, c["page"])].long()
        bias = torch.zeros(T, n + T, dtype=torch.float64, device=DEV)
        bias[:, n:] = torch.full((T, T), -math.inf, dtype=torch.float64, device=DEV).triu(1)
        for h in range(H):
            keys, vals = (x[layer, pages, h].reshape(-1, D)[:n + T].double() for x in (s["k"], s["v"]))
            z = torch.einsum("tgd,nd->gtn", s["q"][layer, b, :, h * G:(h + 1) * G].double(), keys) / math.sqrt(D) + bias
            lse[b, :, h * G:(h + 1) * G] = torch.logsumexp(z, 2).T
            out[b, :, h * G:(h + 1) * G] = torch.einsum("gtn,nd->tgd", torch.softmax(z, 2), vals)
    return dict(out=out, lse=lse)


def _exact_verify(s, c):
    """One sequence at a time, as a walk from node 0: normalised weights, children in order, until none is accepted."""
    B, M = c["B"], c["T"] - 1
    lens, nexts, paths = [], [], []
    for b in range(B):
        parents = list(range(-1, M)) if s["parents"] is None else (s["parents"] if s["parents"].dim() == 1 else s["parents"][b]).tolist()
        tokens, u, judge = s["tokens"][b].tolist(), s["u"][b].tolist(), s["judge"][b].tolist()
        cur, path = 0, []
        while True:
            w, went = s["p"][b, cur].double(), None
            children = [i for i in range(1, M + 1) if parents[i] == cur]
            q = s["pd"][b, cur].double().clone() if children else None
            for i in children:
                x = tokens[i - 1]
                std = u[i - 1] * float(q[x]) < float(w[x])
                jdg = judge[i - 1] > torch.tensor(s["tau"], dtype=torch.float32).item()
                if {"standard": std, "judge": jdg, "judge_or_standard": std or jdg}[c["mode"]]:
                    went = i
                    break
                keep = 1.0
                if c["siblings"] == "distinct":
                    keep = 1.0 - float(q[x])
                left = (w - q).clamp(min=0)
                w = left / left.sum() if float(left.sum()) > 0 else left
                if c["siblings"] == "distinct":
                    q[x] = 0
                    q /= keep
            if went is None:
                break
            path.append(went)
            cur = went
        if float(w.sum()) == 0:
            w = s["p"][b, cur].double()
        run_ = w.cumsum(0)
        lens.append(len(path))
        nexts.append(int((run_ <= float(s["us"][b]) * run_[-1]).sum().clamp(max=c["V"] - 1)))
        paths.append(path + [-1] * (M - len(path)))
    made = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    return dict(accept_len=made(lens), next_token=made(nexts), path=made(paths).view(B, M))


# ------------------------------------------------------------------------------------------------ floors
def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "verify":     # the rows that the walk ends at, read once, and the drafted tokens' entries
        return dict(bytes=2 * c["B"] * c["V"] * e + 32 * c["B"] * c["T"], flops=6 * c["B"] * c["V"])
    T, H, Hq, D = c.get("T", 1), c["kv_heads"], c["q_heads"], c["D"]
    if c["op"] == "shared":
        rows = c["convs"] * c["prefix"] + sum(_lengths(c, c["own_lo"], c["own_hi"])) + c["B"] * T
        seen = sum(c["prefix"] + n + T for n in _lengths(c, c["own_lo"], c["own_hi"]))
        heads = c["B"] * T * Hq
        return dict(bytes=c["L"] * (2 * rows * H * D * e + 2 * heads * D * e + 4 * heads), flops=c["L"] * 4 * T * Hq * D * seen)
    n = c["N"] if "N" in c else c["B"] * T
    heads = n * (Hq + H)
    if c["op"] == "heads":
        return dict(bytes=2 * heads * D * e + 4 * n, flops=(4 * D + 3 * c["rot"]) * heads)
    if c["op"] == "heads_grad":
        return dict(bytes=3 * heads * D * e + 4 * n, flops=(12 * D + 3 * c["rot"]) * heads)
    return dict(bytes=2 * n * (Hq + 2 * H) * D * e, flops=(4 * D + 3 * c["rot"]) * heads)
