"""Verification of drafted chains and trees from probabilities against the CPU model in float64: decisions, paths and tokens are equal, not near."""
import numpy as np
import pytest
import torch

import cache_testlib as L
from oracle import step_oracle as S
from paper_2501_19309_b200 import jd

pytestmark = pytest.mark.gpu
MODES = ["standard", "judge", "judge_or_standard"]


def inputs(B, T, V, dtype, seed, style="tree", shared=False, sharp=2.0):
    """Peaked distributions, the draft's near the target's; tokens drawn from the draft's at their parents."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    z = torch.randn(B, T, V, generator=gen, device="cuda") * sharp
    d = z[:, :-1] + 0.7 * torch.randn(B, T - 1, V, generator=gen, device="cuda")
    s = dict(target=torch.softmax(z, 2).to(L.DT[dtype]), draft=torch.softmax(d, 2).to(L.DT[dtype]))
    one = L.random_tree(T, rng, style)
    parents = np.array([one] * B if shared else [L.random_tree(T, rng, style) for _ in range(B)])
    at = torch.as_tensor(parents[:, 1:], device="cuda")
    if T > 1:
        w = s["draft"].float().gather(1, at[..., None].expand(B, T - 1, V))
        s["tokens"] = (w.log() - torch.empty_like(w).exponential_(generator=gen).log()).argmax(2).to(torch.int32)
    else:
        s["tokens"] = torch.zeros(B, 0, dtype=torch.int32, device="cuda")
    s["accept_u"], s["sample_u"] = torch.rand(B, T - 1, generator=gen, device="cuda"), torch.rand(B, generator=gen, device="cuda")
    s["judge_scores"] = torch.rand(B, T - 1, generator=gen, device="cuda")
    return s, parents


def check(s, parents, got, num_nodes=None, mode="standard", resample="residual", siblings="independent", tau=0.5, **kw):
    p, q = L.f64(s["target"]), L.f64(s["draft"])
    tok, u, us = s["tokens"].cpu().numpy(), L.f64(s["accept_u"]), L.f64(s["sample_u"])
    judged = s["judge_scores"].cpu().numpy() > np.float32(tau)
    status = 0
    for b in range(p.shape[0]):
        n = p.shape[1] if num_nodes is None else int(num_nodes[b])
        if n == 0:
            continue
        path, token, st = S.verify(p[b, :n], q[b, :n - 1], tok[b], u[b], us[b], parents[b], judged[b], mode, resample, siblings == "distinct")
        status = status or st
        assert int(got["accept_len"][b]) == len(path), b
        assert got["path"][b].tolist() == path + [-1] * (p.shape[1] - 1 - len(path)), b
        assert int(got["next_token"][b]) == token, b
    return status


def call(s, parents, chain=False, shared=False, **kw):
    where = None if chain else L.ints(parents[0] if shared else parents)
    return jd.verify_probs(s["target"], s["draft"], s["tokens"], s["accept_u"], s["sample_u"], parents=where, judge_scores=s["judge_scores"], **kw)


SHAPES = [(1, 2, 1, "f32"), (3, 5, 2, "bf16"), (1, 9, 7, "f32"), (70, 6, 1000, "bf16"), (5, 17, 4099, "f32"), (2, 33, 32000, "bf16"), (150, 4, 515, "f32"),
          (300, 3, 64, "bf16"), (2, 128, 300, "f32"), (3, 1, 999, "f32"), (1, 4, 128257, "bf16"), (20, 8, 16384, "f32"), (40, 5, 2049, "f32")]


@pytest.mark.parametrize("siblings", ["independent", "distinct"])
@pytest.mark.parametrize("B,T,V,dtype", SHAPES)
def test_against_the_model(B, T, V, dtype, siblings):
    for seed, style in enumerate(("tree", "star", "chain")):
        s, parents = inputs(B, T, V, dtype, seed, style)
        for mode in MODES if V < 5000 else MODES[:1]:
            kw = dict(mode=mode, siblings=siblings, tau=0.7, resample="target_p" if seed == 1 and mode == "standard" else "residual")
            check(s, parents, call(s, parents, chain=style == "chain", **kw), **kw)


def test_one_tree_for_all_padded_batches_and_strided_rows():
    B, T, V = 9, 8, 1003
    s, parents = inputs(B, T, V, "f32", 4, shared=True)
    num = L.ints([8, 0, 3, 8, 1, 5, 0, 8, 2])
    for pad in (0, 5, 13):             # rows of a padded vocabulary: on 16 bytes and off them
        t = dict(s)
        for name in ("target", "draft"):
            x = torch.full((B, s[name].shape[1], V + pad), float("nan"), device="cuda")
            x[..., :V] = s[name]
            t[name] = x[..., :V]
        out = dict(accept_len=torch.full((B,), -7, dtype=torch.int32, device="cuda"), next_token=torch.full((B,), -7, dtype=torch.int32, device="cuda"),
                   path=torch.full((B, T - 1), -7, dtype=torch.int32, device="cuda"))
        got = call(t, parents, shared=True, num_nodes=num, out=out)
        assert got is out
        check(s, parents, got, num_nodes=num)
        for b in (1, 6):
            assert got["accept_len"][b] == got["next_token"][b] == -7 and (got["path"][b] == -7).all()
    lean = call(s, parents, shared=True, out=dict(accept_len=out["accept_len"], next_token=out["next_token"]))
    assert "path" not in lean


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_numbers_at_the_borders(dtype):
    """Sums that are exact in both: uniform weights over powers of two, and draws that fall on their edges; the smallest and largest numbers."""
    V = 1024
    p = torch.full((1, 2, V), 1 / V, device="cuda").to(L.DT[dtype])
    q = torch.zeros(1, 1, V, device="cuda").to(L.DT[dtype])
    q[0, 0, :512] = 1 / 512
    for u, us in [(0.0, 0.0), (0.5, 0.0), (0.5, 0.5), (0.499999, 0.25), (0.75, 1 / V), (0.75, 1 - 2.0 ** -24), (1 - 2.0 ** -24, 511 / 512), (0.5, 0.125)]:
        for x in (0, 511, 512, 1023):
            s = dict(target=p, draft=q, tokens=L.ints([[x]]), accept_u=torch.tensor([[u]], device="cuda"), sample_u=torch.tensor([us], device="cuda"),
                     judge_scores=torch.zeros(1, 1, device="cuda"))
            check(s, [[-1, 0]], call(s, [[-1, 0]], chain=True))


def test_weights_that_leave_nothing():
    """p = q rejected by a judge: nothing is left, the target's own row counts. Weight on one token, on the last, on none."""
    V = 300
    s, parents = inputs(4, 4, V, "f32", 0, "star")
    s["draft"][:] = s["target"][:, :1]
    kw = dict(mode="judge", tau=1.0)
    check(s, parents, call(s, parents, **kw), **kw)
    s["target"].zero_()
    s["target"][0, :, V - 1] = 1
    s["target"][1, :, 0] = 1
    s["target"][2, :, 177] = 1e-30
    for siblings in ("independent", "distinct"):
        got = call(s, parents, siblings=siblings)
        check(s, parents, got, siblings=siblings)
        assert int(got["next_token"][3]) == V - 1                      # a row without mass


def test_numbers_outside_the_interval_end_in_range():
    s, parents = inputs(6, 4, 700, "f32", 0)
    s["sample_u"] = torch.tensor([1.0, 2.0, float("nan"), float("inf"), -1.0, float("-inf")], device="cuda")
    s["accept_u"][:, 0] = float("nan")
    got = call(s, parents)
    t = got["next_token"]
    assert ((t >= 0) & (t < 700)).all() and (s["target"][torch.arange(6), 0, t.long()] > 0).any()


def test_bad_tokens_and_parents_are_reported():
    s, parents = inputs(3, 5, 200, "f32", 1)
    for bad, code in (([0, 200], jd.JD_ERR_BAD_TOKEN), ([1, -1], jd.JD_ERR_BAD_TOKEN), ([2, 2 ** 31 - 1], jd.JD_ERR_BAD_TOKEN)):
        t = dict(s, tokens=s["tokens"].clone())
        t["tokens"][bad[0], 1] = bad[1]
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = call(t, parents, status=status)
        assert check(t, parents, got) == code == int(status)
    for bad in (3, 4, -1, 2 ** 31 - 1, -2 ** 31):                      # of node 3
        p = parents.copy()
        p[1, 3] = bad
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = call(s, p, status=status)
        assert check(s, p, got) == jd.JD_ERR_BAD_INDEX == int(status)
    status.fill_(jd.JD_ERR_TIMEOUT)
    call(s, p, status=status)
    assert int(status) == jd.JD_ERR_TIMEOUT                            # the first problem stays


@pytest.mark.parametrize("siblings", ["independent", "distinct"])
@pytest.mark.parametrize("style,T", [("chain", 2), ("star", 3), ("star", 4)])
def test_emitted_tokens_have_the_targets_law(style, T, siblings):
    """60,000 sequences of the same distributions: the first emitted token against p. chi^2 of 5 degrees of freedom is above 45 once in 10^8 runs."""
    B, V = 60000, 6
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    p = torch.tensor([0.3, 0.05, 0.25, 0.1, 0.1, 0.2], device="cuda")
    q = torch.tensor([0.1, 0.3, 0.1, 0.3, 0.1, 0.1], device="cuda")
    keys = q.log() - torch.empty(B, T - 1, V, device="cuda").exponential_(generator=gen).log()
    tokens = keys[:, 0].topk(T - 1, 1).indices if siblings == "distinct" and style == "star" else keys.argmax(2)
    u, us = torch.rand(B, T - 1, generator=gen, device="cuda"), torch.rand(B, generator=gen, device="cuda")
    tokens = tokens.to(torch.int32)
    got = jd.verify_probs(p.expand(B, T, V).contiguous(), q.expand(B, T - 1, V).contiguous(), tokens, u, us, parents=L.ints([-1] + [0] * (T - 1)), siblings=siblings)
    first = got["path"][:, 0].long()
    emitted = torch.where(first > 0, tokens.gather(1, (first - 1).clamp(min=0)[:, None])[:, 0], got["next_token"])
    count = torch.bincount(emitted.long(), minlength=V).double()
    want = p.double() / p.double().sum() * B
    assert float(((count - want) ** 2 / want).sum()) < 45


def test_a_sequence_gives_the_same_whatever_stands_beside_it():
    """One sequence takes the largest cluster, hundreds a block each: sums in another order, the same tokens."""
    s, parents = inputs(2, 9, 50000, "f32", 8)
    alone = [call({k: v[b:b + 1].contiguous() for k, v in s.items()}, parents[b:b + 1]) for b in range(2)]
    for copies in (12, 30, 60, 160):
        got = call({k: v.repeat(copies, *[1] * (v.dim() - 1)) for k, v in s.items()}, np.tile(parents, (copies, 1)))
        for k in got:
            for b in range(2):
                assert (got[k][b::2] == alone[b][k]).all()


def test_streams_graphs_and_repeats():
    s, parents = inputs(11, 9, 3001, "f32", 3)
    want = call(s, parents)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(20):
        for x in streams:
            with torch.cuda.stream(x):
                got.append(call(s, parents))
    torch.cuda.synchronize()
    assert all(torch.equal(g[k], want[k]) for g in got for k in want)
    where, graph = L.ints(parents), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = jd.verify_probs(s["target"], s["draft"], s["tokens"], s["accept_u"], s["sample_u"], parents=where)
    t, other = inputs(11, 9, 3001, "f32", 4)
    for k in s:
        s[k].copy_(t[k])
    where.copy_(L.ints(other))
    graph.replay()
    torch.cuda.synchronize()
    check(t, other, out)


def test_refusals():
    s, parents = inputs(3, 5, 64, "f32", 1)
    good = dict(target=s["target"], draft=s["draft"], tokens=s["tokens"], accept_u=s["accept_u"], sample_u=s["sample_u"])
    for kw in (dict(target=s["target"].half()), dict(target=s["target"][0]), dict(draft=s["draft"][:, :3]), dict(draft=s["draft"].bfloat16()), dict(draft=None),
               dict(tokens=s["tokens"].long()), dict(tokens=s["tokens"].cpu()), dict(accept_u=s["accept_u"].double()), dict(sample_u=s["sample_u"][:2]),
               dict(parents=L.ints([0, 1])), dict(parents=L.ints(parents).long()), dict(num_nodes=L.ints([1, 2])), dict(mode="judge"), dict(status=L.ints([0, 0])),
               dict(target=s["target"].transpose(0, 1).contiguous().transpose(0, 1)), dict(target=s["target"][:1].expand(3, 5, 64)), dict(target=s["target"].clone().requires_grad_()),
               dict(out=dict(accept_len=L.ints([0, 0, 0]), next_token=L.ints([0])))):
        with pytest.raises(ValueError):
            jd.verify_probs(**dict(good, **kw))
    with pytest.raises(jd.JdError):
        jd.verify_probs(**good, mode="judge", judge_scores=s["judge_scores"], tau=2.0)
    with pytest.raises(KeyError):
        jd.verify_probs(**good, siblings="some")
    big, q, tok, u = torch.ones(1, 130, 4, device="cuda"), torch.ones(1, 129, 4, device="cuda"), torch.zeros(1, 129, dtype=torch.int32, device="cuda"), torch.zeros(1, 129, device="cuda")
    with pytest.raises(jd.JdError):
        jd.verify_probs(big, q, tok, u, torch.zeros(1, device="cuda"))


# ------------------------------------------------------------------------------------------- confident drafts
def confident(which, dtype):
    """(target, draft) rows of four tokens."""
    logits = torch.tensor([20., 0, 0.5, -1] if which == 1 else [20., 19, 0.5, -1])
    draft = torch.softmax(logits, 0) if which in (1, 2) else torch.tensor({.9: [.9, .04, .03, .03], .99: [.99, .004, .003, .003], .999: [.999, .0004, .0003, .0003]}[which])
    return torch.tensor([.5, .2, .2, .1]).to(L.DT[dtype]), draft.to(L.DT[dtype])


def siblings_of(p, q, B, n, seed):
    """B stars of n siblings drawn from q without replacement."""
    gen = torch.Generator().manual_seed(seed)
    keys = q.double().log() - torch.empty(B, len(q), dtype=torch.float64).exponential_(generator=gen).log()
    s = dict(target=p.expand(B, n + 1, len(p)), draft=q.expand(B, n, len(q)), tokens=keys.topk(n, 1).indices.to(torch.int32), accept_u=torch.rand(B, n, generator=gen),
             sample_u=torch.rand(B, generator=gen), judge_scores=torch.rand(B, n, generator=gen))
    return {k: v.contiguous().cuda() for k, v in s.items()}, np.array([[-1] + [0] * n] * B)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [2, 3, 4])
@pytest.mark.parametrize("which", [1, 2, .9, .99, .999])
def test_distinct_siblings_of_a_confident_draft(which, n, dtype):
    p, q = confident(which, dtype)
    s, parents = siblings_of(p, q, 1500, n, seed=n)
    for mode in MODES:
        check(s, parents, call(s, parents, siblings="distinct", mode=mode, tau=0.7), siblings="distinct", mode=mode, tau=0.7)


@pytest.mark.parametrize("n", [2, 3, 4])
@pytest.mark.parametrize("which", [1, 2, .9, .99, .999])
def test_the_targets_law_behind_a_confident_draft(which, n):
    """60,000 sequences, float32 rows whose sums are 1 within 2^-23: chi^2 of 3 degrees of freedom is above 41 once in 10^8 runs."""
    p, q = confident(which, "f32")
    s, parents = siblings_of(p, q, 60000, n, seed=10 + n)
    got = jd.verify_probs(s["target"], s["draft"], s["tokens"], s["accept_u"], s["sample_u"], parents=L.ints(parents[0]), siblings="distinct")
    first = got["path"][:, 0].long()
    emitted = torch.where(first > 0, s["tokens"].gather(1, (first - 1).clamp(min=0)[:, None])[:, 0], got["next_token"])
    count, want = torch.bincount(emitted.long(), minlength=4).double().cpu(), p.double() / p.double().sum() * 60000
    assert float(((count - want) ** 2 / want).sum()) < 41


@pytest.mark.parametrize("V,dtype", [(5000, "f32"), (33001, "f32"), (5000, "bf16")])
def test_confident_rows_of_a_vocabulary(V, dtype):
    """Rows that put 0.9 to 1 on a token: chains, and trees whose nodes have several children."""
    for seed, style in enumerate(("tree", "star", "chain")):
        s, parents = inputs(40, 9, V, dtype, seed, style, sharp=8.0)
        for siblings in ("independent", "distinct"):
            check(s, parents, call(s, parents, chain=style == "chain", siblings=siblings), siblings=siblings)


@pytest.mark.parametrize("siblings", ["independent", "distinct"])
def test_many_rejections_leave_the_rest_of_the_target(siblings):
    """127 siblings of confident rows, all rejected: the products of what is left on the way are far below float64's smallest number."""
    rng = np.random.default_rng(5)
    V, n, B = 2000, 127, 24
    p, q = (torch.softmax(torch.as_tensor(12 * rng.normal(size=V)), 0).numpy() for _ in range(2))
    tokens = np.argsort(-(np.log(q) + rng.gumbel(size=V)))[:n]
    left = q.copy()
    for x in tokens:
        p[x] = left[x] / left.sum() / 250
        left[x] = 0
    other = np.setdiff1d(np.arange(V), tokens)
    p[other] *= (1 - p[tokens].sum()) / p[other].sum()
    put = lambda x, *shape: torch.as_tensor(x, dtype=torch.float32, device="cuda").expand(*shape).contiguous()   # noqa: E731
    s = dict(target=put(p, B, n + 1, V), draft=put(q, B, n, V), tokens=L.ints(np.tile(tokens, (B, 1))), accept_u=put(0.999, B, n), sample_u=put(np.linspace(0.001, 0.999, B), B),
             judge_scores=put(0.0, B, n))
    parents = np.array([[-1] + [0] * n] * B)
    got = call(s, parents, siblings=siblings)
    check(s, parents, got, siblings=siblings)
    if siblings == "distinct":
        assert not np.isin(got["next_token"].cpu().numpy(), tokens).any()      # the target's own row would give some of them


@pytest.mark.parametrize("siblings", ["independent", "distinct"])
@pytest.mark.parametrize("V,dtype", [(3, "f32"), (1000, "f32"), (70001, "f32"), (5000, "bf16")])
def test_weights_whose_sum_float32_does_not_hold(V, dtype, siblings):
    """Finite, not negative, their sums whatever they are."""
    for seed, style in enumerate(("chain", "star", "tree")):
        s, parents = inputs(6, 6, V, "f32", seed, style)
        s["target"], s["draft"] = ((torch.rand(x.shape, generator=torch.Generator().manual_seed(seed + i)) * 3.3e38).to(L.DT[dtype]).cuda() for i, x in enumerate((s["target"], s["draft"])))
        s["accept_u"] = s["accept_u"] * 0.3 + 0.7
        check(s, parents, call(s, parents, chain=style == "chain", siblings=siblings), siblings=siblings)


def test_outputs_of_sequences_without_nodes():
    """Outputs that the call makes itself hold -1 there, whatever the memory held before, on whatever stream."""
    s, parents = inputs(9, 8, 100, "f32", 4, shared=True)
    num, want = L.ints([8, 0, 3, 8, 1, 5, 0, 8, 2]), None
    for stream in (None, torch.cuda.Stream()):
        for _ in range(3):
            junk = torch.full((9 * 9,), 12345, dtype=torch.int32, device="cuda")
            torch.cuda.synchronize()
            del junk
            got = call(s, parents, shared=True, num_nodes=num, stream=stream)
            torch.cuda.synchronize()
            check(s, parents, got, num_nodes=num)
            for b in (1, 6):
                assert got["accept_len"][b] == got["next_token"][b] == -1 and (got["path"][b] == -1).all()
