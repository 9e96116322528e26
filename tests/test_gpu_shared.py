"""Attention of sequences that share a prefix against the CPU model, which knows nothing of plans."""
import numpy as np
import pytest
import torch

import cache_testlib as L
from oracle import cache_oracle as O
from paper_2501_19309_b200 import jd

pytestmark = pytest.mark.gpu


def rand(shape, seed, dtype="bf16"):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda").to(L.DT[dtype])


def forked(prefixes, members, own, T, *, page=16, q_heads=4, kv_heads=2, D=64, dtype="bf16", seed=0, order=None, layers=1):
    """A cache in which members[i] sequences follow conversation i for prefixes[i] tokens and have own[..] tokens more, pages for T nodes held.
    Slots 0.. are the conversations, then the members. Returns the cache and the members' slots (shuffled unless order is given)."""
    n = sum(members)
    room = n * (max(own) + T + 2 * page) + sum(prefixes) + len(prefixes) * page + 4000
    c = L.empty_cache(layers, room // page + 2 * n + 8, page, q_heads, kv_heads, D, len(prefixes) + n, (max(prefixes) + max(own) + T + 800) // page + 3, max(T, 8), dtype, fill=seed)
    slots = torch.arange(len(prefixes), len(prefixes) + n, dtype=torch.int32, device="cuda")
    for i, p in enumerate(prefixes):
        if p:
            c.reserve(p, slots=L.ints([i]))
    c.seq_len[:len(prefixes)] = L.ints(prefixes)
    c.fork(L.ints(np.repeat(np.arange(len(prefixes)), members)), slots)
    c.reserve(max(own) + T, slots=slots)
    c.seq_len[len(prefixes):] += L.ints(own)
    c.k.copy_(rand(c.k.shape, seed + 1, dtype)), c.v.copy_(rand(c.v.shape, seed + 2, dtype))     # the copies of parted pages too: only pages count
    assert c.status() == jd.JD_OK
    perm = np.random.default_rng(seed).permutation(n) if order is None else order
    return c, slots[torch.as_tensor(np.asarray(perm), device="cuda")].contiguous()


def forms(c):
    """By cost, and every form in which the cache's calls can share."""
    return (0, 32, 64, 128, 256) if c.dtype == torch.bfloat16 and c.head_dim in (64, 128) else (0, 4, 16)


def arrays(plan):
    """The plan's arrays behind its counter, each from a multiple of 256 bytes: first members, tokens of the groups, members, groups of the entries."""
    torch.cuda.synchronize()
    ints, step = plan.buffer[256:].view(torch.int32), ((plan.B + 1) * 4 + 255) // 256 * 64
    return [ints[k * step:k * step + n].tolist() for k, n in ((2, plan.B // 2), (3, plan.B // 2), (5, plan.B), (6, plan.B))]


def shares(plan):
    return any(n > 0 for n in arrays(plan)[1])


def tree_of(T, seed, style="tree"):
    parents = L.random_tree(T, np.random.default_rng(seed), style)
    return L.device_tree(parents), O.visible(parents)[0]


def check(c, q, see, got, slots, num_nodes=None, layer=0):
    """out and lse of a call against the model; rows that no node has are not looked at."""
    m, scale = L.model_of(c), c.head_dim ** -0.5
    s = L.f64(slots).astype(int)
    n = None if num_nodes is None else L.f64(num_nodes).astype(int)
    want, lse = m.attend(layer, L.f64(q), see, scale, s, n)
    live = ~np.isnan(lse)
    tol, tol_lse = L.attend_tolerance(m, layer, L.f64(q), see, scale, np.nan_to_num(want), "bf16" if c.dtype == torch.bfloat16 else "f32", s, n)
    assert (np.abs(L.f64(got["out"]) - want)[live] <= np.nan_to_num(tol)[live]).all()
    fin = live & np.isfinite(lse)
    assert (np.abs(L.f64(got["lse"]) - lse)[fin] <= np.nan_to_num(tol_lse)[fin] + 2.0 ** -22 * np.abs(lse[fin])).all()


CASES = [  # prefixes, members, own tokens, T, page, q heads, kv heads, head_dim, dtype
    ([700], [5], [0, 40, 3, 200, 129], 1, 16, 8, 2, 128, "bf16"),              # one token each: rows lie four times over
    ([1500], [9], [10] * 9, 5, 64, 8, 2, 128, "bf16"),                          # 180 rows: pairs
    ([640, 300], [4, 3], [0, 300, 5, 17, 128, 0, 64], 9, 8, 4, 2, 64, "bf16"),  # two conversations
    ([2000], [3], [7, 0, 1], 26, 32, 16, 1, 64, "bf16"),                        # more rows of a sequence than a block takes
    ([1300], [12], [3] * 12, 2, 128, 6, 2, 128, "bf16"),
    ([500], [4], [30, 0, 700, 2], 5, 16, 6, 2, 80, "bf16"),                     # CUDA cores
    ([900], [5], [0, 40, 3, 200, 129], 1, 8, 4, 4, 64, "f32"),
    ([1100, 1100, 260], [2, 3, 2], [9] * 7, 4, 16, 9, 3, 40, "f32"),
    ([600], [3], [5, 5, 5], 7, 32, 4, 1, 200, "f32"),
    ([100], [6], [40] * 6, 3, 16, 4, 2, 64, "bf16"),                            # too short to share
    ([3000], [2], [0, 0], 1, 16, 1, 1, 128, "bf16"),
]


@pytest.mark.parametrize("prefixes,members,own,T,page,q_heads,kv_heads,D,dtype", CASES)
def test_shared_attention(prefixes, members, own, T, page, q_heads, kv_heads, D, dtype):
    c, slots = forked(prefixes, members, own, T, page=page, q_heads=q_heads, kv_heads=kv_heads, D=D, dtype=dtype)
    tree, see = tree_of(T, 3)
    q = rand((len(own), T, q_heads, D), 9, dtype)
    plan = None
    for rows in forms(c) + (4, 16):
        plan = c.share(T, slots=slots, plan=plan, rows=rows)
        for variant in ("auto", "simt"):
            got = c.attend(0, q, tree, slots=slots, shared=plan, variant=variant)
            check(c, q, see, got, slots)
            again = c.attend(0, q, tree, slots=slots, shared=plan, variant=variant)
            assert torch.equal(got["out"], again["out"]) and torch.equal(got["lse"], again["lse"])     # bit for bit
    assert c.status() == jd.JD_OK


@pytest.mark.parametrize("seed", range(8))
def test_random_batches(seed):
    """Padding entries, padded trees, sequences without nodes, a slot named twice, conversations themselves among their forks."""
    rng = np.random.default_rng(seed)
    kv, group, D = int(rng.choice([1, 2, 3])), int(rng.choice([1, 2, 5])), int(rng.choice([64, 128]))
    T = int(rng.choice([1, 3, 8, 17]))
    prefixes = [int(x) for x in rng.integers(0, 1200, size=3)]
    members = [int(x) for x in rng.integers(1, 5, size=3)]
    own = [int(x) for x in rng.integers(0, 300, size=sum(members))]
    c, slots = forked(prefixes, members, own, T, page=int(rng.choice([8, 32])), q_heads=kv * group, kv_heads=kv, D=D, seed=seed)
    c.reserve(T, slots=L.ints([0]))                                    # conversation 0 goes on by itself
    names = list(L.f64(slots).astype(int)) + [0, -1, int(slots[0])]
    rng.shuffle(names)
    slots = L.ints(names)
    nodes = L.ints(rng.integers(0, T + 1, size=len(names)))
    parents = L.random_tree(T, rng)
    tree, see = L.device_tree(parents, num_nodes=nodes), O.visible(parents)[0]
    q = rand((len(names), T, kv * group, D), seed)
    for rows in forms(c):
        out = dict(out=torch.full_like(q, 7.0), lse=torch.full(q.shape[:3], 7.0, device="cuda"))
        plan = c.share(T, slots=slots, rows=rows)
        c.attend(0, q, tree, slots=slots, shared=plan, out=out)
        check(c, q, see, out, slots, nodes)
        for b, n in enumerate(nodes.tolist()):
            n = 0 if names[b] < 0 else n
            assert (out["out"][b, n:] == 7).all() and (out["lse"][b, n:] == 7).all()      # rows behind the nodes are left as they were


@pytest.mark.parametrize("dtype,D,rows", [("bf16", 128, 32), ("bf16", 128, 256), ("f32", 64, 4), ("f32", 64, 16), ("bf16", 64, 0)])
def test_plans_that_the_tables_have_left_behind(dtype, D, rows):
    """A plan is made, then a member is cut back into the prefix and grows again, the leader is, a slot is emptied and becomes something else, pages move: results stay
    right with the old plan, and with one of other slots."""
    c, slots = forked([800, 700], [4, 3], [20] * 7, 4, q_heads=4, kv_heads=2, D=D, dtype=dtype, order=np.arange(7))
    tree, see = tree_of(4, 1)
    q = rand((7, 4, 4, D), 5, dtype)
    plan = c.share(4, slots=slots, rows=rows)

    def right(now):
        c.reserve(4, slots=slots)
        assert c.status() == jd.JD_OK
        check(c, q, see, c.attend(0, q, tree, slots=now, shared=plan), now)

    def cut(slot, to, again):
        c.truncate(L.ints([to]), slots=L.ints([slot]))
        c.reserve(again, slots=L.ints([slot]))
        c.seq_len[slot] += again

    right(slots)
    cut(int(slots[2]), 300, 600)                                       # a member parts inside the prefix
    right(slots)
    cut(int(slots[4]), 10, 50)                                         # the second group's first entry, now shorter than the prefix
    right(slots)
    c.free(slots[1:2].contiguous())
    c.fork(L.ints([1]), slots[1:2].contiguous())                        # another conversation in its place
    right(slots)
    right(slots.flip(0).contiguous())                                   # other slots than the plan's
    c.compact()
    right(slots)
    plan = c.share(4, slots=slots, plan=plan, rows=rows)                # and made anew
    right(slots)


def test_numbers_of_the_callers():
    """Groups by number: right whatever they say, and the prefix of what belongs together is found where first pages would mix two levels."""
    c, slots = forked([512], [6], [0] * 6, 3, q_heads=4, kv_heads=1, D=64, order=np.arange(6))
    c.reserve(600, slots=slots[:1].contiguous())
    c.seq_len[int(slots[0])] += 600
    c.free(slots[1:3].contiguous())
    c.fork(slots[:1].repeat(2).contiguous(), slots[1:3].contiguous())   # 0, 1, 2 share 1112 tokens, all six 512
    c.reserve(3, slots=slots)
    tree, see = tree_of(3, 1)
    q = rand((6, 3, 4, 64), 2)
    for numbers in (None, [0, 0, 0, 1, 1, 1], [5, 5, -1, 5, -7, 5], [0, 1, 2, 3, 4, 5], [0, 1, 0, 1, 0, 1]):
        plan = c.share(3, slots=slots, groups=None if numbers is None else L.ints(numbers), rows=32)
        check(c, q, see, c.attend(0, q, tree, slots=slots, shared=plan), slots)
    assert c.status() == jd.JD_OK


def test_prefixes_are_found():
    """The plan's own arrays: what is shared, in whole tiles, by whom."""
    c, slots = forked([1000, 640], [3, 2], [30, 0, 500, 9, 9], 1, order=[3, 0, 4, 1, 2])
    plan = c.share(1, slots=slots, rows=64)
    start, tokens, member, entry = arrays(plan)
    # entries 1, 3 and 4 share 1000 tokens, 992 in full pages, seven tiles of 128; 0 and 2 share 640, five
    assert (start, tokens, member, entry) == ([0, 2], [640, 896], [0, 2, 1, 3, 4], [0, 1, 0, 1, 1])
    plan = c.share(1, slots=slots, plan=plan)                           # some microseconds for a dozen tiles: not by cost
    assert arrays(plan)[1] == [0, 0] and arrays(plan)[3] == [-1] * 5 and not shares(plan)


def test_what_pays_is_shared():
    """By cost: 40 sequences behind 4000 tokens are, and as lengths have it; pairs of short ones are not."""
    c, slots = forked([4000], [40], [5] * 40, 1, page=16, q_heads=16, kv_heads=4, D=128)
    plan = c.share(1, slots=slots)
    assert arrays(plan)[1][:2] == [3968, 0] and arrays(plan)[3] == [0] * 40
    c.truncate(L.ints([130] * 40), slots=slots)
    assert not shares(c.share(1, slots=slots, plan=plan))
    c, slots = forked([4000], [40], [5] * 40, 1, page=16, q_heads=16, kv_heads=4, D=128, dtype="f32")
    assert arrays(c.share(1, slots=slots))[1][:2] == [3968, 0]


@pytest.mark.parametrize("dtype,D,rows", [("bf16", 128, 64), ("bf16", 64, 256), ("bf16", 64, 0), ("f32", 64, 4), ("f32", 64, 16)])
def test_a_captured_step_replays(dtype, D, rows):
    """Plan and attention in a graph; lengths and what is shared change between replays."""
    c, slots = forked([900], [5], [20] * 5, 4, q_heads=8, kv_heads=2, D=D, dtype=dtype, layers=2)
    tree, see = tree_of(4, 2)
    q = rand((5, 4, 8, D), 5, dtype)
    plan = c.share(4, rows=rows, slots=slots)
    outs = [c.attend(i, q, tree, slots=slots, shared=plan) for i in range(2)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.reserve(4, slots=slots)
        c.share(4, rows=rows, slots=slots, plan=plan)
        outs = [c.attend(i, q, tree, slots=slots, shared=plan) for i in range(2)]
    for i in range(3):
        if i == 1:
            c.commit(L.ints([3, 0, 1, 2, 3]), path_len=3, slots=slots)
        if i == 2:
            c.truncate(L.ints([100]), slots=slots[2:3].contiguous())
        graph.replay()
        torch.cuda.synchronize()
        for layer in range(2):
            check(c, q, see, outs[layer], slots, layer=layer)
    assert c.status() == jd.JD_OK


def test_two_handles_two_plans_two_streams():
    c, slots = forked([1200], [6], [30] * 6, 3, q_heads=8, kv_heads=2, D=128)
    d = jd.PagedCache(c.k, c.v, c.page_table, c.seq_len, c.held, c.refs, c.free_bits, c.q_heads, c.max_nodes)
    tree, _ = tree_of(3, 2)
    q = rand((6, 3, 8, 128), 5)
    plans = [x.share(3, rows=128, slots=slots) for x in (c, d)]
    want = c.attend(0, q, tree, slots=slots, shared=plans[0])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(20):
        for x, plan, s in zip((c, d), plans, streams):
            with torch.cuda.stream(s):
                x.share(3, rows=128, slots=slots, plan=plan)
                got.append(x.attend(0, q, tree, slots=slots, shared=plan))
    torch.cuda.synchronize()
    assert all(torch.equal(x["out"], want["out"]) and torch.equal(x["lse"], want["lse"]) for x in got)


@pytest.mark.parametrize("T,q_heads", [(1, 4), (6, 4), (17, 8)])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_values_that_are_not_finite(dtype, D, T, q_heads):
    """Of prefix tokens they reach every row, of a hidden node none, as without a plan; rows of pages behind the tokens hold NaN."""
    c, slots = forked([600], [4], [5, 0, 77, 130], T, page=16, q_heads=q_heads, kv_heads=1, D=D, dtype=dtype, order=np.arange(4))
    lens = c.seq_len[slots.long()].tolist()
    table = c.page_table
    for s, n in zip(slots.tolist(), lens):
        for x in (c.k, c.v):
            for t in range(n + T, int(c.held[s]) * 16):
                x[0, int(table[s, t // 16]), 0, t % 16] = float("nan")
    c.v[0, int(table[0, 3]), 0, 5, 7] = float("inf")                    # token 53, of all
    c.v[0, int(table[int(slots[2]), (lens[2] - 1) // 16]), 0, (lens[2] - 1) % 16, 9] = float("nan")
    tree, see = tree_of(T, 4, "star" if T > 1 else "tree")
    if T > 1:
        c.v[0, int(table[int(slots[1]), (lens[1] + 1) // 16]), 0, (lens[1] + 1) % 16, 11] = float("-inf")   # node 1 of sequence 1: its own alone
    q = rand((4, T, q_heads, D), 5, dtype)
    for rows in forms(c):
        values_hold(c, q, tree, slots, T, c.attend(0, q, tree, slots=slots, shared=c.share(T, slots=slots, rows=rows)))


def values_hold(c, q, tree, slots, T, got):
    o = got["out"].float()
    assert (o[..., 7] == float("inf")).all() and torch.isnan(o[2, ..., 9]).all()
    hit = torch.zeros_like(o, dtype=torch.bool)
    hit[..., 7] = hit[2, ..., 9] = True
    if T > 1:
        hit[1, 1, :, 11] = True
        assert (o[1, 1, :, 11] == float("-inf")).all()
    assert torch.isfinite(o[~hit]).all() and torch.isfinite(got["lse"]).all()
    plain = c.attend(0, q, tree, slots=slots)["out"].float()
    assert (o[~hit] - plain[~hit]).abs().max() <= 2.0 ** -6 * plain[~hit].abs().max()


def test_a_long_prefix_and_many_sequences():
    c, slots = forked([20000], [60], [1] * 60, 1, page=128, q_heads=4, kv_heads=1, D=64)
    q = rand((60, 1, 4, 64), 5)
    for rows in forms(c):
        check(c, q, np.ones((1, 1), dtype=bool), c.attend(0, q, slots=slots, shared=c.share(1, slots=slots, rows=rows)), slots)


def test_more_sequences_than_threads():
    """The most that a plan takes, conversations of two in turn."""
    n = 256
    c, slots = forked([1200] * 2, [n, n], [0] * (2 * n), 1, page=64, q_heads=1, kv_heads=1, D=64, order=np.arange(2 * n).reshape(2, n).T.reshape(-1))
    q = rand((2 * n, 1, 1, 64), 5)
    plain = c.attend(0, q, slots=slots)
    for rows in forms(c):
        got = c.attend(0, q, slots=slots, shared=c.share(1, slots=slots, rows=rows))
        # weights rounded to bf16 in either call, and both outputs: 4 steps
        assert (got["out"].float() - plain["out"].float()).abs().max() <= 4 * 2.0 ** -8 * c.v.float().abs().max()
        assert (got["lse"] - plain["lse"]).abs().max() <= 1e-5
    with pytest.raises(ValueError, match="512"):
        L.empty_cache(1, 1, 8, 1, 1, 8, 513, 1, 1).share(1)


def test_a_step_with_everything():
    """Forks of two conversations: plan, norms and rotation into the cache, shared attention, verification of the trees by sampling, commit of the paths; against the
    same step without a plan."""
    T, V, B = 6, 500, 7
    parents = [-1, 0, 0, 1, 1, 2]
    freq, _ = jd.rope_frequencies(64)
    r, norm = jd.Rotary(freq.cuda()), jd.HeadNorm(1 + 0.1 * rand((64,), 1, "f32"), None)
    lens = []
    for shared in (False, True):
        c, slots = forked([500, 400], [4, 3], [0, 5, 9, 13, 2, 2, 70], T, q_heads=4, kv_heads=2, D=64, layers=2)
        tree = L.device_tree(parents)
        outs = []
        for step in range(3):
            c.reserve(T, slots=slots)
            plan = c.share(T, slots=slots, rows=32) if shared else None
            for layer in range(2):
                q, k, v = (rand((B, T, h, 64), 10 * step + 3 * layer + i) for i, h in enumerate((4, 2, 2)))
                q = c.append(layer, k, v, tree, rotary=r, q=q, slots=slots, norm=norm)
                outs.append(c.attend(layer, q, tree, slots=slots, shared=plan)["out"])
            p, d = (torch.softmax(2 * rand((B, n, V), 50 + step + i, "f32"), 2) for i, n in enumerate((T, T - 1)))
            u = torch.rand(B, T, generator=torch.Generator(device="cuda").manual_seed(step), device="cuda")
            tokens = torch.randint(0, V, (B, T - 1), generator=torch.Generator(device="cuda").manual_seed(step), device="cuda").to(torch.int32)
            ver = jd.verify_probs(p, d, tokens, u[:, 1:].contiguous(), u[:, 0].contiguous(), parents=L.ints(parents), siblings="independent")
            c.commit(ver["accept_len"][:, None], ver["path"][:, None].contiguous(), slots=slots)
            lens.append(ver["accept_len"].tolist())
        assert c.status() == jd.JD_OK
        if not shared:
            want, want_len = outs, c.seq_len.tolist()
    assert c.seq_len.tolist() == want_len and lens[:3] == lens[3:] and sum(map(sum, lens)) > 0
    for a, b in zip(outs, want):
        assert (a.float() - b.float()).abs().max() <= 4 * 2.0 ** -8 * c.v.float().abs().max()


def test_refusals():
    c, slots = forked([300], [3], [1, 2, 3], 4, D=64)
    d, _ = forked([300], [3], [1, 2, 3], 4, D=64)
    q = rand((3, 4, 4, 64), 0)
    plan = c.share(2, slots=slots)
    for bad in (lambda: c.attend(0, q, slots=slots, shared=plan), lambda: d.attend(0, q[:, :2], slots=slots, shared=plan), lambda: c.share(9, slots=slots),
                lambda: c.share(0, slots=slots), lambda: c.share(4, slots=slots, plan=plan), lambda: c.share(2, slots=slots[:2].contiguous(), plan=plan),
                lambda: d.share(2, slots=slots, plan=plan), lambda: c.attend(0, q[:2, :2].contiguous(), slots=slots[:2].contiguous(), shared=plan),
                lambda: c.share(2, slots=slots, groups=torch.zeros(3, device="cuda")), lambda: c.share(2, slots=slots, groups=L.ints([0, 1])),
                lambda: c.share(2, slots=slots, rows=8)):
        with pytest.raises(ValueError):
            bad()
    lib, a = c._lib, jd.jd_attend_args_t()
    small = jd.jd_shared_t(3, 2, plan.c.buffer, plan.c.bytes - 1)
    off = jd.jd_shared_t(3, 2, plan.c.buffer + 16, plan.c.bytes)
    for x in (small, off, jd.jd_shared_t(3, 2, 0, plan.c.bytes), jd.jd_shared_t(0, 2, plan.c.buffer, plan.c.bytes), jd.jd_shared_t(513, 2, plan.c.buffer, plan.c.bytes)):
        assert lib.jd_cache_share(c.h, x, slots.data_ptr(), None, None) == jd.JD_ERR_INVALID_ARG
        assert lib.jd_cache_attend_shared(c.h, a, x, None) == jd.JD_ERR_INVALID_ARG
    for rows, want in ((8, jd.JD_ERR_INVALID_ARG), (-4, jd.JD_ERR_INVALID_ARG), (512, jd.JD_ERR_INVALID_ARG)):
        x = jd.jd_shared_t(3, 2, plan.c.buffer, plan.c.bytes, rows)
        assert lib.jd_cache_share(c.h, x, slots.data_ptr(), None, None) == want
    e, _ = forked([300], [3], [1, 2, 3], 4, D=64, dtype="f32")
    with pytest.raises(jd.JdError):
        e.share(2, slots=slots, rows=64)                                # no tensor cores for it
    bad = L.ints([3, 99, 4])
    c.attend(0, q[:, :2].contiguous(), slots=bad, shared=c.share(2, slots=bad, plan=plan))
    assert c.status() == jd.JD_ERR_BAD_INDEX


def test_more_work_than_the_division_counts():
    """Caches whose sequences could have more tiles and rows than 32 bits hold: the call is the one without a plan."""
    B, T, heads = 8, 128, 64
    c = L.empty_cache(1, 40, 1024, heads, 1, 8, B + 1, 1 << 14, T, "f32", fill=1)
    c.reserve(2100, slots=L.ints([B]))
    c.seq_len[B:] = L.ints([2100])
    slots = torch.arange(B, dtype=torch.int32, device="cuda")
    c.fork(L.ints([B] * B), slots)
    c.reserve(T, slots=slots)
    q = rand((B, T, heads, 8), 3, "f32")
    plan = c.share(T, slots=slots, rows=16)
    assert shares(plan) and c.status() == jd.JD_OK
    got, want = c.attend(0, q, slots=slots, shared=plan), c.attend(0, q, slots=slots)
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"]) and torch.isfinite(want["out"]).all()


def test_a_plan_that_is_dropped_while_its_calls_run():
    """What is allocated behind the calls must not be the plan's memory as long as another stream's kernels have yet to use it."""
    c, slots = forked([1200], [6], [30] * 6, 3, q_heads=8, kv_heads=2, D=128)
    tree, _ = tree_of(3, 2)
    q, side = rand((6, 3, 8, 128), 5), torch.cuda.Stream()
    want = c.attend(0, q, tree, slots=slots)
    for given in (True, False):                    # as an argument, and as the current stream of the calls
        out = {name: torch.empty_like(x) for name, x in want.items()}
        plan = c.share(3, rows=128, slots=slots)
        need = plan.buffer.numel()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(50_000_000)          # some 30 ms
            if not given:
                c.attend(0, q, tree, slots=slots, shared=plan, out=out)
        if given:
            c.share(3, rows=128, slots=slots, plan=plan, stream=side)
            c.attend(0, q, tree, slots=slots, shared=plan, out=out, stream=side)
        del plan
        later = [torch.full((need,), 77, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert all(bool((x == 77).all()) for x in later)
        # weights are rounded to bf16 against another maximum, outputs once
        assert float((out["out"].float() - want["out"].float()).abs().max()) <= 4 * 2.0 ** -8 * float(c.v.abs().max())
        del later
