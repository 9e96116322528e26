"""Rotary positions, the paged cache and the attention of a drafted block against the CPU model in float64."""
import numpy as np
import pytest
import torch

import cache_testlib as L
from oracle import cache_oracle as O
from paper_2501_19309_b200 import jd

pytestmark = pytest.mark.gpu


def rand(shape, seed, dtype="bf16", scale=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(L.DT[dtype])


# ------------------------------------------------------------------------------------------- rotary positions
ROPE = [  # tokens, heads, head_dim, rot_dim, layout, dtype
    (1, 1, 64, 64, "half", "bf16"), (26, 40, 128, 128, "half", "bf16"), (7, 3, 128, 64, "half", "f32"),
    (300, 5, 80, 48, "interleaved", "bf16"), (33, 2, 256, 256, "interleaved", "f32"), (5, 4, 20, 6, "half", "bf16"),
    (9, 1, 7, 2, "interleaved", "f32"), (1025, 9, 96, 96, "half", "f32"), (4, 80, 128, 32, "interleaved", "bf16")]


def rope_bound(x, freq, pos, amplitude, dtype):
    """A turned element is two products of |x| <= X and a cosine that is off by 2^-22 (half turns rounded to float32: pi 2^-25;
    sincospi 2 ulp), summed in float32, and rounded once."""
    X = np.abs(x).max() * amplitude
    return 2 * X * 2.0 ** -21 + X * np.sqrt(2) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23)


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("n,heads,D,rot,layout,dtype", ROPE)
def test_rotate(n, heads, D, rot, layout, dtype, inverse):
    x = rand((n, heads, D), 1, dtype)
    pos = torch.randint(-3, 1 << 20, (n,), generator=torch.Generator().manual_seed(2)).to(torch.int32)
    if n > 2:
        pos[0], pos[1] = 2 ** 31 - 1, -2 ** 31
    freq, amp = jd.rope_frequencies(rot, 10000.0, "yarn", 4.0, 2048.0, 1.0, 32.0)
    r = jd.Rotary(freq.cuda(), layout, amp)
    want = O.rope(L.f64(x), pos.numpy(), freq.numpy(), layout, amp, inverse)
    got = r.rotate(x, pos.cuda(), inverse=inverse)
    assert np.abs(L.f64(got) - want).max() <= rope_bound(L.f64(x), freq, pos, amp, dtype)
    assert torch.equal(got[..., rot:], x[..., rot:])                    # what does not turn keeps its bits
    inplace = x.clone()
    assert r.rotate(inplace, pos.cuda(), out=inplace, inverse=inverse) is inplace
    assert torch.equal(inplace, got)


def test_rotate_strided_rows_leave_the_rest_alone():
    n, heads, D = 19, 4, 64
    for offset in (0, 1):            # the second one is not on 16 bytes: single elements
        buf = torch.full((n, 900), 7.0, dtype=torch.bfloat16, device="cuda")
        x = buf[:, offset:offset + heads * D].view(n, heads, D) if offset == 0 else buf.as_strided((n, heads, D), (900, D, 1), 1)
        x.copy_(rand((n, heads, D), 3))
        pos = L.ints(np.arange(n) * 1000)
        freq, _ = jd.rope_frequencies(64)
        r = jd.Rotary(freq.cuda())
        want = r.rotate(x.clone(memory_format=torch.contiguous_format), pos)
        got = r.rotate(x, pos, out=x)
        assert torch.equal(got, want)
        rest = torch.ones_like(buf, dtype=torch.bool)
        rest[:, offset:offset + heads * D] = False
        assert bool((buf[rest] == 7.0).all())


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_gradient(layout):
    """inverse=True is the transpose: against the formula's products and against differences (the map is linear, so a difference
    over a step of 1 is exact up to rounding)."""
    n, heads, D, rot = 3, 2, 16, 12
    freq, amp = jd.rope_frequencies(rot, 10000.0, "yarn", 8.0, 64.0)
    r = jd.Rotary(freq.cuda(), layout, amp)
    pos = L.ints([5, 100, 77777])
    x, gy = rand((n, heads, D), 4, "f32"), rand((n, heads, D), 5, "f32")
    gx = r.rotate(gy, pos, inverse=True)
    want = O.rope(L.f64(gy), pos.cpu().numpy(), freq.numpy(), layout, amp, inverse=True)
    assert np.abs(L.f64(gx) - want).max() <= rope_bound(L.f64(gy), freq, pos, amp, "f32")
    y0 = L.f64(r.rotate(x, pos))
    num = np.zeros((n, heads, D))
    for d in range(D):
        e = x.clone()
        e[..., d] += 1.0
        num[..., d] = ((L.f64(r.rotate(e, pos)) - y0) * L.f64(gy)).sum(-1)
    # each of the D products holds two rounded values of at most 5 x amplitude
    assert np.abs(num - L.f64(gx)).max() <= D * 2 * 2.0 ** -20 * 6 * np.abs(L.f64(gy)).max() * amp


def test_rotate_no_tokens():
    freq, _ = jd.rope_frequencies(8)
    x = torch.empty(0, 3, 8, device="cuda")
    assert jd.Rotary(freq.cuda()).rotate(x, torch.empty(0, dtype=torch.int32, device="cuda")).shape == (0, 3, 8)


# ------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("dtype,D,rot,layout", [("bf16", 128, 128, "half"), ("bf16", 64, 32, "interleaved"), ("f32", 40, 24, "half"),
                                                ("f32", 72, 72, "interleaved"), ("bf16", 64, 0, "half")])
@pytest.mark.parametrize("packed", [False, True])
def test_append(dtype, D, rot, layout, packed):
    rng = np.random.default_rng(3)
    lens, T, Hq, H = [0, 5, 31, 200, 16], 6, 4, 2
    c = L.filled_cache(lens, T, D=D, q_heads=Hq, kv_heads=H, layers=3, dtype=dtype, max_nodes=8)
    m = L.model_of(c)
    B = 4
    slots, nodes = L.ints([3, 0, -1, 1]), L.ints([6, 2, 6, 0])
    parents = [L.random_tree(T, rng) for _ in range(B)]
    tree = L.device_tree(parents, num_nodes=nodes)
    if packed:                       # q, k and v as slices of one projection
        qkv = rand((B, T, Hq + 2 * H, D), 6, dtype)
        q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
    else:
        q, k, v = rand((B, T, Hq, D), 6, dtype), rand((B, T, H, D), 7, dtype), rand((B, T, H, D), 8, dtype)
    freq = jd.rope_frequencies(rot, 10000.0)[0] if rot else None
    rotary = jd.Rotary(freq.cuda(), layout) if rot else None
    q_out = torch.full((B, T, Hq, D), 9.0, dtype=L.DT[dtype], device="cuda")
    k_before, v_before = c.k.clone(), c.v.clone()
    c.append(1, k, v, tree, rotary=rotary, q=q, q_out=q_out, slots=slots)
    assert c.status() == jd.JD_OK
    L.same_books(c, m)
    touched = torch.zeros_like(c.k, dtype=torch.bool)
    for b, slot in enumerate([3, 0, None, 1]):
        see, depth = O.visible(parents[b])
        n = int(nodes[b])
        if slot is None or n == 0:
            assert bool((q_out[b] == 9.0).all())
            continue
        pos = lens[slot] + depth
        if rot:
            wk, wq = (O.rope(L.f64(x[b]), pos, freq.numpy(), layout) for x in (k, q))
        else:
            wk, wq = L.f64(k[b]), L.f64(q[b])
        bound = rope_bound(L.f64(qkv if packed else q), freq, pos, 1.0, dtype) if rot else 0.0
        bound = max(bound, rope_bound(L.f64(k), freq, pos, 1.0, dtype)) if rot else 0.0
        assert np.abs(L.f64(q_out[b, :n]) - wq[:n]).max() <= bound
        assert bool((q_out[b, n:] == 9.0).all())
        for t in range(n):
            p, r = m.row(slot, lens[slot] + t)
            assert np.abs(L.f64(c.k[1, p, :, r]) - wk[t]).max() <= bound
            assert torch.equal(c.v[1, p, :, r], v[b, t])
            touched[1, p, :, r] = True
    assert torch.equal(c.k[~touched], k_before[~touched]) and torch.equal(c.v[~touched], v_before[~touched])


def test_append_reports_rows_without_a_page_of_their_own():
    c = L.filled_cache([14, 20], 0, layers=2, max_nodes=8)
    T = 4
    k, v = rand((2, T, 2, 64), 1), rand((2, T, 2, 64), 2)
    c.append(0, k, v)                                  # pages for 16 and 32 tokens: nodes 2, 3 of the first have none
    assert c.status() == jd.JD_ERR_BAD_INDEX
    assert torch.equal(c.v[0, int(c.page_table[0, 0]), :, 14:16].transpose(0, 1), v[0, :2])
    page = int(c.page_table[1, 1])
    assert torch.equal(c.v[0, page, :, 4:8].transpose(0, 1), v[1])
    c.refs[page] += 1                                  # another owner
    before = c.v.clone()
    c.append(0, k[1:], rand((1, T, 2, 64), 3), slots=L.ints([1]))
    assert c.status() == jd.JD_ERR_BAD_INDEX and torch.equal(c.v, before)
    c.append(0, k, v, slots=L.ints([1, 1]))            # the same slot twice
    assert c.status() == jd.JD_ERR_BAD_INDEX
    c.append(0, k, v, slots=L.ints([7, -5]))
    assert c.status() == jd.JD_ERR_BAD_INDEX
    assert c.status() == jd.JD_OK                      # a query clears it


# ------------------------------------------------------------------------------------------- attention
ATTEND = [  # lens, T, page, q_heads, kv_heads, D, dtype, variant, tree
    ([0], 1, 16, 1, 1, 64, "bf16", "simt", "chain"),
    ([1, 0, 63, 64, 65, 127, 128, 129], 5, 16, 4, 2, 64, "bf16", "simt", "tree"),
    ([300, 2], 9, 32, 6, 2, 80, "f32", "simt", "star"),
    ([37], 128, 8, 5, 1, 200, "f32", "simt", "tree"),
    ([1000], 3, 128, 8, 8, 8, "f32", "simt", "chain"),
    ([500, 1], 33, 64, 16, 1, 128, "bf16", "simt", "tree"),
    ([0], 1, 16, 1, 1, 64, "bf16", "tensor", "chain"),
    ([0, 1, 2], 1, 8, 8, 1, 128, "bf16", "tensor", "chain"),
    ([1, 0, 63, 64, 65, 127, 128, 129], 5, 16, 4, 2, 64, "bf16", "tensor", "tree"),
    ([255, 256, 257, 120, 383], 9, 32, 8, 2, 128, "bf16", "tensor", "tree"),
    ([700, 33], 26, 64, 8, 1, 128, "bf16", "tensor", "star"),             # 208 rows: two row tiles
    ([500, 127], 26, 128, 32, 2, 128, "bf16", "tensor", "tree"),          # 416 rows: two blocks
    ([100, 4000, 3], 128, 16, 4, 1, 64, "bf16", "tensor", "tree"),        # 512 rows
    ([2000, 5], 127, 256, 3, 1, 128, "bf16", "tensor", "chain"),
    ([5000], 1, 1024, 5, 5, 64, "bf16", "tensor", "chain"),
    ([9000, 17, 12000], 4, 8, 4, 1, 128, "bf16", "tensor", "tree"),
    ([20000], 2, 16, 16, 1, 128, "bf16", "tensor", "tree")]               # one segment over all SMs


def run_attend(c, m, T, parents, dtype, variant, seed, slots=None, num_nodes=None, scale=None, layer=0, B=None):
    B = len(c.seq_len) if B is None else B
    q = rand((B, T, c.q_heads, c.head_dim), seed, dtype)
    see = np.stack([O.visible(p)[0] for p in parents]) if isinstance(parents[0], list) else O.visible(parents)[0]
    tree = L.device_tree(parents, num_nodes=num_nodes)
    out = dict(out=torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda"), lse=torch.full(q.shape[:3], 5.0, device="cuda"))
    c.attend(layer, q, tree, scale=scale, out=out, slots=slots, variant=variant)
    assert c.status() == jd.JD_OK
    scale = c.head_dim ** -0.5 if scale is None else scale
    host = dict(slots=None if slots is None else slots.cpu().numpy(), num_nodes=None if num_nodes is None else num_nodes.cpu().numpy())
    want, lse = m.attend(layer, L.f64(q), see, scale, **host)
    tol, ltol = L.attend_tolerance(m, layer, L.f64(q), see, scale, np.nan_to_num(want), dtype, **host)
    return out, want, lse, tol, ltol


def check_attend(out, want, lse, tol, ltol):
    got, glse = L.f64(out["out"]), L.f64(out["lse"])
    rows = ~np.isnan(lse)
    assert (got[~rows] == 5.0).all() and (glse[~rows] == 5.0).all()       # rows that no node has are left as they were
    err = np.abs(got - want)[rows]
    assert (err <= tol[rows]).all(), (err.max(), (err - tol[rows]).max(), np.argwhere((err > tol[rows])).tolist()[:5])
    dead = np.isneginf(lse) & rows
    assert (got[dead] == 0).all() and np.isneginf(glse[dead]).all()
    live = rows & ~dead
    assert (np.abs(glse[live] - lse[live]) <= ltol[live] + 2.0 ** -22 * np.abs(lse[live])).all()


@pytest.mark.parametrize("lens,T,page,q_heads,kv_heads,D,dtype,variant,style", ATTEND)
def test_attend(lens, T, page, q_heads, kv_heads, D, dtype, variant, style):
    rng = np.random.default_rng(T)
    c = L.filled_cache(lens, T, page=page, q_heads=q_heads, kv_heads=kv_heads, D=D, dtype=dtype, max_nodes=T, seed=T)
    parents = [L.random_tree(T, rng, style) for _ in lens]
    r = run_attend(c, L.model_of(c), T, parents, dtype, variant, 11)
    check_attend(*r)
    again = run_attend(c, L.model_of(c), T, parents, dtype, variant, 11)
    assert torch.equal(r[0]["out"], again[0]["out"]) and torch.equal(r[0]["lse"], again[0]["lse"])


@pytest.mark.parametrize("T,q_heads,kv_heads,D,ctx", [(17, 10, 2, 128, 5338), (17, 6, 2, 128, 5338), (16, 32, 8, 64, 3333), (1, 8, 8, 128, 7000),
                                                      (26, 16, 2, 128, 3000), (3, 8, 8, 64, 2049)])
def test_attend_many_pieces_repeat_bit_for_bit(T, q_heads, kv_heads, D, ctx):
    """Sequences cut into pieces of odd numbers of tiles whose last tile ends behind the sequence: the same bits every time."""
    rng = np.random.default_rng(T)
    c = L.filled_cache([ctx] * 16, T, page=32, q_heads=q_heads, kv_heads=kv_heads, D=D, max_nodes=T, seed=1)
    q = rand((16, T, q_heads, D), 3)
    tree = L.device_tree([L.random_tree(T, rng) for _ in range(16)])
    first = c.attend(0, q, tree)
    simt = c.attend(0, q, tree, variant="simt")
    runs = [c.attend(0, q, tree) for _ in range(30)]
    torch.cuda.synchronize()
    for r in runs:
        assert torch.equal(r["out"], first["out"]) and torch.equal(r["lse"], first["lse"])
    # both kernels' outputs are weighted means of values of size 1: a weight that is off by 2^-8 moves them by no more than
    # 2^-8 of the sum of weight x |value|, which is below 1 here, and each rounds its output once
    assert (first["out"].float() - simt["out"].float()).abs().max() <= 2.0 ** -8 * (1 + 2 * simt["out"].float().abs().max())


@pytest.mark.parametrize("variant,dtype,D", [("simt", "f32", 72), ("tensor", "bf16", 64), ("tensor", "bf16", 128)])
@pytest.mark.parametrize("T,q_heads", [(1, 8), (5, 8), (26, 16), (26, 48)])
def test_attend_short_calls_behind_a_long_one(variant, dtype, D, T, q_heads):
    """A call that gives work to a part of the SMs reads nothing that an earlier, larger one left in the workspace."""
    c = L.filled_cache([7000], T, page=16, q_heads=q_heads, kv_heads=4, D=D, dtype=dtype, max_nodes=T, seed=3)
    parents = L.random_tree(T, np.random.default_rng(T), "tree")
    for n in (7000, 2500, 1300, 701, 300, 120, 3):
        c.truncate(L.ints([n]))
        c.reserve(T)
        check_attend(*run_attend(c, L.model_of(c), T, parents, dtype, variant, n))


@pytest.mark.parametrize("seed,kv_heads,group,D", [(0, 2, 4, 64), (1, 1, 8, 128), (2, 8, 1, 128), (3, 3, 10, 64)])
def test_attend_random_calls_on_one_cache(seed, kv_heads, group, D):
    """Calls of every size in turn, both kernels, on one workspace: none sees what another left."""
    rng = np.random.default_rng(seed)
    lens = [0, 1, 127, 400, 2000, 5000]
    c = L.filled_cache(lens, 40, page=16, q_heads=kv_heads * group, kv_heads=kv_heads, D=D, max_nodes=64, seed=seed)
    for call in range(24):
        if call % 3 == 2:                              # shorter, and longer again as far as the rows go
            b = int(rng.integers(0, 6))
            if int(c.seq_len[b]) > 0:
                c.seq_len[b] = int(rng.integers(0, lens[b] + 1))
        T = int(rng.choice([1, 2, 5, 9, 17, 33, 64]))
        slots = rng.choice([-1, 0, 1, 2, 3, 4, 5], int(rng.integers(1, 8)), replace=True).tolist()
        while len(slots) > 6:
            slots.pop()
        nodes = L.ints(rng.integers(0, T + 1, len(slots))) if rng.random() < 0.4 else None
        parents = [L.random_tree(T, rng, "tree") for _ in slots]
        variant = "simt" if rng.random() < 0.3 else "tensor"
        check_attend(*run_attend(c, L.model_of(c), T, parents, "bf16", variant, call, slots=L.ints(slots), num_nodes=nodes, B=len(slots)))


@pytest.mark.parametrize("T,group", [(32, 1), (33, 1), (16, 4), (65, 1), (128, 1), (43, 3), (16, 16), (86, 3), (128, 4), (1, 128)])
@pytest.mark.parametrize("D", [64, 128])
def test_attend_where_the_kernel_changes_its_form(T, group, D):
    """Rows (nodes x query heads of a kv head) on both sides of 32, 64, 128 and 256."""
    rng = np.random.default_rng(T + group)
    lens = [700, 130, 0]
    c = L.filled_cache(lens, T, page=16, q_heads=2 * group, kv_heads=2, D=D, max_nodes=T, seed=T)
    parents = [L.random_tree(T, rng) for _ in lens]
    check_attend(*run_attend(c, L.model_of(c), T, parents, "bf16", "tensor", 21))


VARIANTS = [("simt", "bf16", 64), ("simt", "f32", 72), ("tensor", "bf16", 64), ("tensor", "bf16", 128)]


@pytest.mark.parametrize("variant,dtype,D", VARIANTS)
def test_attend_slots_padding_layers_and_masks_that_leave_nothing(variant, dtype, D):
    """Padding entries, the same slot twice, padded blocks, another layer; a mask with empty rows on an empty sequence."""
    lens, T = [0, 70, 500, 3], 7
    c = L.filled_cache(lens, T, D=D, dtype=dtype, layers=3, max_nodes=T, seed=4)
    m = L.model_of(c)
    slots, nodes = L.ints([2, -1, 0, 1, 2, 3]), L.ints([7, 7, 5, 0, 3, -4])
    q = rand((6, T, 4, D), 9, dtype)
    see = np.tril(np.ones((T, T), dtype=bool))
    see[2] = False
    see[0, 0] = False
    tree = jd.Tree(T, mask=jd.mask_words(torch.from_numpy(see)).cuda(), num_nodes=nodes)
    out = dict(out=torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda"), lse=torch.full(q.shape[:3], 5.0, device="cuda"))
    c.attend(2, q, tree, scale=0.3, out=out, slots=slots, variant=variant)
    assert c.status() == jd.JD_OK
    host = dict(slots=slots.cpu().numpy(), num_nodes=nodes.cpu().numpy())
    want, lse = m.attend(2, L.f64(q), see, 0.3, **host)
    assert np.isneginf(lse[2, 0]).all() and np.isneginf(lse[2, 2]).all()       # the empty sequence's rows that see nothing
    check_attend(out, want, lse, *L.attend_tolerance(m, 2, L.f64(q), see, 0.3, np.nan_to_num(want), dtype, **host))


@pytest.mark.parametrize("variant,dtype,D", VARIANTS)
def test_attend_ignores_what_stands_in_hidden_rows(variant, dtype, D):
    """Rows behind the block, other pages and hidden nodes hold infinities and NaN; a node that is not finite spoils the rows
    that see it and no other."""
    lens, T = [130, 0, 257], 12
    c = L.filled_cache(lens, T, D=D, dtype=dtype, max_nodes=T, seed=5)
    m = L.model_of(c)
    parents = L.random_tree(T, np.random.default_rng(8), "star")
    clean = run_attend(c, m, T, parents, dtype, variant, 12)
    check_attend(*clean)
    junk = torch.tensor([float("nan"), float("inf"), float("-inf")], device="cuda").to(L.DT[dtype])
    used = torch.zeros(c.k.shape[1], c.k.shape[3], dtype=torch.bool, device="cuda")
    for s, n in enumerate(lens):
        for t in range(n + T):
            p, r = m.row(s, t)
            used[p, r] = True
    hidden = ~used[None, :, None, :, None].expand(c.k.shape)
    c.k[hidden] = junk[torch.arange(int(hidden.sum()), device="cuda") % 3]
    c.v[hidden] = junk[torch.arange(int(hidden.sum()), device="cuda") % 3]
    got = run_attend(c, m, T, parents, dtype, variant, 12)
    assert torch.equal(got[0]["out"], clean[0]["out"]) and torch.equal(got[0]["lse"], clean[0]["lse"])
    # node 3 of every sequence: only node 3's own rows see it
    for s, n in enumerate(lens):
        p, r = m.row(s, n + 3)
        c.k[0, p, :, r] = float("nan")
        c.v[0, p, 0, r, 5] = float("inf")
        c.v[0, p, 1, r, 6] = float("nan")
    got = run_attend(c, m, T, parents, dtype, variant, 12)[0]
    keep = [t for t in range(T) if t != 3]
    assert torch.equal(got["out"][:, keep], clean[0]["out"][:, keep]) and torch.equal(got["lse"][:, keep], clean[0]["lse"][:, keep])
    assert bool(torch.isnan(got["out"][:, 3]).all())
    # values alone: the element is spoilt, its row's other elements are not
    for s, n in enumerate(lens):
        p, r = m.row(s, n + 3)
        c.k[0, p, :, r] = 0.25
    got = run_attend(c, m, T, parents, dtype, variant, 12)[0]["out"].float()
    assert torch.equal(got[:, keep], clean[0]["out"].float()[:, keep])
    assert bool(torch.isinf(got[:, 3, :2, 5]).all()) and bool(torch.isnan(got[:, 3, 2:, 6]).all())
    assert bool(torch.isfinite(got[:, 3, :2, 6]).all()) and bool(torch.isfinite(got[:, 3, 2:, 5]).all())


@pytest.mark.parametrize("variant,dtype,D", VARIANTS)
def test_attend_extreme_scores(variant, dtype, D):
    """Maxima that jump from tile to tile, scores of hundreds, and keys of the type's lowest value."""
    lens, T = [900], 4
    c = L.filled_cache(lens, T, D=D, dtype=dtype, max_nodes=T, seed=6)
    gen = torch.Generator().manual_seed(1)
    order = L.f64(c.page_table[0, :-4]).astype(int)
    for i, p in enumerate(order):                       # growing keys, then a jump, then small ones
        c.k[0, p] *= (0.1 + 0.2 * i) if i < 40 else (20.0 if i == 41 else 0.01)
    c.k[0, order[3], :, 2] = torch.finfo(L.DT[dtype]).min / 1e30
    r = run_attend(c, L.model_of(c), T, L.random_tree(T, np.random.default_rng(2)), dtype, variant, 13)
    # scores of hundreds: the bound's A is large, so compare where it says something
    got, want, tol = L.f64(r[0]["out"]), r[1], r[3]
    assert np.isfinite(got).all() and (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("variant,dtype,D", VARIANTS)
def test_attend_strided_queries_and_outputs(variant, dtype, D):
    c = L.filled_cache([40, 9], 5, D=D, dtype=dtype, max_nodes=5)
    qkv = rand((2, 5, 8, D), 3, dtype)
    q = qkv[:, :, :4]
    buf = torch.zeros(2, 5, 6, D, dtype=q.dtype, device="cuda")
    a = c.attend(0, q, variant=variant)
    b = c.attend(0, q.contiguous(), out=dict(out=buf[:, :, 1:5]), variant=variant)
    assert torch.equal(a["out"], b["out"]) and bool((buf[:, :, 0] == 0).all()) and bool((buf[:, :, 5] == 0).all())


@pytest.mark.parametrize("variant", ["simt", "tensor"])
def test_attend_beyond_four_gigabytes(variant):
    """The sequence's pages lie at both ends of a pool of more than 2^32 bytes and 2^31 elements."""
    page, H, D, layers = 64, 8, 128, 2
    pages = (1 << 31) // (layers * H * page * D) + 40
    c = L.empty_cache(layers, pages, page, 8, H, D, 1, 8, 4)
    assert c.k.numel() > 1 << 31
    rows = [pages - 1, 0, pages - 2, pages // 2, 1]
    c.page_table[0, :5] = L.ints(rows)
    c.refs[rows] = 1
    c.seq_len[0], c.held[0] = 300, 5
    small = L.filled_cache([300], 4, page=page, q_heads=8, kv_heads=H, D=D, max_nodes=4, seed=9)
    for i, p in enumerate(rows):
        c.k[1, p], c.v[1, p] = small.k[0, int(small.page_table[0, i])], small.v[0, int(small.page_table[0, i])]
    q = rand((1, 4, 8, D), 5)
    a, b = c.attend(1, q, variant=variant), small.attend(0, q, variant=variant)
    assert c.status() == jd.JD_OK
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])
    k, v = rand((1, 4, H, D), 6), rand((1, 4, H, D), 7)
    c.append(1, k, v)
    at = [(rows[t // page], t % page) for t in range(300, 304)]
    assert all(torch.equal(c.k[1, p, :, r], k[0, i]) and torch.equal(c.v[1, p, :, r], v[0, i]) for i, (p, r) in enumerate(at))
    c.close()


# ------------------------------------------------------------------------------------------- pages
@pytest.mark.parametrize("seed,dtype,page,layers,H,D", [(0, "bf16", 8, 2, 1, 8), (1, "f32", 8, 1, 2, 16), (2, "bf16", 16, 3, 2, 64),
                                                        (3, "bf16", 32, 1, 3, 40), (4, "f32", 64, 2, 1, 8)])
def test_random_programs_against_the_model(seed, dtype, page, layers, H, D):
    """Reserve, append, commit, fork, truncate and compact in random order, bad entries among them: tables, owners and the
    sequences' rows stay those of the model, bit for bit."""
    rng = np.random.default_rng(seed)
    seqs, per_seq, T = 12, 6, 9
    c = L.empty_cache(layers, 40, page, H, H, D, seqs, per_seq, T, dtype, fill=seed)
    m = L.model_of(c)

    def pick(n, bad=0.1):
        s = rng.permutation(seqs)[:n].tolist()
        return [int(rng.choice([-1, seqs, -3, s[0]])) if rng.random() < bad else x for x in s]

    for step in range(60):
        m.status = O.OK
        n = int(rng.integers(1, 6))
        op = rng.choice(["step", "step", "step", "fork", "truncate", "free", "reserve", "compact"])
        if op == "step":
            slots = pick(n)
            t = int(rng.integers(1, T + 1))
            c.reserve(t, L.ints(slots)); m.reserve(t, slots)
            for layer in range(layers):
                k, v = rand((n, t, H, D), 1000 + step, dtype), rand((n, t, H, D), 2000 + step, dtype)
                c.append(layer, k, v, slots=L.ints(slots)); m.append(layer, L.f64(k), L.f64(v), slots)
            if t == 1 or rng.random() < 0.3:
                acc = rng.integers(-1, t + 1, n)
                c.commit(L.ints(acc), slots=L.ints(slots), path_len=t - 1); m.commit(acc, None, slots, t - 1)
            else:
                paths = np.sort(rng.permuted(np.tile(np.arange(1, t), (n, 3, 1)), axis=2)[:, :, :int(rng.integers(1, t))], axis=2)
                if rng.random() < 0.15:
                    paths[0, 0, -1] = rng.integers(-2, T + 2)
                acc = rng.integers(0, paths.shape[2] + 1, (n, 3))
                chosen = c.commit(L.ints(acc), L.ints(paths), slots=L.ints(slots)).cpu().numpy()
                for i, want in m.commit(acc, paths, slots).items():
                    assert chosen[i] == want
        elif op == "reserve":
            slots, t = pick(n), int(rng.integers(1, 3 * page))
            c.reserve(t, L.ints(slots)); m.reserve(t, slots)
        elif op == "fork":
            src = rng.integers(0, seqs, n).tolist()
            empty = [s for s in range(seqs) if m.held[s] == 0 and m.len[s] == 0]
            dst = [int(rng.choice(empty)) if empty and rng.random() < 0.8 else int(rng.integers(-2, seqs + 1)) for _ in range(n)]
            c.fork(L.ints(src), L.ints(dst)); m.fork(src, dst)
        elif op == "truncate":
            slots = pick(n)
            to = [int(rng.integers(-1, m.len[s] + 2)) if 0 <= s < seqs else 0 for s in slots]
            c.truncate(L.ints(to), L.ints(slots)); m.truncate(to, slots)
        elif op == "free":
            slots = pick(n)
            c.free(L.ints(slots)); m.truncate(None, slots, n)
        else:
            assert int(c.compact()) == m.compact()
        status = c.status()
        assert (status == jd.JD_OK) == (m.status == O.OK), (step, op, status, m.status)
        L.same_books(c, m)
        for s in range(seqs):
            for layer in range(layers):
                for h in range(H):
                    want = m.sequence(layer, h, s)
                    pages = torch.as_tensor(m.table[s, :m.held[s]], device="cuda")
                    for x, w in zip((c.k, c.v), want):
                        got = L.f64(x[layer, pages, h].reshape(-1, D)[:len(w)])
                        assert np.array_equal(got, w), (step, op, s)


def test_reserve_is_all_or_nothing_and_takes_the_lowest_pages():
    c = L.empty_cache(1, 70, 8, 1, 1, 8, 3, 64, 4)
    c.reserve(33 * 8, L.ints([0]))                      # pages 0..32: past a word of the bitmap
    assert c.status() == jd.JD_OK and c.page_table[0, :33].cpu().tolist() == list(range(33))
    before = [x.clone() for x in (c.page_table, c.held, c.refs, c.free_bits)]
    c.reserve(20 * 8, L.ints([1, 2]))                   # 40 pages of 37
    assert c.status() == jd.JD_ERR_PAGES
    c.reserve(65 * 8, L.ints([1]))                      # more than a table has
    assert c.status() == jd.JD_ERR_PAGES
    c.reserve((1 << 31) - 1, L.ints([1]))
    assert c.status() == jd.JD_ERR_PAGES
    assert all(torch.equal(x, y) for x, y in zip(before, (c.page_table, c.held, c.refs, c.free_bits)))
    c.reserve(37 * 8, L.ints([1]))                      # the last 37
    assert c.status() == jd.JD_OK and bool((c.free_bits == 0).all())
    c.free(L.ints([0]))
    c.reserve(1, L.ints([2]))
    assert c.status() == jd.JD_OK and int(c.page_table[2, 0]) == 0 and int(c.held[0]) == 0


def test_large_pool_and_many_sequences():
    """A pool of more words than the reserving block has threads, and a call of 1024 sequences."""
    c = L.empty_cache(1, 50000, 8, 1, 1, 8, 1024, 64, 4)
    c.reserve(8 * 48)                                   # 49152 pages
    assert c.status() == jd.JD_OK
    assert torch.equal(c.page_table[:, :48].flatten().cpu(), torch.arange(49152, dtype=torch.int32))
    c.reserve(8 * 49)
    assert c.status() == jd.JD_ERR_PAGES
    odd = torch.arange(1, 1024, 2, dtype=torch.int32, device="cuda")
    c.free(odd)
    assert c.status() == jd.JD_OK and int((c.refs == 0).sum()) == 50000 - 49152 + 512 * 48
    assert int(c.compact()) == 512 * 48
    assert bool((c.refs[:512 * 48] == 1).all()) and bool((c.refs[512 * 48:] == 0).all())


def test_forks_share_until_they_write():
    c = L.empty_cache(2, 16, 8, 1, 1, 8, 4, 4, 4, fill=3)
    c.reserve(4, L.ints([0]))
    for layer in range(2):
        c.append(layer, rand((1, 4, 1, 8), layer), rand((1, 4, 1, 8), 9), slots=L.ints([0]))
    c.commit(L.ints([2]), slots=L.ints([0]))            # 3 tokens in one page
    c.fork(L.ints([0, 0]), L.ints([1, 3]))
    assert c.status() == jd.JD_OK and int(c.refs[0]) == 3 and c.seq_len.cpu().tolist() == [3, 3, 0, 3]
    c.append(0, rand((1, 1, 1, 8), 1), rand((1, 1, 1, 8), 2), slots=L.ints([1]))      # not reserved: shared
    assert c.status() == jd.JD_ERR_BAD_INDEX
    c.reserve(2, L.ints([1, 0, 3]))                     # the last of the three keeps the page
    assert c.status() == jd.JD_OK
    assert [int(c.page_table[s, 0]) for s in (0, 1, 3)] == [2, 1, 0] and c.refs[:3].cpu().tolist() == [1, 1, 1]
    for s in (0, 1):
        p = int(c.page_table[s, 0])
        assert torch.equal(c.k[:, p, :, :3], c.k[:, 0, :, :3]) and torch.equal(c.v[:, p, :, :3], c.v[:, 0, :, :3])


@pytest.mark.parametrize("tree", [False, True])
def test_commit_leaves_rows_of_shared_pages_alone(tree):
    """A reserve that finds no pages leaves a page shared; the rest of the step then takes and moves nothing in it."""
    c = L.empty_cache(2, 1, 8, 1, 1, 8, 2, 4, 4)
    c.reserve(4, L.ints([0]))
    for layer in range(2):
        c.append(layer, rand((1, 4, 1, 8), layer), rand((1, 4, 1, 8), 9), slots=L.ints([0]))
    c.commit(L.ints([3]), slots=L.ints([0]), path_len=3)
    c.fork(L.ints([0]), L.ints([1]))
    c.truncate(L.ints([1]), L.ints([0]))
    assert c.status() == jd.JD_OK
    k, v = c.k.clone(), c.v.clone()
    c.reserve(4, L.ints([0]))
    assert c.status() == jd.JD_ERR_PAGES
    for layer in range(2):
        c.append(layer, rand((1, 4, 1, 8), 5), rand((1, 4, 1, 8), 6), slots=L.ints([0]))
    c.commit(L.ints([[1]]), L.ints([[[2]]]) if tree else None, slots=L.ints([0]), path_len=3)
    assert c.status() == jd.JD_ERR_BAD_INDEX
    assert torch.equal(c.k, k) and torch.equal(c.v, v) and c.seq_len.cpu().tolist() == [1, 4] and c.refs.cpu().tolist() == [2]
    c.free(L.ints([1]))                                 # now the page is the first one's alone
    c.reserve(3, L.ints([0]))
    c.commit(L.ints([[1]]), L.ints([[[2]]]), slots=L.ints([0]))
    assert c.status() == jd.JD_OK and int(c.seq_len[0]) == 3 and torch.equal(c.k[:, 0, :, 2], k[:, 0, :, 3])


def test_bits_behind_the_last_page_are_not_handed_out():
    c = L.empty_cache(1, 5, 8, 1, 1, 8, 2, 16, 4)
    c.free_bits.fill_(-1)
    c.reserve(6 * 8, L.ints([0]))
    assert c.status() == jd.JD_ERR_PAGES and int(c.held[0]) == 0
    c.reserve(5 * 8, L.ints([0]))
    assert c.status() == jd.JD_OK and c.page_table[0, :5].cpu().tolist() == [0, 1, 2, 3, 4] and c.refs.cpu().tolist() == [1] * 5


def test_broadcast_inputs_and_gradients_are_refused():
    c = L.filled_cache([20, 30], 4, max_nodes=4)
    q = rand((1, 1, 4, 64), 1).expand(2, 4, 4, 64)
    with pytest.raises(ValueError):
        c.attend(0, q)
    with pytest.raises(ValueError):
        c.append(0, q[:, :, :2], q[:, :, :2])
    with pytest.raises(ValueError):
        c.attend(0, rand((2, 4, 4, 64), 1).requires_grad_())
    assert c.status() == jd.JD_OK


# ------------------------------------------------------------------------------------------- refusals
def refused(f, status=jd.JD_ERR_INVALID_ARG):
    with pytest.raises(jd.JdError) as e:
        f()
    assert e.value.status == status


def test_refusals():
    c = L.filled_cache([20, 30], 4, max_nodes=4)
    q, k = rand((2, 4, 4, 64), 1), rand((2, 4, 2, 64), 2)
    for layer in (-1, 1):
        refused(lambda: c.attend(layer, q))
        refused(lambda: c.append(layer, k, k))
    refused(lambda: c.attend(0, rand((2, 5, 4, 64), 1)))                  # more nodes than max_nodes
    refused(lambda: c.attend(0, rand((3, 4, 4, 64), 1)))                  # more sequences than slots
    refused(lambda: c.attend(0, q, out=dict(out=q)))
    for scale in (float("nan"), float("inf"), 0.0, -0.1):
        refused(lambda: c.attend(0, q, scale=scale))
    refused(lambda: c.attend(0, q, variant=3))
    refused(lambda: c.reserve(0))
    refused(lambda: c.commit(L.ints([1, 1]), path_len=4))
    refused(lambda: c.commit(L.ints([1, 1]), path_len=-1))
    f32 = L.filled_cache([20], 4, dtype="f32", max_nodes=4)
    refused(lambda: f32.attend(0, rand((1, 4, 4, 64), 1, "f32"), variant="tensor"), jd.JD_ERR_UNSUPPORTED)
    odd = L.filled_cache([20], 4, D=72, max_nodes=4)
    refused(lambda: odd.attend(0, rand((1, 4, 4, 72), 1), variant="tensor"), jd.JD_ERR_UNSUPPORTED)
    freq, _ = jd.rope_frequencies(128)
    refused(lambda: c.append(0, k, k, rotary=jd.Rotary(freq.cuda())))     # wider than a head
    # alignment and strides that 16-byte accesses cannot take
    buf = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    refused(lambda: c.attend(0, buf[1:1 + 2 * 4 * 256].view(2, 4, 4, 64)))
    wide = torch.zeros(2, 4, 260, dtype=torch.bfloat16, device="cuda")
    refused(lambda: c.attend(0, wide[..., :256].unflatten(2, (4, 64))))
    with pytest.raises(ValueError):
        c.attend(0, rand((2, 4, 4, 128), 1))
    with pytest.raises(ValueError):
        c.attend(0, q.float())
    with pytest.raises(ValueError):
        c.reserve(1, slots=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        c.attend(0, q, jd.Tree(3))
    with pytest.raises(ValueError):
        c.attend(0, q.transpose(1, 2).contiguous().transpose(1, 2))
    for kw in (dict(page=24), dict(page=4), dict(D=12), dict(D=264), dict(max_nodes=129), dict(q_heads=3)):
        with pytest.raises(jd.JdError):
            L.filled_cache([4], 1, **kw)
    assert c.status() == jd.JD_OK


# ------------------------------------------------------------------------------------------- together
def decode_step(c, layers, T, tree, slots, tokens, rotary, dtype, seed):
    """One step's cache work for a made-up target: every layer's k, v, q are drawn; returns the last layer's outputs."""
    B = slots.shape[0]
    c.reserve(T, slots)
    for layer in range(layers):
        k, v, q = (rand((B, T, h, c.head_dim), seed + 10 * layer + i, dtype) for i, h in enumerate((c.kv_heads, c.kv_heads, c.q_heads)))
        q = c.append(layer, k, v, tree, rotary=rotary, q=q, slots=slots)
        out = c.attend(layer, q, tree, slots=slots)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_with_verification(dtype):
    """Reserve, append, attend, verify, commit as a decoding loop makes them: the accept lengths go from jd_verify to the
    cache on the device, and after every step the cache holds what a cache that got only the kept tokens holds."""
    import jd_testlib as JT
    from paper_2501_19309_b200 import inputs as I
    B, M, layers, Hq, H, D = 3, 5, 2, 4, 2, 64
    d = Hq * D
    wl = I.CONFIGS[1].scaled("steps", B=B, M=M, d=d, V=3000)
    c = L.empty_cache(layers, 64, 8, Hq, H, D, B, 20, M + 1, dtype)
    ref = L.model_of(c)
    freq, _ = jd.rope_frequencies(D, 10000.0)
    rotary = jd.Rotary(freq.cuda())
    tree = jd.Tree(M + 1)
    slots = L.ints([2, 0, 1])
    total = np.zeros(B, dtype=int)
    for step in range(4):
        out = decode_step(c, layers, M + 1, tree, slots, None, rotary, dtype, 100 * step)
        inp = I.make_inputs(wl, step)
        dev = JT.upload(inp)
        ver = JT.make_verifier(inp, dev)
        Hs = out["out"].reshape(B, M + 1, d).to(torch.bfloat16).contiguous()
        res = ver.verify(Hs, dev["x"], dev["dl"], inp.tau, step, "judge_or_standard")
        before = c.seq_len.clone()
        c.commit(res["accept_len"], slots=slots, path_len=M)
        assert c.status() == jd.JD_OK and ver.device_status() == jd.JD_OK
        a = res["accept_len"].cpu().numpy()
        assert np.array_equal((c.seq_len - before)[slots.long()].cpu().numpy(), a + 1)
        # the kept tokens alone, through the model
        ref.reserve(M + 1, slots.cpu().numpy())
        for layer in range(layers):
            k, v = (L.f64(rand((B, M + 1, H, D), 100 * step + 10 * layer + i, dtype)) for i in range(2))
            ref.append(layer, k, v, slots.cpu().numpy())
        ref.commit(a, None, slots.cpu().numpy(), M)
        L.same_books(c, ref)
        for s in range(B):
            for layer in range(layers):
                for h in range(H):
                    k, v = ref.sequence(layer, h, s)
                    pages = torch.as_tensor(ref.table[s, :ref.held[s]], device="cuda")
                    assert np.array_equal(L.f64(c.v[layer, pages, h].reshape(-1, D)[:len(v)]), v)
        total += a + 1
        ver.close()
    assert total.sum() > B


def test_tree_step_equals_the_chain_that_was_kept():
    """A tree is attended and its longest accepted path committed; the same tokens as a chain give the same rows, and the next
    block's attention is bit for bit the same."""
    Hq, H, D, page = 4, 2, 64, 16
    parents = [-1, 0, 0, 1, 1, 2, 3, 5]
    tree = L.device_tree(parents)
    paths = [[[1, 3, 6], [2, 5, 7]]]                       # two root-to-leaf paths
    acc = [[1, 3]]
    freq, _ = jd.rope_frequencies(D, 10000.0)
    rotary = jd.Rotary(freq.cuda())
    a = L.filled_cache([37], 0, page=page, max_nodes=8, seed=3, spare=6)
    b = L.filled_cache([37], 0, page=page, max_nodes=8, seed=3, spare=6)
    T = len(parents)
    k, v, q = rand((1, T, H, D), 1), rand((1, T, H, D), 2), rand((1, T, Hq, D), 3)
    a.reserve(T)
    qa = a.append(0, k, v, tree, rotary=rotary, q=q)
    oa = a.attend(0, qa, tree)
    chosen = a.commit(L.ints(acc), L.ints(paths))
    assert a.status() == jd.JD_OK and chosen.cpu().tolist() == [1]
    keep = [0, 2, 5, 7]
    b.reserve(4)
    qb = b.append(0, k[:, keep].contiguous(), v[:, keep].contiguous(), rotary=rotary, q=q[:, keep].contiguous())
    ob = b.attend(0, qb)
    b.commit(L.ints([3]), path_len=3)
    assert torch.equal(qa[:, keep], qb)
    # same rows, other tile columns: the softmax weights' sums run in another order
    assert (oa["out"][:, keep].float() - ob["out"].float()).abs().max() <= 2.0 ** -7 * ob["out"].float().abs().max()
    assert torch.equal(a.seq_len, b.seq_len) and torch.equal(a.held, b.held)
    nxt = rand((1, 3, Hq, D), 7)
    for c in (a, b):
        c.reserve(3)
        c.append(0, rand((1, 3, H, D), 8), rand((1, 3, H, D), 9))
    oa, ob = a.attend(0, nxt), b.attend(0, nxt)
    assert torch.equal(oa["out"], ob["out"]) and torch.equal(oa["lse"], ob["lse"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_captured_step_replays(dtype):
    """A whole step in a CUDA graph, replayed while lengths grow: the lengths are read on the device."""
    B, T, layers, Hq, H, D = 2, 3, 2, 4, 2, 64
    freq, _ = jd.rope_frequencies(D, 10000.0)
    rotary = jd.Rotary(freq.cuda())
    eager = L.filled_cache([30, 2], 0, page=8, layers=layers, max_nodes=T, dtype=dtype, spare=40, seed=1)
    graph = L.filled_cache([30, 2], 0, page=8, layers=layers, max_nodes=T, dtype=dtype, spare=40, seed=1)
    k, v, q = rand((B, T, H, D), 1, dtype), rand((B, T, H, D), 2, dtype), rand((B, T, Hq, D), 3, dtype)
    acc = L.ints([2, 1])

    def step(c, q_out, out, chosen):
        c.reserve(T)
        for layer in range(layers):
            c.append(layer, k, v, rotary=rotary, q=q, q_out=q_out)
            c.attend(layer, q_out, out=out)
        c.commit(acc, chosen=chosen, path_len=T - 1)

    bufs = [(torch.empty_like(q), dict(out=torch.empty_like(q), lse=torch.empty(B, T, Hq, device="cuda")),
             torch.empty(B, dtype=torch.int32, device="cuda")) for _ in range(2)]
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        step(graph, *bufs[1])
    for _ in range(5):
        step(eager, *bufs[0])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(bufs[0][1]["out"], bufs[1][1]["out"]) and torch.equal(bufs[0][1]["lse"], bufs[1][1]["lse"])
        for name in ("page_table", "seq_len", "held", "refs", "free_bits", "k", "v"):
            assert torch.equal(getattr(eager, name), getattr(graph, name)), name
    assert eager.seq_len.cpu().tolist() == [45, 12]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_in_a_row_equal_calls_that_are_waited_for(dtype):
    """Kernels start behind one another's launch: many steps without a wait leave what the same steps leave with one after every call."""
    B, T, layers, Hq, H, D = 5, 7, 3, 8, 2, 64
    freq, _ = jd.rope_frequencies(D, 10000.0)
    rotary = jd.Rotary(freq.cuda(), "interleaved")
    rng = np.random.default_rng(4)
    parents = L.random_tree(T, rng)
    tree = L.device_tree(parents)
    paths = np.sort(np.stack([rng.permuted(np.arange(1, T))[:4] for _ in range(B * 3)]).reshape(B, 3, 4), axis=2)
    results = []
    for wait in (True, False):
        sync = torch.cuda.synchronize if wait else (lambda: None)
        c = L.filled_cache([60, 5, 130, 0, 33], 0, page=8, layers=layers, q_heads=Hq, kv_heads=H, D=D, max_nodes=T, dtype=dtype, spare=200,
                           extra_seqs=2, seed=7)
        kept = []
        torch.cuda.synchronize()
        for step in range(12):
            k, v, q = (rand((B, T, h, D), 10 * step + i, dtype) for i, h in enumerate((H, H, Hq)))
            acc = torch.randint(0, 5, (B, 3), generator=torch.Generator().manual_seed(step)).to(torch.int32).cuda()
            slots = L.ints([0, 1, 2, 3, 4])
            c.reserve(T, slots); sync()
            for layer in range(layers):
                qq = c.append(layer, k, v, tree, rotary=rotary, q=q, slots=slots); sync()
                o = c.attend(layer, qq, tree, slots=slots); sync()
                kept += [qq, o["out"], o["lse"]]
            kept.append(c.commit(acc, L.ints(paths), slots=slots)); sync()
            if step == 5:
                c.fork(L.ints([2, 0]), L.ints([5, 6])); sync()
                c.truncate(L.ints([3]), L.ints([1])); sync()
            if step == 8:
                c.free(L.ints([5])); sync()
                kept.append(c.compact()); sync()
        # the first sequence outgrows its table of 12 pages on the way: from there on reserves are refused, which has to repeat as well
        assert c.status() == jd.JD_ERR_PAGES
        results.append(kept + [c.k, c.v, c.page_table, c.seq_len, c.held, c.refs, c.free_bits])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_two_handles_attend_on_two_streams():
    """Handles on the same buffers, each with its own workspace, at the same time."""
    a = L.filled_cache([5000, 700], 9, q_heads=8, kv_heads=1, D=128, max_nodes=9, seed=2)
    b = jd.PagedCache(a.k, a.v, a.page_table, a.seq_len, a.held, a.refs, a.free_bits, q_heads=8, max_nodes=9)
    qa, qb = rand((2, 9, 8, 128), 1), rand((2, 9, 8, 128), 2)
    want = a.attend(0, qa), a.attend(0, qb)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for _ in range(20):
        outs.append((a.attend(0, qa, stream=sa), b.attend(0, qb, stream=sb)))
    torch.cuda.synchronize()
    for x, y in outs:
        assert torch.equal(x["out"], want[0]["out"]) and torch.equal(y["out"], want[1]["out"])


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_a_captured_step_with_a_side_stream(dtype, D):
    """Calls that start early, between branches that part and meet: the same as one after another."""
    c = L.filled_cache([300, 2000], 8, D=D, dtype=dtype, max_nodes=8, seed=4)
    q, k, v = (rand((2, 8, h, D), i, dtype) for i, h in enumerate((4, 2, 2)))
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    first, second = ({"out": torch.zeros_like(q)} for _ in range(2))
    turned, other = torch.zeros_like(q), torch.zeros_like(q)

    def step(branch):
        torch.add(q, 0, out=turned)
        c.append(0, k, v)
        c.attend(0, turned, out=first)
        if branch:
            side.wait_stream(main)
        with torch.cuda.stream(side if branch else main):
            torch.mul(first["out"], 2, out=other)
            torch.neg(turned, out=turned)
        c.append(0, v, k)
        if branch:
            main.wait_stream(side)
        torch.add(other, turned, out=other)
        c.attend(0, other, out=second)

    torch.cuda.synchronize()
    with torch.cuda.stream(main):
        step(False)
        torch.cuda.synchronize()
        want = [first["out"].clone(), second["out"].clone()]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=main):
            step(True)
        for _ in range(3):
            first["out"].zero_(), second["out"].zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(first["out"], want[0]) and torch.equal(second["out"], want[1])
    assert c.status() == jd.JD_OK


@pytest.mark.parametrize("layers,H,D", [(1, 1, 8), (3, 2, 64)])
def test_commit_of_paths_with_several_bad_nodes(layers, H, D):
    """Nodes behind a cut count for nothing, whatever they say: negative ones in a row, a row that falls and rises again, tables used to
    their last entry."""
    per_seq, page, T = 2, 8, 8
    paths = [[-5, -3, -1], [7, 1, 2], [1, 3, 2], [-1, 0, 2], [2, 1, 3], [9, 10, 11], [2, 2, 3], [1, 2, 4]]
    for room in (1, 3, 8):
        for order in (paths, paths[::-1]):
            B = len(order)
            c = L.empty_cache(layers, B * per_seq + 2, page, H, H, D, B, per_seq, T, fill=room)
            c.reserve(per_seq * page)
            c.commit(L.ints([6] * B), path_len=6)                              # 7 tokens
            c.reserve(per_seq * page - 7)
            if page * per_seq - room > 7:
                c.commit(L.ints([min(page * per_seq - room - 8, 7)] * B), path_len=7)
                c.reserve(room)
            assert c.status() == jd.JD_OK and bool((c.held == per_seq).all())
            m = L.model_of(c)
            chosen = c.commit(L.ints([[3]] * B), L.ints([[p] for p in order]))
            m.commit([[3]] * B, np.array([[p] for p in order]), list(range(B)))
            assert c.status() == jd.JD_ERR_BAD_INDEX and m.status == O.BAD_INDEX and bool((chosen == 0).all())
            L.same_books(c, m)
            assert np.array_equal(L.f64(c.k), m.k) and np.array_equal(L.f64(c.v), m.v)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,group", [(26, 8), (26, 16), (12, 8), (12, 4), (6, 4)])
def test_values_that_are_not_finite_in_pieces_that_follow_one_another(D, T, group):
    """A CTA's pieces are of sequences with trees and node counts of their own, most of them a tile long; in every third sequence
    a node's value is infinite. Each row gets the infinities of the nodes that it sees, and no others."""
    B = 600
    rng = np.random.default_rng(T)
    lens = [int(x) for x in rng.integers(0, 100, B)]
    c = L.filled_cache(lens, T, page=16, q_heads=group, kv_heads=1, D=D, max_nodes=T, seed=1)
    parents = [L.random_tree(T, rng, ("chain", "star", "star")[b % 3]) for b in range(B)]
    count = [(T, 1, T)[b % 3] for b in range(B)]
    tree = L.device_tree(parents, num_nodes=L.ints(count))
    q = rand((B, T, group, D), 2)
    clean = c.attend(0, q, tree)["out"].float()
    at = torch.tensor(lens)[::3] + 3                          # node 3 of sequences 0, 3, ..
    page, row = c.page_table[::3].cpu()[torch.arange(len(at)), at // 16].long().cuda(), (at % 16).cuda()
    c.v[0, page, 0, row, 5] = float("inf")
    c.v[0, page, 0, row, D - 1] = float("-inf")
    alive = (torch.arange(T)[None, :] < torch.tensor(count)[:, None]).cuda()
    want = clean.clone()
    want[::3, 3:, :, 5] = float("inf")                       # of a chain, every node from 3 on sees node 3
    want[::3, 3:, :, D - 1] = float("-inf")
    for _ in range(20):
        got = c.attend(0, q, tree)["out"].float()
        same = (got == want)[alive]
        assert bool(same.all()), int((~same).sum())
    assert c.status() == jd.JD_OK


def test_a_reserve_of_two_to_the_31_pages_is_refused():
    """1024 sequences that ask for 2^21 pages each: the sum does not fit 31 bits."""
    c = jd.PagedCache.allocate(1, 16, 8, 1, 1, 8, 1024, 1 << 21, 4)
    c.reserve(1 << 24)
    assert c.status() == jd.JD_ERR_PAGES and bool((c.held == 0).all()) and bool((c.refs == 0).all())
    c.reserve(8, L.ints([1000, 3]))
    assert c.status() == jd.JD_OK and c.page_table[[1000, 3], 0].cpu().tolist() == [0, 1]
    c.close()


def test_padding_entries_of_a_fork_name_nothing():
    """An entry with -1 on either side is no source and no target for the others."""
    c = L.empty_cache(1, 8, 8, 1, 1, 8, 6, 4, 4)
    c.reserve(4, L.ints([0]))
    c.commit(L.ints([2]), slots=L.ints([0]), path_len=3)
    m = L.model_of(c)
    src, dst = [4, 0, -1, 0, 0, -1], [-1, 4, 2, 2, 5, 3]
    c.fork(L.ints(src), L.ints(dst)), m.fork(src, dst)
    assert c.status() == jd.JD_OK and m.status == O.OK
    assert c.seq_len.cpu().tolist() == [3, 0, 3, 0, 3, 3] and int(c.refs[0]) == 4
    L.same_books(c, m)


FORMS = [(12, 2), (20, 2), (25, 4), (26, 8), (52, 8)]     # nodes x query heads of a kv head: 24, 40, 100, 208, 416 rows


@pytest.mark.parametrize("variant,dtype,D", VARIANTS)
@pytest.mark.parametrize("T,group", [(1, 1)] + FORMS)
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_many_billions(variant, dtype, D, T, group, sign):
    """One key so far above the others (or all but one so far below) that its weight is 1: the output is its value, the logarithm of the
    sum its score, whose size alone must not spoil either."""
    lens = [300, 5, 1000]
    c = L.filled_cache(lens, T, q_heads=2 * group, D=D, dtype=dtype, max_nodes=T, seed=5)
    q = torch.full((3, T, 2 * group, D), 1.171875 * 2.0 ** 15, device="cuda").to(L.DT[dtype])        # whole multiples of a power of two
    best = [77, 0, 640]
    if sign > 0:
        c.k.fill_(1.0)
    else:
        c.k.fill_(-1.328125 * 2.0 ** 20)
    want = torch.empty_like(q)
    for s, token in enumerate(best):
        page, row = int(c.page_table[s, token // 16]), token % 16
        c.k[0, page, :, row] = 1.328125 * 2.0 ** 20 if sign > 0 else -1.0
        for h in range(2):
            want[s, :, h * group:(h + 1) * group] = c.v[0, page, h, row]
    scale = D ** -0.5
    top = D * scale * 1.171875 * 2.0 ** 15 * (1.328125 * 2.0 ** 20 if sign > 0 else -1.0)
    got = c.attend(0, q, variant=variant)
    # D sums, the scale and log2 e, there and back: each off by 2^-24 of the score, which is far from any other
    assert bool(((got["lse"].double() - top).abs() <= (D + 6) * 2.0 ** -24 * abs(top)).all())
    if variant == "simt":
        assert torch.equal(got["out"], want)
    else:      # the weight, 2^(s c2 - base) with base rounded, is near 1; it is rounded to bf16 for the product and not for the sum: 2^-8, and 2^-8 for the output
        assert bool(((got["out"].double() - want.double()).abs() <= (2.0 ** -7 + 2.0 ** -15) * want.double().abs()).all())
    assert c.status() == jd.JD_OK


@pytest.mark.parametrize("variant,dtype,D", VARIANTS)
@pytest.mark.parametrize("T,group", [(1, 1)] + FORMS)
def test_infinite_values_of_context_tokens(variant, dtype, D, T, group):
    """A value of a token that every row sees: an infinity stays that infinity, two of opposite signs and a NaN give NaN, and other
    elements keep their bits - also where the sequence is cut, where an infinity is a node's as well, and in more than one tile."""
    lens = [300, 1, 1000, 140]
    c = L.filled_cache(lens, T, q_heads=2 * group, D=D, dtype=dtype, max_nodes=T, seed=5)
    q = rand((4, T, 2 * group, D), 12, dtype)
    clean = c.attend(0, q, variant=variant)
    want = clean["out"].clone()

    def put(s, token, head, d, x):
        c.v[0, int(c.page_table[s, token // 16]), head, token % 16, d] = x

    inf, nan = float("inf"), float("nan")
    for s, token, head, d, x, y in [(0, 0, 0, 0, inf, inf), (0, 299, 1, 1, -inf, -inf), (2, 77, 0, D - 1, inf, inf), (2, 900, 0, D - 1, inf, inf),
                                    (2, 5, 1, 7, inf, nan), (2, 6, 1, 7, -inf, nan), (3, 139, 0, 9, nan, nan), (3, 10, 0, 9, inf, nan), (1, 0, 1, 3, -inf, -inf),
                                    (0, 300, 0, 0, inf, inf), (3, 50, 1, 2, inf, inf), (3, 51, 1, 2, inf, inf)]:
        put(s, token, head, d, x)
        want[s, :, head * group:(head + 1) * group, d] = y
    got = c.attend(0, q, variant=variant)
    assert bool(((got["out"] == want) | (got["out"].isnan() & want.isnan())).all()) and torch.equal(got["lse"], clean["lse"])
    # scores that are no numbers stay so whatever the values are
    c.k[0, int(c.page_table[3, 0]), 0, 3, 0] = nan
    got = c.attend(0, q, variant=variant)
    assert bool(got["out"][3, :, :group].isnan().all()) and bool(got["lse"][3, :, :group].isnan().all())
    assert c.status() == jd.JD_OK


@pytest.mark.parametrize("variant,dtype,D", VARIANTS)
@pytest.mark.parametrize("T,group", FORMS)
@pytest.mark.parametrize("B", [3, 90])
def test_hidden_and_spoilt_rows_in_every_form(variant, dtype, D, T, group, B):
    """What stands in hidden rows has no effect, and a node that is not finite spoils those that see it alone, for every number of rows
    and with several pieces on a CTA."""
    lens = [(130, 0, 257, 61)[b % 4] + b % 7 for b in range(B)]
    c = L.filled_cache(lens, T, q_heads=2 * group, D=D, dtype=dtype, max_nodes=T, seed=5)
    rng = np.random.default_rng(8)
    parents = [L.random_tree(T, rng, ("star", "chain")[b % 2]) for b in range(B)]
    see = torch.from_numpy(np.stack([O.visible(p)[0] for p in parents])).cuda()
    tree = L.device_tree(parents)
    q = rand((B, T, 2 * group, D), 12, dtype)
    clean = c.attend(0, q, tree, variant=variant)
    table = c.page_table.cpu()
    used = torch.zeros(c.k.shape[1], c.k.shape[3], dtype=torch.bool)
    at = []
    for s, n in enumerate(lens):
        t = torch.arange(n + T)
        used[table[s, t // 16].long(), t % 16] = True
        at.append((int(table[s, (n + 3) // 16]), (n + 3) % 16))
    hidden = (~used).cuda()[None, :, None, :, None].expand(c.k.shape)
    junk = torch.tensor([float("nan"), float("inf"), float("-inf")], device="cuda").to(L.DT[dtype])[torch.arange(int(hidden.sum()), device="cuda") % 3]
    c.k[hidden], c.v[hidden] = junk, junk
    got = c.attend(0, q, tree, variant=variant)
    assert torch.equal(got["out"], clean["out"]) and torch.equal(got["lse"], clean["lse"])
    sees = see[:, :, 3][:, :, None].expand(B, T, 2 * group)
    page, row = (torch.tensor(x, device="cuda") for x in zip(*at))
    c.v[0, page, 0, row, 5], c.v[0, page, 1, row, 6] = float("inf"), float("nan")
    got = c.attend(0, q, tree, variant=variant)
    want = clean["out"].clone()
    want[:, :, :group, 5][sees[:, :, :group]] = float("inf")
    want[:, :, group:, 6][sees[:, :, group:]] = float("nan")
    assert bool(((got["out"] == want) | (got["out"].isnan() & want.isnan())).all()) and torch.equal(got["lse"], clean["lse"])
    c.k[0, page, :, row] = float("nan")
    got = c.attend(0, q, tree, variant=variant)
    assert torch.equal(got["out"][~sees], clean["out"][~sees]) and torch.equal(got["lse"][~sees], clean["lse"][~sees])
    assert bool(got["out"][sees].isnan().all()) and bool(got["lse"][sees].isnan().all())
    assert c.status() == jd.JD_OK


def attend64(c, q, see, scale):
    """Softmax attention of blocks q [B, T, heads, D] in float64 on the device, over all pages of every sequence at once, and the bound that
    attend_tolerance of the library's tests derives, with each row's own |q|: (out, lse, bound of out, bound of lse)."""
    B, T, Hq, D = q.shape
    H = c.kv_heads
    outs = []
    for b in range(B):
        n = int(c.seq_len[b])
        at = torch.arange(n + T, device="cuda")
        page, row = c.page_table[b].long()[at // c.k.shape[3]], at % c.k.shape[3]
        k, v = (x[0, page, :, row].double().transpose(0, 1) for x in (c.k, c.v))                       # [H, n + T, D]
        qb = q[b].double().view(T, H, Hq // H, D).permute(1, 2, 0, 3)                                  # [H, G, T, D]
        s = scale * (qb @ k[:, None].transpose(2, 3))
        s[..., n:].masked_fill_(~see[b], float("-inf"))
        lse = s.logsumexp(-1)
        p = (s - lse[..., None]).exp()
        A = scale * qb.norm(dim=-1) * k.norm(dim=-1).max()
        w = 2 * (D + 4) * 2.0 ** -24 * A + 2.0 ** -20 + (n + T) * 2.0 ** -24
        out = p @ v[:, None]
        extra, step = (2.0 ** -8, 2.0 ** -8) if q.dtype == torch.bfloat16 else (0.0, 2.0 ** -24)
        tol = (p @ v.abs()[:, None]) * (w + extra)[..., None] + out.abs() * step + 1e-30
        back = lambda x: x.movedim(2, 0).flatten(1, 2)                                                 # noqa: E731
        outs.append((back(out), back(lse), back(tol), back(w + 2.0 ** -22 * lse.abs())))
    return [torch.stack(x) for x in zip(*outs)]


@pytest.mark.parametrize("variant,dtype,D", VARIANTS)
@pytest.mark.parametrize("T,group", FORMS)
@pytest.mark.parametrize("falling", [False, True])
def test_scores_that_grow_from_tile_to_tile(variant, dtype, D, T, group, falling):
    """Every tile's scores lie some 6 above the last one's (or below, or jump), so that sums and numerators found so far are weighed again and again
    by factors that count, in rows that differ in how fast: out and lse within the bound."""
    lens = [1500, 700, 1024, 90] * 10                         # 80 segments: pieces of many tiles
    B = len(lens)
    c = L.filled_cache(lens, T, q_heads=2 * group, D=D, dtype=dtype, max_nodes=T, seed=5)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    u = torch.randn(D, generator=gen, device="cuda")
    u /= u.norm()
    q = torch.randn(B, T, 2 * group, D, generator=gen, device="cuda")
    q += u * (torch.randint(0, 4, (B, T, 2 * group, 1), generator=gen, device="cuda") - 1) * D ** 0.5   # rows along u, against it and across
    q = q.to(L.DT[dtype])
    for b, n in enumerate(lens):
        at = torch.arange(n + T, device="cuda")
        page, row = c.page_table[b].long()[at // 16], at % 16
        height = at.float() * (0.05 if b % 3 else 0.02)
        if falling:
            height = height.flip(0)
        if b % 4 == 2:
            height = (at // 128 % 3).float() * 15
        c.k[0, page, :, row] = (torch.randn(n + T, 2, D, generator=gen, device="cuda") + height[:, None, None] * u).to(L.DT[dtype])
    rng = np.random.default_rng(2)
    parents = [L.random_tree(T, rng) for _ in lens]
    see = torch.from_numpy(np.stack([O.visible(p)[0] for p in parents])).cuda()
    out, lse, tol, ltol = attend64(c, q, see, D ** -0.5)
    got = c.attend(0, q, L.device_tree(parents), variant=variant)
    assert c.status() == jd.JD_OK
    assert float(lse.max()) > 20 and float((tol / out.abs().clamp_min(0.1)).median()) < 0.05           # the bound says something
    err = (got["out"].double() - out).abs()
    assert bool((err <= tol).all()), float((err - tol).max())
    assert bool(((got["lse"].double() - lse).abs() <= ltol).all())


@pytest.mark.parametrize("D", [8, 40, 72, 80, 96, 112, 136, 192, 256])
@pytest.mark.parametrize("T,q_heads,kv_heads", [(1, 2, 2), (2, 4, 2), (6, 6, 2), (11, 8, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_head_widths(D, T, q_heads, kv_heads, dtype):
    """Widths on both sides of 128 and types, four rows and sixteen, whole segments and split ones; the tensor-core kernel is
    refused where it has no form."""
    lens = [0, 65, 3, 900]
    c = L.filled_cache(lens, T, q_heads=q_heads, kv_heads=kv_heads, D=D, dtype=dtype, max_nodes=T, seed=D)
    rng = np.random.default_rng(D)
    parents = [L.random_tree(T, rng) for _ in lens]
    check_attend(*run_attend(c, L.model_of(c), T, parents, dtype, "auto", D))
    with pytest.raises(jd.JdError) as e:
        c.attend(0, rand((4, T, q_heads, D), 1, dtype), variant="tensor")
    assert e.value.status == jd.JD_ERR_UNSUPPORTED


@pytest.mark.parametrize("variant,dtype,D", VARIANTS + [("simt", "bf16", 192)])
@pytest.mark.parametrize("B", [257, 385, 1024])
def test_attend_many_sequences(variant, dtype, D, B):
    """More sequences than a block has threads, padding and empty ones among them."""
    T, seqs = 2, 60
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, 150, seqs)]
    c = L.filled_cache(lens, T, q_heads=2, kv_heads=1, D=D, dtype=dtype, max_nodes=T, seed=2)
    slots = rng.integers(-1, seqs, B)
    nodes = rng.integers(0, T + 1, B)
    check_attend(*run_attend(c, L.model_of(c), T, [-1, 0], dtype, variant, 3, slots=L.ints(slots), num_nodes=L.ints(nodes), B=B))


@pytest.mark.parametrize("variant,dtype,D", VARIANTS)
def test_a_prompt_in_blocks(variant, dtype, D):
    """Prompts of different lengths go in as chains of up to 128 tokens that are kept whole; every row attends to what stands in
    front of it, as one pass over the prompts has it."""
    T, Hq, H, lens = 128, 4, 2, [300, 128, 1, 257]
    B, n = len(lens), max(lens)
    c = L.empty_cache(1, 80, 16, Hq, H, D, B, 24, T, dtype)
    k, v, q = (rand((B, n, h, D), i, dtype) for i, h in enumerate((H, H, Hq)))
    out = torch.zeros(B, n, Hq, D, dtype=q.dtype, device="cuda")
    for at in range(0, n, T):
        m = min(T, n - at)
        left = [min(max(x - at, 0), m) for x in lens]
        slots = L.ints([b if left[b] else -1 for b in range(B)])
        c.reserve(m, slots)
        tree = jd.Tree(m, num_nodes=L.ints(left))
        part = [x[:, at:at + m].contiguous() for x in (k, v, q)]
        c.append(0, part[0], part[1], tree, slots=slots)
        out[:, at:at + m] = c.attend(0, part[2], tree, slots=slots, variant=variant)["out"]
        c.commit(L.ints([max(x - 1, 0) for x in left]), slots=slots, path_len=m - 1)
    assert c.status() == jd.JD_OK and c.seq_len.cpu().tolist() == lens
    for b, x in enumerate(lens):
        kk, vv = (t[b, :x].double().transpose(0, 1).repeat_interleave(Hq // H, 0) for t in (k, v))
        s = D ** -0.5 * (q[b, :x].double().transpose(0, 1) @ kk.transpose(1, 2))
        s.masked_fill_(torch.ones(x, x, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
        p = s.softmax(-1)
        want, spread = p @ vv, p @ vv.abs()
        A = D ** -0.5 * q[b, :x].double().norm(dim=-1).max() * kk.norm(dim=-1).max()
        w = 2 * (D + 4) * 2.0 ** -24 * A + 2.0 ** -20 + x * 2.0 ** -24
        extra, step = (2.0 ** -8, 2.0 ** -8) if dtype == "bf16" else (0.0, 2.0 ** -24)
        assert bool(((out[b, :x].double().transpose(0, 1) - want).abs() <= spread * (w + extra) + want.abs() * step + 1e-30).all())


@pytest.mark.parametrize("variant,dtype,D", VARIANTS)
@pytest.mark.parametrize("T,group", [(128, 160), (127, 400)])
def test_attend_more_row_blocks_than_multiprocessors(variant, dtype, D, T, group):
    """So many query heads of a kv head that one block a row block is all that the grid has."""
    lens = [70, 0, 300]
    c = L.filled_cache(lens, T, q_heads=group, kv_heads=1, D=D, dtype=dtype, max_nodes=T, seed=5)
    q = rand((3, T, group, D), 4, dtype)
    parents = [L.random_tree(T, np.random.default_rng(s)) for s in range(3)]
    see = torch.from_numpy(np.stack([O.visible(p)[0] for p in parents])).cuda()
    got = c.attend(0, q, L.device_tree(parents), variant=variant)
    assert c.status() == jd.JD_OK
    out, lse, tol, ltol = attend64(c, q, see, D ** -0.5)
    assert bool(((got["out"].double() - out).abs() <= tol).all()) and bool(((got["lse"].double() - lse).abs() <= ltol).all())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,group", [(1, 4), (20, 2)])
def test_infinite_values_in_every_column_of_long_pieces(D, T, group):
    """150 segments of 100,000 tokens, about one to a CTA: finding the infinities takes no time that a wait inside the kernel
    would run out in, and a NaN behind them is found as well."""
    n, B, page = 100000, 75, 64
    per = -(-(n + T) // page)
    c = L.empty_cache(1, per, page, 2 * group, 2, D, B, per, T, fill=3)
    c.page_table.copy_(torch.arange(per, dtype=torch.int32, device="cuda").expand(B, per))       # all sequences read the same pages
    c.refs.fill_(B)
    c.free_bits.zero_()
    c.seq_len.fill_(n)
    c.held.fill_(per)
    c.v[0, 5 // page, :, 5] = float("inf")
    c.v[0, 6 // page, :, 6, 3] = float("-inf")
    c.v[0, (n - 1) // page, :, (n - 1) % page, 7] = float("nan")
    q = rand((B, T, 2 * group, D), 4)
    got = c.attend(0, q, variant="tensor")
    assert c.status() == jd.JD_OK
    want = torch.full_like(q, float("inf"))
    want[..., [3, 7]] = float("nan")
    assert bool(((got["out"] == want) | (got["out"].isnan() & want.isnan())).all()) and bool(got["lse"].isfinite().all())
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    c.attend(0, q, variant="tensor")
    end.record()
    assert c.status() == jd.JD_OK
    assert start.elapsed_time(end) < 100                # ms; 2 without infinities. The waits' limit is some 1,800
