"""Norms of query and key heads with their rotation, forward, backward and into the cache, against the CPU model in float64."""
import numpy as np
import pytest
import torch

import cache_testlib as L
from oracle import step_oracle as S
from paper_2501_19309_b200 import jd

pytestmark = pytest.mark.gpu
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}     # half a step of a value, relative


def rand(shape, seed, dtype="f32", scale=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(L.DT[dtype])


def setup(n, heads, D, rot, layout, of, dtype, seed=0):
    q, k = rand((n, heads[0], D), seed, dtype), rand((n, heads[1], D), seed + 1, dtype)
    host = torch.Generator().manual_seed(seed)
    pos = torch.randint(-3, 1 << 20, (n,) if of is None else (n, max(of) + 1), generator=host).to(torch.int32)
    if n > 2:
        pos[0], pos[1] = 2 ** 31 - 1, -2 ** 31
    freq, amp = jd.rope_frequencies(rot, 10000.0, "yarn", 4.0, 2048.0, 1.0, 32.0)
    r = jd.Rotary(freq.cuda(), layout, amp, axes=of)
    return q, k, pos, r, S.angles(pos.numpy(), freq.numpy(), of), amp


def error_of(D):
    """Relative error of n w in float32: D squares summed in any order count half in the root, which is off by 2^-22, and two products more; and of a
    turned pair: two products with a cosine off by 2^-22 (half turns rounded to float32: pi 2^-25; sincospi 2 ulp)."""
    return (D / 2 + 4) * 2.0 ** -24 + 2.0 ** -22, 2.0 ** -20


def forward_bound(x, w, eps, amp, dtype, want):
    big = np.abs(S.normed(x, w, eps)[0]).max() * amp * np.sqrt(2)
    return big * sum(error_of(x.shape[-1])) + np.abs(want) * STEP[dtype]


def grad_bounds(g, x, w, eps, amp, dtype, dx):
    """dx = r (g w - n mean(g w n)): |mean| <= max|g w|, as mean n^2 <= 1. dw: every term g n by its own size, the sum by the number of additions that a term
    goes through: a lane's items, 256 lanes' groups, 592 blocks."""
    D = x.shape[-1]
    e = 4 * sum(error_of(D)) + (D + 8) * 2.0 ** -24
    _, n, r = S.normed(x, w, eps)
    G, W, N = np.abs(g).max() * amp * np.sqrt(2), np.abs(w).max(), np.abs(n).max()
    terms = amp * np.sqrt(2) * np.abs(g).max() * np.abs(n).reshape(-1, D).sum(0)
    return r.max() * G * W * (1 + N) * e + np.abs(dx) * STEP[dtype], terms * (e + (g.size / D / 8 + 256 + 592) * 2.0 ** -24)


HEADS = [  # tokens, (query, key heads), head_dim, rot_dim, layout, axes, dtype
    (1, (1, 1), 64, 64, "half", 1, "bf16"), (26, (32, 8), 128, 128, "half", 3, "bf16"), (7, (3, 1), 128, 64, "half", 1, "f32"),
    (300, (5, 2), 80, 48, "interleaved", 2, "bf16"), (33, (2, 2), 256, 256, "interleaved", 3, "f32"), (5, (4, 1), 20, 6, "half", 1, "bf16"),
    (9, (1, 3), 7, 2, "interleaved", 1, "f32"), (1025, (9, 3), 96, 96, "half", 4, "f32"), (4, (80, 16), 128, 32, "interleaved", 1, "bf16"),
    (70, (300, 1), 8, 8, "half", 2, "f32"), (2, (1, 1), 256, 16, "half", 1, "bf16"), (600, (7, 5), 255, 254, "interleaved", 3, "f32"), (11, (2, 1), 16, 16, "half", 1, "bf16")]


def axis_list(n, rot):
    return None if n == 1 else [i * n // (rot // 2) if rot // 2 >= n else 0 for i in range(rot // 2)]


@pytest.mark.parametrize("n,heads,D,rot,layout,num_axes,dtype", HEADS)
def test_rotate_qk(n, heads, D, rot, layout, num_axes, dtype):
    of = axis_list(num_axes, rot)
    q, k, pos, r, angle, amp = setup(n, heads, D, rot, layout, of, dtype)
    w = [1 + 0.3 * rand((D,), 7), None]
    q[0, 0] = 0                                                            # a head of zeroes: eps alone
    norm = jd.HeadNorm(w[0], w[1], eps=1e-5)
    got = r.rotate_qk(q, k, pos.cuda(), norm=norm)
    for x, y, wt in zip((q, k), got, w):
        wt = np.ones(D) if wt is None else L.f64(wt)
        want = S.heads(L.f64(x), wt, 1e-5, angle, layout, amp)
        assert (np.abs(L.f64(y) - want) <= forward_bound(L.f64(x), wt, 1e-5, amp, dtype, want)).all()
    again = r.rotate_qk(q.clone(), None, pos.cuda(), norm=norm)
    assert again[1] is None and torch.equal(again[0], got[0])
    a, b = q.clone(), k.clone()
    assert r.rotate_qk(a, b, pos.cuda(), norm=norm, q_out=a, k_out=b) == (a, b) and torch.equal(a, got[0]) and torch.equal(b, got[1])   # in place
    # without a norm: what rotate() does to each
    for x, y in zip((q, k), r.rotate_qk(q, k, pos.cuda())):
        one = r.rotate(x, pos.cuda())
        # which product of a pair is rounded before the sum is the compiler's choice in either kernel: half a step of a product each, and the results' own
        assert float((one.float() - y.float()).abs().max()) <= (4 * 2.0 ** -24 + 2 * STEP[dtype]) * float(x.abs().max()) * amp * np.sqrt(2)
        assert torch.equal(y[..., rot:], x[..., rot:])
        back = r.rotate(one, pos.cuda(), inverse=True)
        big, whole = float(x.abs().max()) * amp ** 2, x.float()
        whole[..., :rot] *= amp ** 2                                       # what does not turn has no amplitude either
        assert float((back.float() - whole).abs().max()) <= 4 * big * (2.0 ** -20 + STEP[dtype]) * np.sqrt(2)


@pytest.mark.parametrize("n,heads,D,rot,layout,num_axes,dtype", HEADS + [(20000, (2, 1), 64, 64, "half", 3, "bf16")])
def test_rotate_qk_grad(n, heads, D, rot, layout, num_axes, dtype):
    of = axis_list(num_axes, rot)
    q, k, pos, r, angle, amp = setup(n, heads, D, rot, layout, of, dtype, seed=3)
    gq, gk = rand(q.shape, 11, dtype), rand(k.shape, 12, dtype)
    w = [1 + 0.3 * rand((D,), 7), 1 + 0.3 * rand((D,), 8)]
    q[0, 0] = 0
    norm = jd.HeadNorm(*w, eps=1e-2)
    got = r.rotate_qk_grad(gq, gk, q, k, pos.cuda(), norm)
    for name, g, x, wt in (("q", gq, q, w[0]), ("k", gk, k, w[1])):
        g, x, wt = L.f64(g), L.f64(x), L.f64(wt)
        dx, dw = S.heads_grad(g, x, wt, 1e-2, angle, layout, amp)
        bx, bw = grad_bounds(g, x, wt, 1e-2, amp, dtype, dx)
        assert (np.abs(L.f64(got[name]) - dx) <= bx).all()
        assert (np.abs(L.f64(got[name + "_weight"]) - dw) <= bw).all()
    again = r.rotate_qk_grad(gq, gk, q, k, pos.cuda(), norm)
    assert all(torch.equal(again[x], got[x]) for x in got)                 # bit for bit
    lean = r.rotate_qk_grad(gq, None, q, None, pos.cuda(), norm, weights=False)
    assert set(lean) == {"q", "k"} and lean["k"] is None and torch.equal(lean["q"], got["q"])
    over = dict(q=gq.clone(), k=k.clone())                                 # over its own inputs
    over = r.rotate_qk_grad(over["q"], gk, q, over["k"], pos.cuda(), norm, out=over)
    assert torch.equal(over["q"], got["q"]) and torch.equal(over["k"], got["k"]) and torch.equal(over["k_weight"], got["k_weight"])


def test_strided_rows_leave_the_rest_alone():
    """Queries and keys as they lie in one projection's rows; the second time off 16 bytes, so element by element."""
    n, D = 19, 64
    freq, _ = jd.rope_frequencies(64)
    norm, pos = jd.HeadNorm(1 + 0.3 * rand((D,), 5)), L.ints(np.arange(n) * 1000)
    r = jd.Rotary(freq.cuda())
    for off in (0, 1):
        buf = torch.full((n, 900), 7.0, dtype=torch.bfloat16, device="cuda")
        q, k = buf.as_strided((n, 4, D), (900, D, 1), off), buf.as_strided((n, 2, D), (900, D, 1), off + 4 * D)
        q.copy_(rand(q.shape, 1)), k.copy_(rand(k.shape, 2))
        want = r.rotate_qk(q.clone(memory_format=torch.contiguous_format), k.clone(memory_format=torch.contiguous_format), pos, norm=norm)
        gq, gk = rand(q.shape, 3, "bf16"), rand(k.shape, 4, "bf16")
        grads = [r.rotate_qk_grad(gq, gk, x, y, pos, norm) for x, y in ((q, k), (q.clone(memory_format=torch.contiguous_format), k.clone(memory_format=torch.contiguous_format)))]
        for x in grads[0]:       # the other form adds in another order
            assert torch.allclose(grads[0][x].float(), grads[1][x].float(), rtol=2.0 ** -7, atol=1e-4)
        r.rotate_qk(q, k, pos, norm=norm, q_out=q, k_out=k)
        for x, y in zip((q, k), want):
            assert torch.allclose(x.float(), y.float(), rtol=2.0 ** -7, atol=1e-6)
        left = torch.ones(n, 900, dtype=torch.bool, device="cuda")
        left[:, off:off + 6 * D] = False
        assert (buf[left] == 7).all()


def test_no_tokens_no_keys_and_sums_of_nothing():
    freq, _ = jd.rope_frequencies(8)
    r, norm = jd.Rotary(freq.cuda()), jd.HeadNorm()
    q, k, pos = (torch.zeros(s, device="cuda", dtype=t) for s, t in (((0, 2, 8), torch.float32), ((0, 1, 8), torch.float32), ((0,), torch.int32)))
    a, b = r.rotate_qk(q, k, pos, norm=norm)
    assert a.shape == q.shape and b.shape == k.shape
    got = r.rotate_qk_grad(q, k, q, k, pos, norm)
    assert not got["q_weight"].any() and not got["k_weight"].any()
    got = r.rotate_qk_grad(rand((3, 2, 8), 0), None, rand((3, 2, 8), 1), None, torch.zeros(3, dtype=torch.int32, device="cuda"), norm)
    assert got["q_weight"].any() and not got["k_weight"].any()


def test_values_that_are_not_finite_stay_in_their_head():
    freq, _ = jd.rope_frequencies(128)
    r, norm, pos = jd.Rotary(freq.cuda()), jd.HeadNorm(), L.ints(np.arange(4))
    q = rand((4, 3, 128), 0, "bf16")
    want = r.rotate_qk(q, None, pos, norm=norm)[0]
    bad = q.clone()
    bad[1, 1, 5], bad[2, 0, 100], bad[3, 2, 0] = float("nan"), float("inf"), 3e38
    got = r.rotate_qk(bad, None, pos, norm=norm)[0]
    hit = torch.zeros(4, 3, dtype=torch.bool, device="cuda")
    hit[1, 1] = hit[2, 0] = hit[3, 2] = True
    assert torch.equal(got[~hit], want[~hit]) and not torch.isfinite(got[1, 1]).any()


def test_two_streams_and_a_captured_step():
    """Forward and backward have no state of their own: two streams at once, and a captured pair replayed on new values."""
    freq, _ = jd.rope_frequencies(128)
    r, norm, n = jd.Rotary(freq.cuda(), axes=[0] * 20 + [1] * 44), jd.HeadNorm(rand((128,), 1)), 3000
    q, k, g, h = (rand((n, m, 128), i, "bf16") for i, m in enumerate((8, 2, 8, 2)))
    pos = torch.randint(0, 5000, (n, 2), device="cuda", dtype=torch.int32)
    want, wgrad = r.rotate_qk(q, k, pos, norm=norm), r.rotate_qk_grad(g, h, q, k, pos, norm)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(10):
        for s in streams:
            with torch.cuda.stream(s):
                got.append((r.rotate_qk(q, k, pos, norm=norm), r.rotate_qk_grad(g, h, q, k, pos, norm)))
    torch.cuda.synchronize()
    for out, grad in got:
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]) and all(torch.equal(grad[x], wgrad[x]) for x in wgrad)
    static = q.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, grad = r.rotate_qk(static, k, pos, norm=norm), r.rotate_qk_grad(g, h, static, k, pos, norm)
    static.copy_(rand(q.shape, 99, "bf16"))
    graph.replay()
    torch.cuda.synchronize()
    again = r.rotate_qk_grad(g, h, static, k, pos, norm)
    assert torch.equal(out[0], r.rotate_qk(static, k, pos, norm=norm)[0]) and all(torch.equal(grad[x], again[x]) for x in again)


def test_refusals():
    freq, _ = jd.rope_frequencies(8)
    r, r2 = jd.Rotary(freq.cuda()), jd.Rotary(freq.cuda(), axes=[0, 1, 0, 1])
    q, k, pos = torch.ones(3, 2, 8, device="cuda"), torch.ones(3, 1, 8, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    norm = jd.HeadNorm(torch.ones(8, device="cuda"))
    for bad in (lambda: r.rotate_qk(q[0], k, pos), lambda: r.rotate_qk(q.half(), k, pos), lambda: r.rotate_qk(q, k.bfloat16(), pos), lambda: r.rotate_qk(q, k[:2], pos),
                lambda: r.rotate_qk(q, k[..., :4], pos), lambda: r.rotate_qk(q, k, pos.long()), lambda: r.rotate_qk(q, k, pos[:2]), lambda: r2.rotate_qk(q, k, pos),
                lambda: r.rotate_qk(q, k, pos[:, None].expand(3, 2).contiguous()), lambda: r2.rotate(q, pos), lambda: r.rotate_qk(q, k, pos, q_out=k),
                lambda: r.rotate_qk(q, k, pos, norm=jd.HeadNorm(torch.ones(7, device="cuda"))), lambda: r.rotate_qk(q.transpose(0, 1), None, pos[:2]),
                lambda: r.rotate_qk(q[:1].expand(3, 2, 8), None, pos), lambda: r.rotate_qk(q.clone().requires_grad_(), k, pos),
                lambda: r.rotate_qk_grad(q, None, q, k, pos, norm), lambda: r.rotate_qk_grad(q, k, q, k, pos, norm, workspace=torch.empty(4, dtype=torch.uint8, device="cuda")),
                lambda: r.rotate_qk_grad(q, k, q, k, pos, norm, out=dict(q_weight=torch.ones(4, device="cuda"))), lambda: r.rotate_qk_grad(k, k, q, k, pos, norm),
                lambda: jd.HeadNorm(torch.ones(8, device="cuda", requires_grad=True)), lambda: jd.HeadNorm(torch.ones(8, device="cuda").bfloat16()),
                lambda: jd.HeadNorm(torch.ones(8, device="cuda"), torch.ones(4, device="cuda"))):
        with pytest.raises(ValueError):
            bad()


# ------------------------------------------------------------------------------------------- into the cache
@pytest.mark.parametrize("dtype,D,rot,layout,num_axes,given", [("bf16", 128, 128, "half", 1, False), ("bf16", 64, 64, "interleaved", 3, True), ("f32", 80, 40, "half", 2, True),
                                                               ("bf16", 128, 64, "half", 2, False), ("f32", 24, 12, "interleaved", 1, True), ("bf16", 256, 0, "half", 1, False)])
def test_append_with_norms(dtype, D, rot, layout, num_axes, given):
    lens, T, Hq, Hk = [0, 5, 33, 120], 6, 8, 2
    c = L.filled_cache(lens, T, page=16, q_heads=Hq, kv_heads=Hk, D=D, layers=2, max_nodes=8, dtype=dtype)
    parents = [-1, 0, 0, 1, 3, 2]
    num = L.ints([6, 0, 3, 6])
    tree = L.device_tree(parents, num_nodes=num)
    depth = np.array([0, 1, 1, 2, 3, 2])
    qkv = rand((4, T, Hq + 2 * Hk, D), 3, dtype)
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hk], qkv[:, :, Hq + Hk:]
    of = axis_list(num_axes, rot) if rot else None
    r, w = None, [1 + 0.3 * rand((D,), 1), 1 + 0.3 * rand((D,), 2)]
    pos = np.asarray(lens)[:, None] + depth[None]
    where = None
    if rot:
        freq, _ = jd.rope_frequencies(rot)
        r = jd.Rotary(freq.cuda(), layout, axes=of)
        if given:
            pos = np.random.default_rng(0).integers(0, 10000, size=(4, T) if of is None else (4, T, num_axes))
            where = L.ints(pos)
        angle = S.angles(pos, freq.numpy(), None if of is None or not given else of)
    else:
        angle = np.zeros((4, T, 0))
    before_k, before_v = c.k.clone(), c.v.clone()
    q_out = torch.full((4, T, Hq, D), 7.0, dtype=L.DT[dtype], device="cuda")
    norm = jd.HeadNorm(*w, eps=1e-5)
    assert c.append(1, k, v, tree, rotary=r, q=q, q_out=q_out, norm=norm, positions=where) is q_out
    assert c.status() == jd.JD_OK
    want_q, want_k = (S.heads(L.f64(x), L.f64(wt), 1e-5, angle, layout) for x, wt in ((q, w[0]), (k, w[1])))
    bq, bk = (forward_bound(L.f64(x), L.f64(wt), 1e-5, 1.0, dtype, want) for x, wt, want in ((q, w[0], want_q), (k, w[1], want_k)))
    for b, n in enumerate(num.tolist()):
        assert (np.abs(L.f64(q_out[b, :n]) - want_q[b, :n]) <= bq[b, :n]).all() and (q_out[b, n:] == 7).all()
        for t in range(n):
            page, row = int(c.page_table[b, (lens[b] + t) // 16]), (lens[b] + t) % 16
            assert (np.abs(L.f64(c.k[1, page, :, row]) - want_k[b, t]) <= bk[b, t]).all()
            assert torch.equal(c.v[1, page, :, row], v[b, t])
            before_k[1, page, :, row], before_v[1, page, :, row] = c.k[1, page, :, row], c.v[1, page, :, row]
    assert torch.equal(before_k, c.k) and torch.equal(before_v, c.v)


def test_append_with_axes_and_no_norm_is_append():
    c = L.filled_cache([3, 40], 4, D=64, dtype="bf16", max_nodes=4)
    freq, _ = jd.rope_frequencies(64)
    q, k, v = (rand((2, 4, h, 64), i, "bf16") for i, h in enumerate((4, 2, 2)))
    out = c.append(0, k, v, rotary=jd.Rotary(freq.cuda()), q=q)
    kept = c.k.clone()
    for pos in (None, L.ints([[[n + t] * 2 for t in range(4)] for n in (3, 40)])):
        c.k.zero_()
        again = c.append(0, k, v, rotary=jd.Rotary(freq.cuda(), axes=[0, 1] * 16), q=q, positions=pos)
        # either kernel rounds a pair's first product where its compiler chose, and the result once: a step apart at most
        assert (again.float() - out.float()).abs().max() <= 2 * (2.0 ** -8 + 2.0 ** -23) * q.float().abs().max() * 2 ** 0.5
        new = c.k != 0
        assert new.any() and (c.k.float() - kept.float())[new].abs().max() <= 2 * (2.0 ** -8 + 2.0 ** -23) * k.float().abs().max() * 2 ** 0.5


def test_append_with_norms_refusals_and_bad_pages():
    c = L.filled_cache([3, 40], 4, D=64, dtype="bf16", max_nodes=4)
    freq, _ = jd.rope_frequencies(64)
    r, norm = jd.Rotary(freq.cuda(), axes=[0, 1] * 16), jd.HeadNorm(torch.ones(64, device="cuda"))
    k = rand((2, 4, 2, 64), 0, "bf16")
    pos = torch.zeros(2, 4, 2, dtype=torch.int32, device="cuda")
    for bad in (lambda: c.append(0, k, k, rotary=r, positions=pos[..., 0].contiguous()), lambda: c.append(0, k, k, rotary=r, positions=pos.long()),
                lambda: c.append(0, k, k, positions=pos), lambda: c.append(0, k, k, norm=jd.HeadNorm(torch.ones(63, device="cuda"))),
                lambda: c.append(0, k, k, rotary=r, positions=pos[:1])):
        with pytest.raises(ValueError):
            bad()
    before = c.k.clone()
    c.page_table[1, 2] = -1                                                # tokens 32..47: sequence 1 has no page for its block
    q = rand((2, 4, 4, 64), 1, "bf16")
    out = c.append(0, k, k, rotary=r, q=q, norm=norm, positions=pos)
    assert c.status() == jd.JD_ERR_BAD_INDEX and torch.isfinite(out).all()
    assert (c.k != before).any(-1).sum() <= 4 * 2                          # sequence 0's rows alone
    c.append(0, k, k, norm=norm, slots=L.ints([0, 0]))
    assert c.status() == jd.JD_ERR_BAD_INDEX                               # a slot named twice


@pytest.mark.parametrize("n,heads,D,rot,layout,dtype", [
    (3, (1, 1), 128, 128, "half", "bf16"), (3, (1, 3), 128, 64, "interleaved", "f32"), (5, (3, 1), 64, 64, "half", "f32"), (1, (2, 1), 64, 64, "interleaved", "bf16"),
    (1, (1, 1), 16, 16, "half", "bf16"), (33, (5, 3), 80, 48, "interleaved", "bf16"), (7, (1, 2), 20, 6, "half", "f32")])
def test_gradients_without_eps(n, heads, D, rot, layout, dtype):
    """eps = 0 and no head of zeroes: groups of lanes that have no head in a block's last step stay out of the weights' sums."""
    q, k, pos, r, angle, amp = setup(n, heads, D, rot, layout, None, dtype, seed=5)
    gq, gk = rand(q.shape, 11, dtype), rand(k.shape, 12, dtype)
    w = [1 + 0.3 * rand((D,), 7), 1 + 0.3 * rand((D,), 8)]
    got = r.rotate_qk_grad(gq, gk, q, k, pos.cuda(), jd.HeadNorm(*w, eps=0.0))
    for name, g, x, wt in (("q", gq, q, w[0]), ("k", gk, k, w[1])):
        g, x, wt = L.f64(g), L.f64(x), L.f64(wt)
        dx, dw = S.heads_grad(g, x, wt, 0.0, angle, layout, amp)
        bx, bw = grad_bounds(g, x, wt, 0.0, amp, dtype, dx)
        assert (np.abs(L.f64(got[name]) - dx) <= bx).all()
        assert (np.abs(L.f64(got[name + "_weight"]) - dw) <= bw).all()


def test_weight_gradients_hold_no_workspace():
    """What a program keeps of a call is its gradients, not the room for their partial sums."""
    q, k, pos, r, _, _ = setup(9, (2, 1), 128, 128, "half", None, "f32")
    got = r.rotate_qk_grad(q, k, q, k, pos.cuda(), jd.HeadNorm())
    assert all(got[name].untyped_storage().nbytes() <= 2 * 128 * 4 for name in ("q_weight", "k_weight"))


def test_a_workspace_of_the_call_on_another_stream():
    """Outputs are given, the workspace is not: what is allocated behind the call must not be memory that its kernels have yet to use."""
    n, D = 512, 128
    q, k, pos, r, _, _ = setup(n, (8, 2), D, D, "half", None, "bf16", seed=9)
    gq, gk, norm, pos = rand(q.shape, 11, "bf16"), rand(k.shape, 12, "bf16"), jd.HeadNorm(1 + 0.3 * rand((D,), 7), 1 + 0.3 * rand((D,), 8)), pos.cuda()
    want = r.rotate_qk_grad(gq, gk, q, k, pos, norm)
    out = {name: torch.empty_like(x) for name, x in want.items()}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)                                      # some 30 ms: the call's kernels run behind what follows
    assert r.rotate_qk_grad(gq, gk, q, k, pos, norm, out=out, stream=side) == out
    later = [torch.full((jd.load().jd_head_rope_grad_workspace_bytes(D),), 77, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert all(bool((x == 77).all()) for x in later)
    assert all(torch.equal(out[name], want[name]) for name in want)
