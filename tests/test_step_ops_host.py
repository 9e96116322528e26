"""Head norms, shared prefixes and verification from probabilities: struct layouts, refusals that need no device, and the CPU model's pins."""
import ctypes as C
import itertools
import os
import re
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import step_oracle as S
from paper_2501_19309_b200 import jd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ["jd_rope_axes_t", "jd_head_norm_t", "jd_head_rope_args_t", "jd_head_rope_grad_args_t", "jd_append_heads_t", "jd_shared_t", "jd_verify_probs_args_t"]


@pytest.mark.parametrize("name", NAMES)
def test_struct_layouts_follow_the_header(name):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "jd.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^{}]*)\} %s;" % name, src).group(1)
    fields = [m.group(1) for decl in body.split(";") for part in decl.split(",") for m in [re.search(r"([A-Za-z_0-9]+)\s*$", part.strip())] if m]
    assert fields == [f[0] for f in getattr(jd, name)._fields_]


def test_struct_sizes_and_packed_layouts(tmp_path):
    import shutil
    import subprocess
    from paper_2501_19309_b200 import cache, probs
    for packer, name in ((cache._HEAD_ROPE_ARGS, "jd_head_rope_args_t"), (cache._HEAD_ROPE_GRAD_ARGS, "jd_head_rope_grad_args_t"),
                         (cache._APPEND_HEADS_ARGS, "jd_append_heads_t"), (probs._ARGS, "jd_verify_probs_args_t")):
        assert packer.size <= C.sizeof(getattr(jd, name)) < packer.size + 8, name
    if shutil.which("gcc") is None:
        pytest.skip("gcc is not installed")
    src = '#include <stdio.h>\n#include "jd.h"\nint main(void) {\n%s  return 0;\n}\n' % "".join('  printf("%%d\\n", (int)sizeof(%s));\n' % n for n in NAMES)
    (tmp_path / "s.c").write_text(src)
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")], check=True)
    got = subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in got] == [C.sizeof(getattr(jd, n)) for n in NAMES]


# pointers of these calls are never followed: every call is refused before it launches anything
def _norm(**kw):
    return jd.jd_head_norm_t(kw.pop("q_weight", 0), kw.pop("k_weight", 0), kw.pop("eps", 1e-6))


def head_args(grad=False, **kw):
    a = (jd.jd_head_rope_grad_args_t if grad else jd.jd_head_rope_args_t)()
    a.tokens, a.q_heads, a.k_heads, a.head_dim, a.dtype, a.positions = 3, 2, 1, 64, jd.JD_DTYPE_BF16, 256
    a.rope = jd.jd_rope_t(256, 64, jd.JD_ROPE_HALF, 1.0)
    for n, t in type(a)._fields_:
        if t is C.c_void_p and n not in ("positions", "norm", "axes", "workspace", "q_weight_grad", "k_weight_grad"):
            setattr(a, n, 4096 if n.startswith("q") else 8192)
    keep = []
    if grad:
        keep.append(_norm())
        a.norm = C.addressof(keep[-1])
    for k, v in kw.items():
        if isinstance(v, C.Structure) and k != "rope":
            keep.append(v)
            v = C.addressof(v)
        setattr(a, k, v)
    a._keep = keep
    return a


def axes(n, of):
    buf = (C.c_uint8 * len(of))(*of)
    a = jd.jd_rope_axes_t(n, C.addressof(buf))
    a._keep = buf
    return a


BAD = [dict(tokens=-1), dict(tokens=1 << 31), dict(q_heads=-1), dict(q_heads=0, k_heads=0), dict(k_heads=65537), dict(head_dim=0), dict(head_dim=257),
       dict(dtype=jd.JD_DTYPE_FP8_E4M3), dict(q=0), dict(k=0), dict(q=4097), dict(positions=0), dict(positions=258), dict(q_stride=100), dict(k_stride=-64),
       dict(rope=jd.jd_rope_t(0, 64, 0, 1.0)), dict(rope=jd.jd_rope_t(256, 63, 0, 1.0)), dict(rope=jd.jd_rope_t(256, 66, 0, 1.0)),
       dict(rope=jd.jd_rope_t(256, 64, 2, 1.0)), dict(rope=jd.jd_rope_t(256, 64, 0, float("nan"))), dict(norm=_norm(eps=-1e-6)),
       dict(norm=_norm(eps=float("inf"))), dict(norm=_norm(q_weight=258)), dict(axes=axes(0, [0] * 32)), dict(axes=axes(5, [0] * 32)),
       dict(axes=axes(2, [0] * 31 + [2]))]


@pytest.mark.parametrize("kw", BAD, ids=lambda kw: "-".join(kw))
def test_head_rope_refusals(kw):
    assert jd.load().jd_head_rope(head_args(**kw), None) == jd.JD_ERR_INVALID_ARG
    assert jd.load().jd_head_rope_grad(head_args(grad=True, **kw), None) == jd.JD_ERR_INVALID_ARG


def test_head_rope_refusals_of_one_direction():
    lib = jd.load()
    assert lib.jd_head_rope(None, None) == jd.JD_ERR_INVALID_ARG and lib.jd_head_rope_grad(None, None) == jd.JD_ERR_INVALID_ARG
    assert lib.jd_head_rope(head_args(inverse=1, norm=_norm()), None) == jd.JD_ERR_INVALID_ARG
    assert lib.jd_head_rope(head_args(inverse=2), None) == jd.JD_ERR_INVALID_ARG
    assert lib.jd_head_rope(head_args(q_out=4096, q_out_stride=256), None) == jd.JD_ERR_INVALID_ARG     # in place, another stride
    assert lib.jd_head_rope(head_args(tokens=0, q=0, k=0, positions=0), None) == jd.JD_OK
    need = lib.jd_head_rope_grad_workspace_bytes(64)
    assert need > 0 and lib.jd_head_rope_grad_workspace_bytes(0) == 0 == lib.jd_head_rope_grad_workspace_bytes(257)
    bad = [dict(norm=0), dict(q_weight_grad=256), dict(q_weight_grad=256, workspace=256, workspace_bytes=need - 1), dict(q_weight_grad=257, workspace=256, workspace_bytes=need),
           dict(q_grad=0), dict(k_out_grad=0), dict(q_grad=4096, q_grad_stride=256)]
    for kw in bad:
        assert lib.jd_head_rope_grad(head_args(grad=True, **kw), None) == jd.JD_ERR_INVALID_ARG, kw


def probs_args(**kw):
    a = jd.jd_verify_probs_args_t()
    a.B, a.nodes, a.V, a.dtype, a.mode, a.tau = 2, 5, 100, jd.JD_DTYPE_F32, jd.JD_MODE_STANDARD, 0.5
    for n in ("target", "draft", "tokens", "accept_u", "sample_u", "accept_len", "next_token"):
        setattr(a, n, 4096)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw", [dict(B=-1), dict(B=65536), dict(nodes=0), dict(nodes=129), dict(V=0), dict(V=(1 << 28) + 1), dict(dtype=2), dict(mode=3), dict(resample=2),
                                dict(siblings=2), dict(per_seq=2), dict(target=0), dict(target=4098), dict(draft=0), dict(tokens=0), dict(tokens=4097), dict(accept_u=0),
                                dict(sample_u=0), dict(accept_len=0), dict(next_token=0), dict(path=4097), dict(parents=4098), dict(num_nodes=4098), dict(device_status=4098),
                                dict(target_stride=99), dict(draft_stride=-1), dict(mode=1), dict(mode=2, judge_scores=4096, tau=1.5),
                                dict(mode=1, judge_scores=4096, tau=float("nan"))], ids=lambda kw: "-".join("%s=%s" % i for i in kw.items()))
def test_verify_probs_refusals(kw):
    assert jd.load().jd_verify_probs(probs_args(**kw), None) == jd.JD_ERR_INVALID_ARG


def test_verify_probs_nothing_to_do():
    assert jd.load().jd_verify_probs(probs_args(B=0, target=0, tokens=0), None) == jd.JD_OK
    assert jd.load().jd_verify_probs(None, None) == jd.JD_ERR_INVALID_ARG


def test_plan_refusals_without_a_handle():
    plan = jd.jd_shared_t(2, 4, 4096, 1 << 30)
    assert jd.load().jd_cache_shared_bytes(None, 2, 4) == 0
    assert jd.load().jd_cache_share(None, plan, None, None, None) == jd.JD_ERR_INVALID_ARG
    assert jd.load().jd_cache_attend_shared(None, jd.jd_attend_args_t(), plan, None) == jd.JD_ERR_INVALID_ARG


def test_objects_refuse_what_they_cannot_mean():
    f = torch.ones(4)
    for bad in ([0, 0, 0], [0, 1, 2, 4], [0, -1, 0, 0]):
        with pytest.raises(ValueError, match="axes"):
            jd.Rotary(f, axes=bad)
    assert jd.Rotary(f, axes=[0, 1, 2, 2]).num_axes == 3
    with pytest.raises(ValueError, match="weights"):
        jd.HeadNorm(torch.ones(4))                                     # on the host
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(ValueError, match="eps"):
            jd.HeadNorm(eps=eps)
    with pytest.raises(ValueError, match="target"):
        jd.verify_probs(torch.ones(1, 2, 3), torch.ones(1, 1, 3), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, 1), torch.zeros(1))


# ------------------------------------------------------------------------------------------- the model
@pytest.mark.parametrize("layout,of", [("half", None), ("interleaved", None), ("half", [0, 1, 1]), ("interleaved", [2, 0, 1])])
def test_model_gradient_against_differences(layout, of):
    """Central differences of a smooth function: off by h^2 times its third derivative (some 10^-8 here) and 2^-53 / h."""
    rng = np.random.default_rng(0)
    x, w, g = rng.normal(size=(2, 3, 8)), rng.normal(size=8), rng.normal(size=(2, 3, 8))
    pos = rng.integers(0, 50, size=(2,) if of is None else (2, 3))
    angle = S.angles(pos, [1.0, 0.3, 0.01], of)
    f = lambda x, w: (g * S.heads(x, w, 1e-3, angle, layout, 1.25)).sum()   # noqa: E731
    dx, dw = S.heads_grad(g, x, w, 1e-3, angle, layout, 1.25)
    h = 1e-5
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = h
        assert abs((f(x + e, w) - f(x - e, w)) / (2 * h) - dx[i]) < 1e-6
    for i in range(8):
        e = np.zeros(8)
        e[i] = h
        assert abs((f(x, w + e) - f(x, w - e)) / (2 * h) - dw[i]) < 1e-6


def test_model_axes_of_one_position_are_one_axis():
    rng = np.random.default_rng(1)
    x, pos = rng.normal(size=(5, 2, 8)), rng.integers(0, 1000, size=5)
    assert np.array_equal(S.turn(x, S.angles(pos, [1., .5, .1, .02]), "half"), S.turn(x, S.angles(np.stack([pos] * 3, 1), [1., .5, .1, .02], [0, 2, 1, 0]), "half"))


def _emitted(p, q, children, distinct):
    """The law of the first emitted token in exact arithmetic: children drawn from q in every possible way, accepted by their probability."""
    law = [Fraction(0)] * len(p)

    def go(k, prob, w, W, d, Q):
        if prob == 0:
            return
        if k == children:
            total = sum(w)
            for v, x in enumerate(w if total else p):
                law[v] += prob * x / (total or sum(p))
            return
        for x in range(len(p)):
            if d[x] == 0:
                continue
            draw = d[x] / Q
            accept = min(Fraction(1), w[x] * Q / (W * d[x])) if W else Fraction(0)
            law[x] += prob * draw * accept
            left = [max(Fraction(0), a * Q - W * b) for a, b in zip(w, d)]
            e, R = list(d), Q
            if distinct:
                R, e[x] = Q - d[x], Fraction(0)
            go(k + 1, prob * draw * (1 - accept), left, sum(left), e, R)

    go(0, Fraction(1), list(p), Fraction(1), list(q), Fraction(1))
    return law


@pytest.mark.parametrize("distinct", [False, True])
@pytest.mark.parametrize("children", [1, 2, 3])
def test_the_rule_keeps_the_targets_law(children, distinct):
    """What the header states, walked exactly: whatever the draft, the emitted token has the target's law."""
    cases = [([5, 1, 2, 0], [1, 1, 1, 1]), ([1, 2, 3, 4], [4, 3, 2, 1]), ([0, 0, 7, 1], [3, 3, 1, 1]), ([1, 1, 1, 1], [1, 1, 1, 1])]
    for a, b in cases:
        p, q = ([Fraction(x, sum(v)) for x in v] for v in (a, b))
        assert _emitted(p, q, children, distinct) == p


@pytest.mark.parametrize("distinct", [False, True])
def test_model_takes_those_decisions(distinct):
    """Two children of node 0 and every pair of numbers of a grid: the model accepts exactly where the exact rule does."""
    p, q = [Fraction(x, 8) for x in (1, 3, 4)], [Fraction(x, 8) for x in (4, 3, 1)]
    for x, y in itertools.product(range(3), repeat=2):
        if distinct and x == y:
            continue
        for i, j in itertools.product(range(16), repeat=2):
            u, v = Fraction(i, 16), Fraction(j, 16)
            if u * q[x] < p[x]:
                want = [1]
            else:
                left = [max(Fraction(0), a - b) for a, b in zip(p, q)]
                d, Q = list(q), Fraction(1)
                if distinct:
                    Q, d[x] = 1 - q[x], Fraction(0)
                want = [2] if v * sum(left) * d[y] < left[y] * Q else []
            got, _, status = S.verify(np.array([[float(a) for a in p]] * 3), np.array([[float(a) for a in q]] * 2), [x, y], [float(u), float(v)], 0.5,
                                      parents=[-1, 0, 0], distinct=distinct)
            assert got == want and status == S.OK


def test_model_reports_and_falls_back():
    p = np.array([[0.5, 0.5], [1.0, 0.0]])
    q = np.array([[0.5, 0.5]])
    assert S.verify(p, q, [2], [0.0], 0.6) == ([], 1, S.BAD_TOKEN)                # nothing subtracted is left: max(0, p - q) = 0, the target's own
    assert S.verify(p, q, [0], [0.0], 0.6, parents=[-1, 1]) == ([], 1, S.BAD_INDEX)
    assert S.verify(p, q, [0], [0.0], 0.99) == ([1], 0, S.OK)
    assert S.verify(p, q, [0], [0.0], 0.99, mode="judge", judged=[False]) == ([], 1, S.OK)
    assert S.verify(np.zeros((1, 3)), np.zeros((0, 3)), [], [], 0.5) == ([], 2, S.OK)


# ------------------------------------------------------------------------------------------- rows as they are stored
def _stored(x, dtype):
    """Float64 values of what float32 or bfloat16 holds of x."""
    return torch.as_tensor(np.asarray(x), dtype=torch.float64).to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype]).double().numpy()


def _stored_softmax(z, dtype):
    return _stored(torch.softmax(torch.as_tensor(np.asarray(z), dtype=torch.float32), 0).numpy(), dtype)


def _edge(holds):
    """The number of [0, 1] up to which holds(u) is true, by halving."""
    lo, hi = 0.0, 1.0
    if not holds(lo):
        return 0.0
    for _ in range(40):
        mid = (lo + hi) / 2
        lo, hi = (mid, hi) if holds(mid) else (lo, mid)
    return hi


def _law_of_the_model(p, q, children, distinct):
    """The law of the first emitted token by the model's own decisions: siblings drawn from the row as a sampler draws them, from what is left over its sum, and
    the borders of every number's interval found by halving."""
    V, T, law = len(p), children + 1, np.zeros(len(p))
    P, D, below = np.tile(p, (T, 1)), np.tile(q, (T - 1, 1)), 1 - 2.0 ** -24

    def emitted(prob, tokens):
        u = [below] * children
        for i in range(children):
            def taken(x):
                return S.verify(P, D, tokens, u[:i] + [x] + u[i + 1:], 0.5, parents=[-1] + [0] * children, distinct=distinct)[0] == [i + 1]
            accept = _edge(taken)
            law[tokens[i]] += prob * accept
            prob *= 1 - accept
            if accept > below:
                return
        edges = [0.0] + [_edge(lambda x: S.verify(P, D, tokens, u, x, parents=[-1] + [0] * children, distinct=distinct)[1] <= v) for v in range(V)]
        law[:] += prob * np.diff(edges)

    def drawn(prob, tokens, d):
        if len(tokens) == children:
            return emitted(prob, tokens)
        for x in range(V):
            if d[x] > 0:
                left = d.copy()
                if distinct:
                    left[x] = 0
                drawn(prob * d[x] / d.sum(), tokens + [x], left)

    drawn(1.0, [], q.copy())
    return law


CONFIDENT = [  # the draft's row and its type: one token holds what the type rounds to 1, or nearly all; two hold all; none does
    (_stored_softmax([20, 0, 0.5, -1], "f32"), "float32, 1 as stored"), (_stored([.9, .04, .03, .03], "f32"), "float32, .9"),
    (_stored([.99, .004, .003, .003], "f32"), "float32, .99"), (_stored_softmax([20, 19, 0.5, -1], "f32"), "float32, two tokens"),
    (_stored([.9, .04, .03, .03], "bf16"), "bf16, .9"), (_stored([.99, .004, .003, .003], "bf16"), "bf16, .99"), (_stored([.999, .0004, .0003, .0003], "bf16"), "bf16, .999"),
    (_stored([.55, .44, .006, .004], "bf16"), "bf16, two tokens"), (_stored([.4, .3, .2, .1], "bf16"), "bf16, flat")]


@pytest.mark.parametrize("distinct", [False, True])
@pytest.mark.parametrize("children", [2, 3, 4])
@pytest.mark.parametrize("row", [r for r, _ in CONFIDENT], ids=[n for _, n in CONFIDENT])
def test_the_targets_law_behind_confident_drafts(row, children, distinct):
    """With e = how far the rows' sums are from 1: acceptances and what is left after the first rejection are off by 2 e in all; a later sibling's by the error of what is taken
    for the rest of the draft's row, at most 2 e of it (subtracted from 1, half of the row is left at least; else it is the sum). Halving and numbers that end below 1: 10^-6."""
    p = _stored([.5, .2, .2, .1], "f32")
    e = abs(row.sum() - 1) + abs(p.sum() - 1)
    law = _law_of_the_model(p, row, children, distinct)
    assert np.abs(law - p).max() <= (2 + 4 * (children - 1)) * e + 1e-6


def test_siblings_of_a_draft_that_has_nothing_left():
    """One token holds the whole row: the rest of the row is nothing, and what it was sampled from cannot reject the target's weights a second time."""
    p, q = np.array([[.5, .3, .2]] * 4), np.array([[1., 0., 0.]] * 3)
    for u, want in ((0.1, 1), (0.59, 1), (0.61, 2), (0.9, 2)):                    # p without token 0: (0, .6, .4)
        assert S.verify(p, q, [0, 1, 2], [0.6, 0.999, 0.999], u, parents=[-1, 0, 0, 0], distinct=True) == ([], want, S.OK)


def _shares(p, q, tokens, distinct):
    """What is left of p after rejections of all tokens, each step divided by its sums."""
    w, d = p.copy(), q.copy()
    for x in tokens:
        if d.sum() > 0 and w.sum() > 0:
            w = np.maximum(0.0, w / w.sum() - d / d.sum())
        if distinct:
            d[x] = 0
    return w / w.sum()


@pytest.mark.parametrize("distinct", [False, True])
def test_many_rejections_leave_the_rest_of_the_target(distinct):
    """127 siblings of confident rows, all rejected: what is left keeps its size, however small the products of what was left on the way."""
    rng = np.random.default_rng(5)
    V, n = 2000, 127
    p, q = (_stored_softmax(12 * rng.normal(size=V), "f32") for _ in range(2))
    tokens = np.argsort(-(np.log(np.maximum(q, 1e-300)) + rng.gumbel(size=V)))[:n] if distinct else rng.choice(V, size=n, p=q / q.sum())
    left = q.copy()
    for x in tokens:                                                              # rejected: the target's weight is 1/250 of the draft's there
        p[x] = left[x] / left.sum() / 250
        if distinct:
            left[x] = 0
    other = np.setdiff1d(np.arange(V), tokens)
    p[other] *= (1 - p[tokens].sum()) / p[other].sum()
    run = np.cumsum(_shares(p, q, tokens, distinct))
    us = np.linspace(0.001, 0.999, 41)
    got = [S.verify(np.tile(p, (n + 1, 1)), np.tile(q, (n, 1)), tokens, [0.999] * n, u, parents=[-1] + [0] * n, distinct=distinct) for u in us]
    assert all(path == [] for path, _, _ in got)
    # sums in another order and rows whose sum is off 1 by 2^-23 move a border between tokens by some 10^-6
    for u, (_, token, _) in zip(us, got):
        assert token in {int(np.searchsorted(run, x, side="right")) for x in (u - 1e-5, u, u + 1e-5)}
