"""What of the cache's interface needs no device: struct layouts, refusals, frequencies, trees, and the CPU model itself."""
import ctypes as C
import math
import os
import re

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2501_19309_b200 import jd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("name", ["jd_rope_t", "jd_rope_args_t", "jd_cache_config_t", "jd_cache_buffers_t", "jd_tree_t",
                                  "jd_append_args_t", "jd_attend_args_t", "jd_commit_args_t"])
def test_struct_layouts_follow_the_header(name):
    src = open(os.path.join(ROOT, "include", "jd.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    body = re.search(r"typedef struct \{([^{}]*)\} %s;" % name, src).group(1)
    fields = []
    for decl in body.split(";"):
        for part in decl.split(","):
            m = re.search(r"([A-Za-z_0-9]+)\s*$", part.strip())
            if m:
                fields.append(m.group(1))
    assert fields == [f[0] for f in getattr(jd, name)._fields_]


def test_struct_sizes_match_a_c_compiler(tmp_path):
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("gcc is not installed")
    names = ["jd_rope_t", "jd_rope_args_t", "jd_cache_config_t", "jd_cache_buffers_t", "jd_tree_t", "jd_append_args_t",
             "jd_attend_args_t", "jd_commit_args_t"]
    src = '#include <stdio.h>\n#include "jd.h"\nint main(void) {\n%s  return 0;\n}\n' % "".join(
        '  printf("%%d\\n", (int)sizeof(%s));\n' % n for n in names)
    (tmp_path / "s.c").write_text(src)
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")], check=True)
    got = subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in got] == [C.sizeof(getattr(jd, n)) for n in names]


def test_packed_arguments_have_the_struct_layout():
    from paper_2501_19309_b200 import cache
    for packer, name in ((cache._ROPE_ARGS, "jd_rope_args_t"), (cache._APPEND_ARGS, "jd_append_args_t"), (cache._ATTEND_ARGS, "jd_attend_args_t"),
                         (cache._COMMIT_ARGS, "jd_commit_args_t")):
        t = getattr(jd, name)
        flat = []

        def leaves(s, base):
            for f, ft in s._fields_:
                off = base + getattr(s, f).offset
                if isinstance(ft, type) and issubclass(ft, C.Structure):
                    leaves(ft, off)
                else:
                    flat.append((off, C.sizeof(ft)))

        leaves(t, 0)
        a = t()
        packer.pack_into(a, 0, *range(1, len(flat) + 1))
        raw = bytes(a)
        for i, (off, size) in enumerate(flat):
            got = int.from_bytes(raw[off:off + size], "little")
            assert got == i + 1 or np.frombuffer(raw[off:off + size], dtype=np.float32)[0] == i + 1, (name, i)
        assert packer.size <= C.sizeof(t)


def config(**kw):
    base = dict(num_layers=2, num_pages=100, page_size=16, q_heads=8, kv_heads=2, head_dim=128, max_seqs=4, max_pages=32,
                max_nodes=26, dtype=jd.JD_DTYPE_BF16, device=0)
    base.update(kw)
    return jd.jd_cache_config_t(*[base[f[0]] for f in jd.jd_cache_config_t._fields_])


BAD = [dict(num_layers=0), dict(num_pages=0), dict(page_size=4), dict(page_size=24), dict(page_size=2048), dict(q_heads=7), dict(q_heads=0),
       dict(kv_heads=0), dict(kv_heads=-2), dict(head_dim=12), dict(head_dim=0), dict(head_dim=264), dict(max_seqs=0), dict(max_pages=0),
       dict(max_pages=1 << 21), dict(max_nodes=0), dict(max_nodes=129), dict(dtype=jd.JD_DTYPE_FP8_E4M3), dict(dtype=5),
       dict(num_pages=1 << 24, num_layers=64)]


def test_workspace_and_configurations():
    need = jd.load().jd_cache_workspace_bytes
    small, large = need(C.byref(config(max_nodes=1))), need(C.byref(config()))
    assert 0 < small < large < 1 << 30
    for kw in BAD:
        assert need(C.byref(config(**kw))) == 0, kw
    assert need(None) == 0


def test_refusals_without_a_device():
    lib = jd.load()
    h = C.c_void_p()
    buf = jd.jd_cache_buffers_t()
    cfg = config()
    assert lib.jd_cache_create(C.byref(h), C.byref(cfg), C.byref(buf)) == jd.JD_ERR_INVALID_ARG        # null buffers
    need = lib.jd_cache_workspace_bytes(C.byref(cfg))
    for name, at in (("k_pages", 8), ("page_table", 2), ("workspace", 128), ("workspace_bytes", need - 1)):
        buf = jd.jd_cache_buffers_t(*([1 << 20] * 8), need)
        setattr(buf, name, at if name == "workspace_bytes" else (1 << 20) + at)
        assert lib.jd_cache_create(C.byref(h), C.byref(cfg), C.byref(buf)) == jd.JD_ERR_INVALID_ARG, name
    bad = config(page_size=24)
    buf = jd.jd_cache_buffers_t(*([1 << 20] * 8), need)
    assert lib.jd_cache_create(C.byref(h), C.byref(bad), C.byref(buf)) == jd.JD_ERR_INVALID_ARG
    assert not h.value
    assert lib.jd_cache_destroy(None) == jd.JD_OK
    one = C.c_int(0)
    for f, args in (("reserve", (1, None, 1, None)), ("append", (C.byref(jd.jd_append_args_t()), None)), ("attend", (C.byref(jd.jd_attend_args_t()), None)),
                    ("commit", (C.byref(jd.jd_commit_args_t()), None)), ("fork", (1, None, None, None)), ("truncate", (1, None, None, None)),
                    ("compact", (None, None)), ("last_status", (C.byref(one),))):
        assert getattr(lib, "jd_cache_" + f)(None, *args) == jd.JD_ERR_INVALID_ARG, f


def rope_args(**kw):
    r = dict(inv_freq=4096, rot_dim=64, layout=0, amplitude=1.0)
    a = dict(tokens=2, heads=2, head_dim=64, dtype=jd.JD_DTYPE_BF16, inverse=0, x=1 << 20, out=1 << 21, x_stride=0, out_stride=0, positions=4096)
    for k, v in kw.items():
        (r if k in r else a)[k] = v
    return jd.jd_rope_args_t(*[a[f[0]] if f[0] != "rope" else jd.jd_rope_t(*[r[g[0]] for g in jd.jd_rope_t._fields_])
                               for f in jd.jd_rope_args_t._fields_])


@pytest.mark.parametrize("kw", [dict(tokens=-1), dict(heads=0), dict(head_dim=0), dict(head_dim=257), dict(dtype=2), dict(x=0), dict(out=0),
                                dict(positions=0), dict(positions=4098), dict(x=(1 << 20) + 1), dict(inv_freq=0), dict(inv_freq=4097),
                                dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=66), dict(layout=2), dict(layout=-1), dict(x_stride=127),
                                dict(out_stride=-128), dict(amplitude=math.nan), dict(amplitude=math.inf), dict(out=1 << 20, x_stride=256)])
def test_rope_refusals(kw):
    """None of these reaches the device."""
    assert jd.load().jd_rope(C.byref(rope_args(**kw)), None) == jd.JD_ERR_INVALID_ARG


def test_rope_nothing_to_do():
    assert jd.load().jd_rope(None, None) == jd.JD_ERR_INVALID_ARG
    assert jd.load().jd_rope(C.byref(rope_args(tokens=0, x=0, out=0, positions=0)), None) == jd.JD_OK


@pytest.mark.parametrize("rot,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (256, 1e6)])
def test_frequencies(rot, base):
    f0 = base ** (-np.arange(0, rot, 2) / rot)
    half_ulp = 2.0 ** -24 * (1 + 1e-9)

    def near(got, want):
        return (np.abs(got.numpy().astype(np.float64) - want) <= half_ulp * want * 2).all()

    got, amp = jd.rope_frequencies(rot, base)
    assert near(got, f0) and amp == 1.0
    got, amp = jd.rope_frequencies(rot, base, "linear", 4.0)
    assert near(got, f0 / 4) and amp == 1.0
    factor, old, low, high = 8.0, 8192.0, 1.0, 4.0
    want = []
    for f in f0:                                         # by wavelength, in three cases
        wave = 2 * math.pi / f
        if wave < old / high:
            want.append(f)
        elif wave > old / low:
            want.append(f / factor)
        else:
            s = (old / wave - low) / (high - low)
            want.append((1 - s) * f / factor + s * f)
    got, amp = jd.rope_frequencies(rot, base, "bands", factor, old, low, high)
    assert near(got, np.array(want)) and amp == 1.0
    got, amp = jd.rope_frequencies(rot, base, "yarn", factor, old, 1.0, 32.0)
    dim = [rot * math.log(old / (t * 2 * math.pi)) / (2 * math.log(base)) for t in (32.0, 1.0)]
    lo, hi = max(math.floor(dim[0]), 0), min(math.ceil(dim[1]), rot // 2 - 1)
    if hi <= lo:
        hi = lo + 0.001
    ramp = np.clip((np.arange(rot // 2) - lo) / (hi - lo), 0, 1)
    assert near(got, f0 / factor * ramp + f0 * (1 - ramp)) and abs(amp - (0.1 * math.log(factor) + 1)) < 1e-6


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=258), dict(base=1.0), dict(base=math.inf), dict(base=math.nan),
                                dict(scaling="linear", factor=0.5), dict(scaling="bands", factor=2.0, low=4.0, high=4.0),
                                dict(scaling="yarn", factor=2.0, original_len=0.0), dict(scaling="yarn", factor=2.0, low=0.0),
                                dict(scaling="linear", factor=math.inf)])
def test_frequency_refusals(kw):
    with pytest.raises(jd.JdError):
        jd.rope_frequencies(kw.pop("rot_dim", 64), **kw)


def test_trees():
    rng = np.random.default_rng(0)
    for T in (1, 2, 31, 32, 33, 100):
        parents = [-1] + [int(rng.integers(0, i)) for i in range(1, T)]
        see, depth = O.visible(parents)
        t = jd.Tree.from_parents(parents, "cpu")
        words = t.mask.numpy().view(np.uint32)
        got = np.array([[(words[i, j // 32] >> (j % 32)) & 1 for j in range(T)] for i in range(T)], dtype=bool)
        assert np.array_equal(got, see) and np.array_equal(t.depth.numpy(), depth) and t.batch == 0
        assert jd.Tree.from_parents([parents, parents], "cpu").batch == 2
    for bad in ([0], [-1, 1], [-1, 0, 3], [-1, -1]):
        with pytest.raises(ValueError):
            jd.Tree.from_parents(bad, "cpu")
    with pytest.raises(ValueError):
        jd.Tree(33, mask=torch.zeros(33, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        jd.Tree(3, mask=torch.zeros(2, 3, 1, dtype=torch.int32), depth=torch.zeros(3, dtype=torch.int32))


def model(seqs=4, pages=12, page=8, per_seq=4, D=4):
    rng = np.random.default_rng(1)
    return O.Cache(rng.standard_normal((1, pages, 1, page, D)), rng.standard_normal((1, pages, 1, page, D)), np.full((seqs, per_seq), -1),
                   np.zeros(seqs), np.zeros(seqs), np.zeros(pages), 8)


def test_model_copies_a_shared_page_before_it_is_written():
    m = model()
    m.reserve(5, [0])
    k = np.arange(20.0).reshape(1, 5, 1, 4)
    m.append(0, k, -k, [0])
    m.commit([4], None, [0], 4)
    m.fork([0], [1])
    assert m.refs[0] == 2 and m.len[1] == 5
    m.reserve(1, [1])
    assert m.refs[0] == 1 and m.table[1, 0] == 1 and np.array_equal(m.sequence(0, 0, 1)[0], m.sequence(0, 0, 0)[0])
    m.append(0, k[:, :1] + 100, k[:, :1], [1])
    assert np.array_equal(m.sequence(0, 0, 0)[0], k[0, :, 0]) and m.status == O.OK
    m.truncate(None, [0])
    assert m.refs.tolist()[:2] == [0, 1] and m.compact() == 1 and m.table[1, 0] == 0


def test_model_commits_a_path():
    m = model()
    m.reserve(8, [2])
    k = np.arange(32.0).reshape(1, 8, 1, 4)
    m.append(0, k, k, [2])
    chosen = m.commit([[1, 3]], np.array([[[1, 2, 3], [2, 4, 7]]]), [2])
    assert chosen == {0: 1} and m.len[2] == 4
    assert np.array_equal(m.sequence(0, 0, 2)[0], k[0, [0, 2, 4, 7], 0])


def test_model_attention_is_a_softmax():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((2, 4)), rng.standard_normal((5, 4)), rng.standard_normal((5, 3))
    see = np.array([[1, 1, 0, 1, 0], [0, 0, 0, 0, 0]], dtype=bool)
    out, lse = O.attend(q, k, v, see, 0.5)
    e = np.exp(0.5 * k[[0, 1, 3]] @ q[0])
    assert np.allclose(out[0], e @ v[[0, 1, 3]] / e.sum()) and np.isclose(lse[0], np.log(e.sum()))
    assert (out[1] == 0).all() and np.isneginf(lse[1])


def test_model_rotation():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 9.0]]])
    f = np.array([0.5, 0.25], dtype=np.float32)
    y = O.rope(x, [2], f, "half")
    assert np.allclose(y[0, 0], [math.cos(1) - 3 * math.sin(1), 2 * math.cos(.5) - 4 * math.sin(.5), 3 * math.cos(1) + math.sin(1),
                                 4 * math.cos(.5) + 2 * math.sin(.5), 9.0])
    y = O.rope(x, [2], f, "interleaved", 2.0)
    assert np.allclose(y[0, 0, :2], [2 * (math.cos(1) - 2 * math.sin(1)), 2 * (2 * math.cos(1) + math.sin(1))])
    assert np.allclose(O.rope(O.rope(x, [7], f, "half"), [7], f, "half", inverse=True), x)


def test_strides_that_steps_cannot_say_are_refused():
    """A step of 0 stands for dense tokens: broadcast and overlapping tokens must not come out as that."""
    from paper_2501_19309_b200.cache import PagedCache, Rotary
    one = torch.zeros(1, 4, 64)
    with pytest.raises(ValueError):
        Rotary._step(one.expand(5, 4, 64), "x", 5, 4, 64)
    with pytest.raises(ValueError):
        Rotary._step(torch.zeros(5 * 256).as_strided((3, 4, 64), (128, 64, 1)), "x", 3, 4, 64)
    assert Rotary._step(one.expand(1, 4, 64), "x", 1, 4, 64) == 0
    assert Rotary._step(torch.zeros(5, 6, 64)[:, :4], "x", 5, 4, 64) == 384
    c = object.__new__(PagedCache)
    c.h, c.dtype, c.index = None, torch.float32, -1
    for B, T in ((1, 5), (5, 1), (2, 5)):
        with pytest.raises(ValueError):
            c._tokens(one.unsqueeze(0).expand(B, T, 4, 64), "q", (B, T, 4, 64))
    with pytest.raises(ValueError):
        c._tokens(torch.zeros(2048).as_strided((1, 3, 4, 64), (256, 128, 64, 1)), "q", (1, 3, 4, 64))
    assert c._tokens(torch.zeros(2, 5, 6, 64)[:, :, :4], "q", (2, 5, 4, 64)) == 384
    assert c._tokens(torch.zeros(2, 5, 4, 64)[:, :1], "q", (2, 1, 4, 64)) == 5 * 256


def test_inputs_that_require_gradients_are_refused():
    from paper_2501_19309_b200.cache import PagedCache, Rotary
    c = object.__new__(PagedCache)
    c.h, c.dtype, c.index = None, torch.float32, -1
    x = torch.zeros(2, 3, 4, 64, requires_grad=True)
    with pytest.raises(ValueError):
        c._tokens(x, "q", (2, 3, 4, 64))
    with pytest.raises(ValueError):
        Rotary._step(x[0], "x", 3, 4, 64)
    with torch.no_grad():
        assert c._tokens(x, "q", (2, 3, 4, 64)) == 0 and Rotary._step(x[0], "x", 3, 4, 64) == 0


def test_a_tree_for_no_sequence_is_refused():
    with pytest.raises(ValueError):
        jd.Tree(3, mask=torch.zeros(0, 3, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        jd.Tree(3, depth=torch.zeros(0, 3, dtype=torch.int32))


def test_model_leaves_rows_of_shared_pages_alone():
    """Without pages to part on, a commit takes and moves nothing in a page that another sequence still reads."""
    m = O.Cache(np.zeros((1, 1, 1, 8, 2)), np.zeros((1, 1, 1, 8, 2)), np.full((2, 1), -1), np.zeros(2, int), np.zeros(2, int), np.zeros(1, int), 4)
    m.reserve(4, [0])
    m.append(0, np.arange(4.).reshape(1, 4, 1, 1).repeat(2, 3), np.zeros((1, 4, 1, 2)), [0])
    m.commit([3], None, [0], 3)
    m.fork([0], [1])
    m.truncate([1], [0])
    m.commit([[1]], np.array([[[2]]]), [0])           # would move row 3 over row 2 of sequence 1
    assert m.status == O.BAD_INDEX and m.len.tolist() == [1, 4] and m.k[0, 0, 0, :4, 0].tolist() == [0, 1, 2, 3]


PATH_HARNESS = r"""
#include <stdio.h>
#include <stdlib.h>
#include "jd_path.h"
int main(int argc, char** argv) {
  const int len = atoi(argv[1]), limit = atoi(argv[2]), max_nodes = atoi(argv[3]), shift = atoi(argv[4]);
  for (int i = 0, before = 0; i + 5 < argc; ++i) {
    const int node = atoi(argv[5 + i]);
    int from = 0, to = 0;
    const bool ok = jd::path_entries(len, limit, i, node, before, max_nodes, shift, &from, &to);
    printf("%d %d %d\n", (int)ok, from, to);
    before = node;
  }
}
"""


def test_no_node_of_a_path_leads_out_of_the_page_table(tmp_path):
    """A commit judges all nodes of a path at once, those behind a cut too: whatever stands there, a node that passes goes from and
    to entries of pages that the sequence holds, and up to the first that does not pass the answers are the definition's."""
    import shutil
    import subprocess
    if shutil.which("g++") is None:
        pytest.skip("g++ is not installed")
    (tmp_path / "p.cpp").write_text(PATH_HARNESS)
    csrc = os.path.join(ROOT, "paper_2501_19309_b200", "csrc")
    subprocess.run(["g++", "-std=c++17", "-I", csrc, str(tmp_path / "p.cpp"), "-o", str(tmp_path / "p")], check=True)
    rng = np.random.default_rng(0)
    far = 2 ** 31
    cases = [(0, 1, [-5, -3]), (0, 1, [-far, -far + 1]), (29, 4, [7, 1, 2]), (28, 4, [9, 1, 2, 3]), (5, 2, [1, 2, 3, 0, 1]), (0, 0, [1, 2]), (8, 1, [1, 2]),
             (0, 3, [far - 1, -far, -1, 0, 1, 2])]
    for _ in range(60):
        held = int(rng.integers(0, 4))
        cases.append((int(rng.integers(0, 8 * held + 1)), held, rng.integers(-4, 12, int(rng.integers(1, 9))).tolist()))
    for length, held, path in cases:
        text = subprocess.run([str(tmp_path / "p"), str(length), str(8 * held), "10", "3", *map(str, path)], capture_output=True, text=True,
                              check=True).stdout
        before, cut = 0, False
        for i, (node, line) in enumerate(zip(path, text.splitlines())):
            ok, at, to = map(int, line.split())
            assert not ok or (0 <= at < held and 0 <= to < held), (length, held, path, i)
            if not cut:
                assert ok == (before < node < 10 and length + node < 8 * held), (length, held, path, i)
            cut, before = cut or not ok, node


def test_model_takes_no_names_from_padding_entries_of_a_fork():
    m = model(seqs=6)
    m.reserve(3, [0])
    m.commit([2], None, [0], 3)
    m.fork([4, 0, -1, 0, 0, -1], [-1, 4, 2, 2, 5, 3])
    assert m.status == O.OK and m.len.tolist() == [3, 0, 3, 0, 3, 3] and m.refs[0] == 4


@pytest.mark.parametrize("rot,base,old,factor,low,high", [(128, 1e4, 65536.0, 4.0, 1.0, 32.0), (128, 1e4, 131072.0, 4.0, 1.0, 32.0), (64, 1e4, 1e6, 8.0, 1.0, 32.0),
                                                          (32, 100.0, 4096.0, 16.0, 2.0, 8.0), (8, 10.0, 1e9, 2.0, 1.0, 4.0), (128, 5e5, 8192.0, 8.0, 1.0, 32.0)])
def test_yarn_blend_runs_past_the_last_frequency(rot, base, old, factor, low, high):
    """From the definition: index x makes old x base^(-2 x / rot) / 2 pi turns; kept up to where that is `high` (rounded down), divided from
    where it is `low` (rounded up, rot - 1 at most), also where that lies behind the last of the rot / 2 indices."""
    f0 = base ** (-np.arange(0, rot, 2) / rot)
    turns = lambda x: old * base ** (-2 * x / rot) / (2 * math.pi)   # noqa: E731
    first = max([x for x in range(0, 40 * rot) if turns(x) >= high], default=0)
    last = min(min(x for x in range(0, 40 * rot) if turns(x) <= low), rot - 1)
    divided = np.clip((np.arange(rot // 2) - first) / (last - first if last > first else 0.001), 0, 1)
    got, amp = jd.rope_frequencies(rot, base, "yarn", factor, old, low, high)
    want = f0 * (1 - divided) + f0 / factor * divided
    assert (np.abs(got.numpy().astype(np.float64) - want) <= 2.0 ** -23 * (1 + 1e-9) * want).all() and abs(amp - (0.1 * math.log(factor) + 1)) < 1e-6


def test_tensors_with_a_tangent_are_refused():
    """Forward-mode derivatives would be lost as silently as a graph."""
    import torch.autograd.forward_ad as fw
    from paper_2501_19309_b200.cache import PagedCache, Rotary
    c = object.__new__(PagedCache)
    c.h, c.dtype, c.index = None, torch.float32, -1
    x = torch.zeros(2, 3, 4, 64)
    with fw.dual_level():
        dual = fw.make_dual(x, torch.ones_like(x))
        with pytest.raises(ValueError):
            c._tokens(dual, "q", (2, 3, 4, 64))
        with pytest.raises(ValueError):
            Rotary._step(fw.make_dual(x[0], torch.ones_like(x[0])), "x", 3, 4, 64)
        assert c._tokens(x, "q", (2, 3, 4, 64)) == 0 and Rotary._step(x[0], "x", 3, 4, 64) == 0
    assert c._tokens(x, "q", (2, 3, 4, 64)) == 0


def test_a_reserve_that_32_bits_do_not_hold_is_refused():
    from paper_2501_19309_b200.cache import PagedCache
    c = object.__new__(PagedCache)
    c.h, c.max_seqs, c.index, c._lib = None, 1, -1, None
    for n in ((1 << 32) + 1, 1 << 31, -(1 << 32) + 5):
        with pytest.raises(ValueError):
            c.reserve(n)


def test_workspace_holds_the_parts_that_the_cache_can_have():
    """Parts of up to 256 rows are the tensor-core kernel's alone; others are of 16 rows, two to each of at most 512 CTAs."""
    need = jd.load().jd_cache_workspace_bytes
    books = 1 << 17                                      # counters, and three numbers a page
    for D in (8, 80, 256):
        for dtype in (jd.JD_DTYPE_F32, jd.JD_DTYPE_BF16):
            got = need(C.byref(config(head_dim=D, dtype=dtype)))
            parts = 512 * 2 * 16 * (D + 4) * 4
            assert parts <= got <= parts + books, (D, dtype)
    for D in (64, 128):
        assert need(C.byref(config(head_dim=D, dtype=jd.JD_DTYPE_F32))) <= 512 * 2 * 16 * (D + 4) * 4 + books
        for nodes, rows in ((1, 32), (8, 32), (9, 36), (26, 104), (128, 256)):     # 4 query heads of a kv head
            got = need(C.byref(config(head_dim=D, max_nodes=nodes)))
            assert 256 * 2 * rows * (D + 4) * 4 <= got <= 256 * 2 * rows * (D + 4) * 4 + books, (D, nodes)


def test_tensor_memory_is_taken_between_the_wait_and_the_trigger():
    """A kernel that holds tensor memory while it waits for the one in front, or lets the next one start before it holds it, can wait for good on an
    SM that two of them share: shown by the order in the source, which no run may try."""
    src = open(os.path.join(ROOT, "paper_2501_19309_b200", "csrc", "jd_attend_sm100.cu")).read()
    body = src[src.index("attend_sm100_kernel("):]
    at = [body.index(x) for x in ("pdl_wait();", "tcgen05.alloc", "unit_prefix(", "pdl_trigger();", "tcgen05.dealloc")]
    assert at == sorted(at) and all(body.count(x) == 1 for x in ("pdl_wait();", "tcgen05.alloc", "pdl_trigger();"))


def test_more_tokens_than_a_rotation_takes_are_a_bad_argument():
    for n in (1 << 31, 1 << 40, (1 << 63) - 1):
        assert jd.load().jd_rope(C.byref(rope_args(tokens=n)), None) == jd.JD_ERR_INVALID_ARG


def test_frequencies_and_pages_that_require_gradients_are_refused():
    from paper_2501_19309_b200.cache import PagedCache
    with pytest.raises(ValueError, match="autograd"):
        jd.Rotary(torch.ones(4, requires_grad=True))
    ints = torch.zeros(1, dtype=torch.int32)
    for i in range(2):
        k, v = (torch.zeros(1, 1, 1, 8, 8, requires_grad=i == j) for j in range(2))
        with pytest.raises(ValueError, match="autograd"):
            PagedCache(k, v, ints.view(1, 1), ints, ints, ints, ints, 1)
