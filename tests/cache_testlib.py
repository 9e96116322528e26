"""Shared pieces of the cache tests: random caches on the device together with their CPU model."""
import numpy as np
import torch

from oracle import cache_oracle as O
from paper_2501_19309_b200 import jd

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.detach().cpu().double().numpy()


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def empty_cache(layers, pages, page, q_heads, kv_heads, D, seqs, per_seq, max_nodes, dtype="bf16", fill=None):
    c = jd.PagedCache.allocate(layers, pages, page, q_heads, kv_heads, D, seqs, per_seq, max_nodes, dtype)
    if fill is not None:
        gen = torch.Generator(device="cuda")
        gen.manual_seed(fill)
        c.k.copy_(torch.randn(c.k.shape, generator=gen, device="cuda"))
        c.v.copy_(torch.randn(c.v.shape, generator=gen, device="cuda"))
    return c


def model_of(c):
    return O.Cache(f64(c.k), f64(c.v), f64(c.page_table), f64(c.seq_len), f64(c.held), f64(c.refs), c.max_nodes)


def filled_cache(lens, room, *, page=16, q_heads=4, kv_heads=2, D=64, layers=1, max_nodes=32, dtype="bf16", seed=0, spare=3, extra_seqs=0):
    """A cache that holds lens[b] tokens and pages for `room` more, its pages scattered over the pool."""
    rng = np.random.default_rng(seed)
    want = [-(-(n + room) // page) for n in lens]
    seqs, P = len(lens) + extra_seqs, sum(want) + spare
    c = empty_cache(layers, P, page, q_heads, kv_heads, D, seqs, max(want + [1]) + 4, max_nodes, dtype, fill=seed)
    order, at = rng.permutation(P), 0
    table = np.full(tuple(c.page_table.shape), -1)
    refs = np.zeros(P, dtype=np.int64)
    for b, n in enumerate(want):
        table[b, :n] = order[at:at + n]
        at += n
    refs[order[:at]] = 1
    c.page_table.copy_(ints(table))
    c.refs.copy_(ints(refs))
    c.seq_len[:len(lens)] = ints(lens)
    c.held[:len(lens)] = ints(want)
    c.free_bits.copy_(free_words(refs))
    return c


def free_words(refs):
    n = len(refs)
    bits = np.zeros(-(-n // 32) * 32, dtype=np.uint64)
    bits[:n] = np.asarray(refs) == 0
    w = (bits.reshape(-1, 32) << np.arange(32, dtype=np.uint64)).sum(1).astype(np.uint32)
    return torch.from_numpy(w.view(np.int32).copy()).cuda()


def same_books(c, m):
    """Tables, lengths, owners and the bitmap agree with the model's."""
    torch.cuda.synchronize()
    for name, want in (("page_table", m.table), ("seq_len", m.len), ("held", m.held), ("refs", m.refs)):
        got = getattr(c, name).cpu().numpy()
        assert np.array_equal(got, want), (name, got, want)
    assert torch.equal(c.free_bits, free_words(m.refs))
    owners = np.zeros(len(m.refs), dtype=np.int64)
    for s in range(len(m.held)):
        for p in m.table[s, :m.held[s]]:
            owners[p] += 1
    assert np.array_equal(owners, m.refs)


def random_tree(T, rng, style="tree"):
    if style == "chain":
        return [i - 1 for i in range(T)]
    if style == "star":
        return [-1] + [0] * (T - 1)
    return [-1] + [int(rng.integers(max(0, i - 5), i)) for i in range(1, T)]


def device_tree(parents, **kw):
    return jd.Tree.from_parents(parents, "cuda", **kw)


def attend_tolerance(m, layer, q, see, scale, want, dtype, slots=None, num_nodes=None):
    """Bound on |out - exact| per element. Weights w_j = p_j / sum p: a score is off by at most (D + 4) 2^-24 A with
    A = scale sum |q_i k_i| (float32 products and sums in any order, scale and log2 e rounded), so a weight by that, twice
    (numerator and sum), and by 2^-20 for exp2 and the sums; bf16 rounds a weight by 2^-8 more, and the output by 2^-8 of its value."""
    D = q.shape[-1]
    big = O.Cache(np.abs(np.nan_to_num(m.k, nan=0., posinf=0., neginf=0.)), np.abs(np.nan_to_num(m.v, nan=0., posinf=0., neginf=0.)),
                  m.table, m.len, m.held, m.refs, m.max_nodes)
    A = scale * np.abs(q).max() * big.k.max() * D
    A = min(A, scale * np.linalg.norm(q, axis=-1).max() * np.linalg.norm(big.k, axis=-1).max())    # Cauchy-Schwarz
    # weights of the true softmax on |v|
    mm = O.Cache(m.k, big.v, m.table, m.len, m.held, m.refs, m.max_nodes)
    spread, _ = mm.attend(layer, q, see, scale, slots, num_nodes)
    tokens = int(m.len.max()) + q.shape[1]
    w = 2 * (D + 4) * 2.0 ** -24 * A + 2.0 ** -20 + tokens * 2.0 ** -24
    if dtype == "bf16":
        return spread * (w + 2.0 ** -8) + np.abs(want) * 2.0 ** -8 + 1e-30, w * (1 + 0 * spread[..., 0])
    return spread * w + np.abs(want) * 2.0 ** -24 + 1e-30, w * (1 + 0 * spread[..., 0])
