"""Attention and verification of trees of drafts, attention weights of stored tokens and eviction, on the GPU against 64 bits."""

import numpy as np
import pytest
import torch

from oracle import serving
from test_gpu_serving import DEV, U, Case, bits, i32, many, tolerance

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def spl():
    from paper_2609_15039_gb300 import spl as binding
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    binding.lib()
    return binding


def raw(t):
    """For comparisons to the bit."""
    return t.view({1: torch.int8, 2: torch.int16, 4: torch.int32}[t.element_size()])


# ---------------------------------------------------------------------------------- trees
def masks_of(parents):
    out = []
    for i, p in enumerate(parents):
        out.append((out[p] if p >= 0 else 0) | 1 << i)
    return out


def words_of(masks, words):
    """int32 [rows, words] of masks as ints."""
    m = np.array([[k >> 32 * w & 0xffffffff for w in range(words)] for k in masks], dtype=np.uint32).reshape(len(masks), words)
    return torch.as_tensor(m.view(np.int32)).to(DEV)


def random_tree(g, n):
    return [-1] + [int(g.integers(max(0, i - 9), i)) for i in range(1, n)] if n else []


def attend_tree(c, masks, words, window=0, scale=None, out=None, q=None):
    out = torch.full((c.rows, c.hq * c.d), float("nan"), device=DEV) if out is None else out
    q = torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV) if q is None else q
    c.spl.spl_tree_attention(out, q, c.cache, c.batch(), words_of(sum(masks, []), words), c.hq, scale=scale, window=window)
    torch.cuda.synchronize()
    return out.cpu().numpy().reshape(c.rows, c.hq, c.d)


def check_tree(c, masks, window=0, scale=None, words=None):
    words = max(1, -(-max(r for r, _ in c.seqs) // 32)) if words is None else words
    got = attend_tree(c, masks, words, window, scale)
    s = 1.0 / np.sqrt(c.d) if scale is None else scale
    for b, (r, n) in enumerate(c.seqs):
        if r == 0:
            continue
        k, v = c.stored("k", b), c.stored("v", b)
        q = c.q[c.start[b]:c.start[b + 1]]
        limit = [m & ((1 << 32 * words) - 1) for m in masks[b]]
        ref, mass = serving.tree_attention(q, k, v, limit, n - r, c.hq // c.hk, s, window)
        mine = got[c.start[b]:c.start[b + 1]]
        assert not np.isnan(mine).any(), f"sequence {b}: NaN"
        if n == 0:
            assert np.all(mine == 0)
            continue
        # as for attention; a probability's low half may lose 2^-33 of the row's largest
        tol = tolerance(q, k, s, n, c.hq // c.hk, mass) + 2.0 ** -32 * n * np.max(np.abs(v))
        err = np.abs(mine.astype(np.float64) - ref)
        assert np.all(err <= tol), f"sequence {b} {r, n}: worst err/tol {np.max(err / tol):.3g}"
        empty = [i for i in range(r) if len(serving.tree_keys(limit[i], n - r, n, window)) == 0]
        assert np.all(mine[empty] == 0)
    assert c.spl.spl_get_device_status() == c.spl.SPL_OK
    return got


TREES = {"one": [(1, 1)], "root": [(1, 300)], "small": [(16, 316), (1, 70), (0, 33), (7, 7), (0, 0), (31, 500)],
         "words": [(32, 532), (33, 33), (64, 164), (65, 365)], "large": [(130, 330), (200, 200), (3, 900)]}


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("heads", [(24, 8, 128), (8, 2, 64), (3, 3, 128), (7, 1, 64)], ids=str)
@pytest.mark.parametrize("name", TREES)
def test_tree_attention(spl, name, heads, fmt):
    """Both kernels, over trees as they are drafted."""
    g = np.random.default_rng(len(name))
    for kernel in (lambda c: c, many):
        c = kernel(Case(spl, TREES[name], heads, fmt, 16 if name == "small" else 64, seed=len(name)))
        c.fill()
        check_tree(c, [masks_of(random_tree(g, r)) for r, _ in c.seqs])


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("window", [1, 2, 5, 31, 33, 64, 150, 1000])
def test_tree_attention_window(spl, window, fmt):
    g = np.random.default_rng(window)
    for kernel in (lambda c: c, many):
        c = kernel(Case(spl, [(40, 340), (70, 70), (1, 500), (5, 133)], (4, 2, 64), fmt, 32, seed=window))
        c.fill()
        check_tree(c, [masks_of(random_tree(g, r)) for r, _ in c.seqs], window=window)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("context", [0, 1, 127, 200])
def test_tree_attention_any_masks(spl, context, fmt):
    """Masks that are no tree's: random ones, later rows among them, none at all, all bits set (past the last row too)."""
    g = np.random.default_rng(context)
    rows = 70
    random = [int.from_bytes(g.bytes(12), "little") for _ in range(rows)]
    for masks in (random, [0] * rows, [(1 << 96) - 1] * rows, [0 if i % 3 else random[i] for i in range(rows)]):
        for kernel in (lambda c: c, many):
            c = kernel(Case(spl, [(rows, rows + context), (3, 3)], (4, 2, 128), fmt, 16, seed=context))
            c.fill()
            for window in (0, 3):
                check_tree(c, [masks, masks[:3]], window=window, words=3)


def test_tree_attention_few_words(spl):
    """Rows past the words are not seen; without words only the context is, and a row without context sees nothing."""
    g = np.random.default_rng(1)
    for words in (0, 1, 2):
        for kernel in (lambda c: c, many):
            c = kernel(Case(spl, [(70, 170), (40, 40)], (4, 2, 64), "f16", 16, seed=2))
            c.fill()
            check_tree(c, [masks_of(random_tree(g, r)) for r, _ in c.seqs], words=words)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
def test_a_chain_is_causal_attention(spl, fmt):
    """A tree without branches: the bits of spl_paged_attention (the same products in the same order)."""
    for seqs in ([(5, 261), (1, 40)], [(130, 333), (64, 64)]):
        c = Case(spl, seqs, (6, 2, 128), fmt, 64, seed=3)
        c.fill()
        masks = [masks_of([i - 1 for i in range(r)]) for r, _ in seqs]
        for window in (0, 50):
            want, got = c.attend(window), attend_tree(c, masks, 5, window)
            assert np.max(np.abs(want - got)) <= 1e-5 * np.max(np.abs(want))


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("which", ["k", "v"])
def test_tree_rows_do_not_meet_what_they_do_not_see(spl, which, fmt):
    """A NaN in a node's vector reaches the rows below it and no others."""
    g = np.random.default_rng(4)
    for rows in (3, 20, 60):
        parents = random_tree(g, rows)
        masks = masks_of(parents)
        for kernel in (lambda c: c, many):
            c = kernel(Case(spl, [(rows, 100 + rows)], (4, 2, 64), fmt, 16, seed=rows))
            c.fill()
            clean = check_tree(c, [masks])
            at = rows // 2
            getattr(c, which)[0][100 + at, 1, 3] = np.nan
            c.fill()
            got = attend_tree(c, [masks], 2)
            below = np.array([m >> at & 1 == 1 for m in masks])
            assert np.array_equal(got[~below], clean[~below]) and np.array_equal(got[:, :2], clean[:, :2])
            assert np.isnan(got[below][:, 2:]).any(axis=2).all()


def test_tree_attention_lengths_and_pages_out_of_range(spl):
    """A length past the table, a negative one, more rows than tokens, pages outside the pool: reported, never followed."""
    g = np.random.default_rng(5)
    for kernel in (lambda c: c, many):
        c = kernel(Case(spl, [(40, 90), (20, 60)], (4, 2, 64), "f16", 16, seed=6))
        c.fill()
        masks = [masks_of(random_tree(g, r)) for r, _ in c.seqs]
        good = check_tree(c, masks)
        batch = c.batch()
        c.batch = lambda all_rows=False, batch=batch: batch
        for lens in ([-4, 60], [1 << 30, 60]):
            batch.kv_len.copy_(i32(lens))
            got = attend_tree(c, masks, 2)
            assert spl.spl_get_device_status() == spl.SPL_EINVAL
            assert np.array_equal(got[40:], good[40:]) or np.allclose(got[40:], good[40:], rtol=0, atol=1e-5)
        batch.kv_len.copy_(i32([90, 60]))
        batch.page_table[0, 1] = -7
        batch.page_table[0, 4] = 1 << 29
        got = attend_tree(c, masks, 2)
        assert spl.spl_get_device_status() == spl.SPL_EINVAL
        seen = [j for j in range(90) if j // 16 not in (1, 4)]
        k, v = c.stored("k", 0), c.stored("v", 0)
        for i in (0, 13, 39):
            keys = [j for j in serving.tree_keys(masks[0][i], 50, 90, 0) if j in seen]
            ref, _ = serving.attention(c.q[i:i + 1], k[keys], v[keys], len(keys), 2, 0.125)
            assert np.allclose(got[i], ref[0], rtol=0, atol=1e-5)
    c = Case(spl, [(6, 2), (50, 3)], (4, 2, 64), "f16", 16, seed=3)  # rows before position 0
    c.fill()
    for kernel in (lambda c: c, many):
        for window in (0, 2):
            got = check_tree(kernel(c), [masks_of(random_tree(g, r)) for r, _ in c.seqs], window=window)
            assert np.all(got[0] == 0)


def test_tree_attention_strides_and_streams(spl):
    g = np.random.default_rng(7)
    c = Case(spl, [(9, 50), (33, 61)], (6, 2, 64), "f16", 16, seed=8)
    c.fill()
    masks = [masks_of(random_tree(g, r)) for r, _ in c.seqs]
    want = check_tree(c, masks)
    wide, out = torch.full((c.rows, 1000), 7.0, device=DEV), torch.full((c.rows, 516), 5.0, device=DEV)
    wide[:, 8:392] = torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV)
    seen = words_of(sum(masks, []), 2)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        late = wide.clone()
        spl.spl_tree_attention(out[:, 64:448], late[:, 8:392], c.cache, c.batch(), seen, 6)
    s.synchronize()
    assert np.array_equal(out[:, 64:448].cpu().numpy().reshape(want.shape), want)
    assert bool((out[:, :64] == 5).all()) and bool((out[:, 448:] == 5).all())


# ---------------------------------------------------------------------------------- verification
def tree_draws(seed, counts, vocab, levels, good=0.7):
    """Trees of so many nodes, with target probabilities that often agree with a draft."""
    g = np.random.default_rng(seed)
    parents = [random_tree(g, n) for n in counts]
    x = [g.integers(0, vocab, n).astype(np.int32) for n in counts]
    p = []
    for n, par, t in zip(counts, parents, x):
        z = np.exp(1.5 * g.standard_normal((n, vocab)))
        z /= z.sum(-1, keepdims=True)
        for i in range(n):
            kids = [j for j in range(n) if par[j] == i]
            if kids:
                z[i] *= 1 - good
                z[i, t[kids]] += good / len(kids)
        p.append(z.astype(np.float32))
    e = np.maximum(g.exponential(size=(len(counts), levels, vocab)), 1e-30).astype(np.float32)
    return p, x, parents, e


def call_verify_tree(spl, p, x, parents, e, **kw):
    counts = [len(t) for t in x]
    start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    n, levels, vocab = e.shape
    accepted, token = i32([-9] * n), i32([-9] * n)
    path = torch.full((n, levels), -9, dtype=torch.int32, device=DEV)
    flat = lambda parts, t: torch.as_tensor(np.concatenate(parts).astype(t)).to(DEV)  # noqa: E731
    P = flat(p, np.float32) if kw.get("P") is None else kw["P"]
    E = torch.as_tensor(e.reshape(-1, vocab)).to(DEV) if kw.get("E") is None else kw["E"]
    spl.spl_verify_tree(accepted, path, token, P, flat(x, np.int32), flat(parents, np.int32), E, i32(start.tolist()))
    torch.cuda.synchronize()
    return accepted.tolist(), path.tolist(), token.tolist()


def check_verify_tree(spl, p, x, parents, e, **kw):
    accepted, path, token = call_verify_tree(spl, p, x, parents, e, **kw)
    levels = e.shape[1]
    for b in range(len(p)):
        if len(x[b]) == 0:
            assert (accepted[b], token[b], path[b]) == (0, -1, [-1] * levels)
            continue
        want, t = serving.verify_tree(p[b], x[b], parents[b], e[b])
        assert (accepted[b], token[b]) == (len(want), t) and path[b] == want + [-1] * (levels - len(want))
    assert spl.spl_get_device_status() == spl.SPL_OK
    return accepted


@pytest.mark.parametrize("vocab", [1, 2, 7, 1000, 4097, 50257, 128256])
def test_verify_tree(spl, vocab):
    taken = 0
    for seed, counts, levels in ((0, [1], 1), (1, [12], 6), (2, [5, 0, 33, 1, 60, 17, 2, 0], 5), (3, [20] * 40, 7)):
        if vocab > 50000 and len(counts) > 8:
            counts = counts[:12]
        taken += sum(check_verify_tree(spl, *tree_draws(seed, counts, vocab, levels)))
    assert taken > 0  # (some drafts are accepted)


def test_verify_tree_levels_end_the_walk(spl):
    """A chain that would be accepted to its end: the walk ends at the last level, with the target's token there."""
    vocab = 500
    p = np.zeros((9, vocab), dtype=np.float32)
    x = np.arange(9, dtype=np.int32) * 3
    for i in range(8):
        p[i, x[i + 1]] = 1
    p[8, 77] = 1
    parents = [i - 1 for i in range(9)]
    for levels, accepted, token in ((1, 0, 3), (4, 3, 12), (9, 8, 77), (20, 8, 77)):
        e = np.ones((1, levels, vocab), dtype=np.float32)
        got, _, t = call_verify_tree(spl, [p], [x], [parents], e)
        assert got == [accepted] and t == [token]
        check_verify_tree(spl, [p], [x], [parents], e)


def test_verify_tree_ties_take_the_first(spl):
    """Equal quotients, and equal children: the lowest token and the first child."""
    vocab = 3000
    p, e = np.ones((4, vocab), dtype=np.float32), np.ones((1, 3, vocab), dtype=np.float32)
    got = call_verify_tree(spl, [p], [np.array([5, 0, 0, 9])], [[-1, 0, 0, 1]], e)
    assert got == ([1], [[1, -1, -1]], [0])
    p[0, :] = np.nan
    assert call_verify_tree(spl, [p], [np.array([5, 0, 0, 9])], [[-1, 0, 0, 1]], e) == ([0], [[-1, -1, -1]], [-1])


def test_verify_tree_parents_out_of_range_are_nobodys_children(spl):
    vocab = 64
    p, e = np.ones((5, vocab), dtype=np.float32), np.ones((1, 4, vocab), dtype=np.float32)
    got = call_verify_tree(spl, [p], [np.array([0, 0, 0, 0, 0])], [[-1, -7, 99, 4, 2 ** 31 - 1]], e)
    assert got[0] == [0] and got[2] == [0]


@pytest.mark.parametrize("pad", [0, 1, 4])
def test_verify_tree_rows_at_any_distance(spl, pad):
    """Rows that are not 16-byte aligned take another path with the same result."""
    p, x, parents, e = tree_draws(5, [9, 30, 4], 1003, 5)
    P = torch.full((43, 1003 + pad), 9.0, device=DEV)
    P[:, :1003] = torch.as_tensor(np.concatenate(p)).to(DEV)
    E = torch.full((15, 1008 + pad), 9.0, device=DEV)
    E[:, :1003] = torch.as_tensor(e.reshape(-1, 1003)).to(DEV)
    check_verify_tree(spl, p, x, parents, e, P=P[:, :1003], E=E[:, :1003])


def test_verify_tree_as_many_sequences_as_there_may_be(spl):
    p, x, parents, e = tree_draws(6, [2] * 4096, 40, 2)
    assert sum(check_verify_tree(spl, p, x, parents, e)) > 1000


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("heads", [(2, 2, 64), (8, 8, 128), (9, 3, 64)], ids=str)
def test_keep_path_moves_the_rows_exactly(spl, heads, fmt):
    """Paths of trees across pages' ends; what is not on a path, and what stays, keeps its bits."""
    seqs = [(9, 40), (20, 20), (1, 33), (0, 17), (33, 100), (6, 2)]
    paths = [[2, 5, 8], [1, 2, 3, 19], [], [], [7, 9, 10, 20, 21, 22, 32], []]
    c = Case(spl, seqs, heads, fmt, 16, seed=9)
    c.fill()
    score = torch.rand(c.cache.k.shape[:3], device=DEV)
    tensors = [t for t in (c.cache.k, c.cache.v, c.cache.k_scale, c.cache.v_scale, score) if t is not None]
    want = [t.clone() for t in tensors]
    for b, (r, n) in enumerate(seqs):
        for i, node in enumerate(paths[b]):
            place = lambda pos: (int(c.table[b, pos // 16]), slice(None), pos % 16)  # noqa: E731, B023
            for t in want:
                t[place(n - r + 1 + i)] = t[place(n - r + node)].clone()
    path = i32([p + [-1] * (8 - len(p)) for p in paths])
    spl.spl_kv_keep_path(c.cache, c.batch(), path, i32([len(p) for p in paths]), score=score)
    for got, t in zip(tensors, want):
        assert torch.equal(raw(got), raw(t))
    assert spl.spl_get_device_status() == spl.SPL_OK


def test_keep_path_of_what_is_no_path(spl):
    """Nodes outside the rows, or not ascending, and counts outside the levels: reported; the rows before them move."""
    c = Case(spl, [(6, 30), (6, 30), (6, 30), (6, 30)], (2, 2, 64), "f16", 16, seed=9)
    c.fill()
    want = bits(c.cache.k).clone()
    for b, node in ((0, 3), (3, 2)):  # path[0] of the first and the last
        want[c.table[b, 25 // 16], :, 25 % 16] = want[c.table[b, (24 + node) // 16], :, (24 + node) % 16]
    path = i32([[3, 6, -1], [-1, 2, 3], [2, 3, 4], [2, 2, 5]])
    spl.spl_kv_keep_path(c.cache, c.batch(), path, i32([2, 3, 4, 3]))
    assert spl.spl_get_device_status() == spl.SPL_EINVAL
    assert torch.equal(bits(c.cache.k), want)


# ---------------------------------------------------------------------------------- weights
def scores_for(c, fill=float("nan")):
    return torch.full(tuple(c.cache.k.shape[:3]), fill, device=DEV)


def few(c):
    """The case with a bound on a chunk's rows that sends the call to the kernel for few rows, however many there are."""
    batch = c.batch

    def bounded(all_rows=False):
        b = batch(all_rows)
        return c.spl.KVBatch(b.row_start, b.kv_len, b.page_table, b.rows, 1)
    c.batch = bounded
    return c


KERNELS = pytest.mark.parametrize("kernel", [few, many], ids=["few", "many"])


def score_of(c, score, b):
    """[kv_heads, tokens] of sequence b."""
    n = c.seqs[b][1]
    j = np.arange(n)
    return score.cpu().numpy()[c.table[b, j // c.page], :, j % c.page].T


def weight_tolerance(q, k, scale, group, rows_of):
    """Of a weight p, relative: twice a score's error (see test_gpu_serving.tolerance) and an exp's 2^-21 for the term and
    the total, roundings of the product and the sums (one for each row and head that adds)."""
    dim = q.shape[-1]
    size = abs(scale) * np.max(np.einsum("ihd,jhd->ihj", np.abs(q).astype(np.float64),
                                         np.repeat(np.abs(k).astype(np.float64), group, axis=1)), initial=0.0)
    score = (2.0 ** -22 + dim / 8 * 2.0 ** -23 + 4 * U) * size
    return 2 * (score + 2.0 ** -21) + (rows_of + len(k) / 32 + 8) * U


def check_weights(c, window=0, scale=None, decay=1.0, before=0.75, batch=None, **kw):
    score = scores_for(c, before)
    q = torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV)
    c.spl.spl_kv_weigh(score, q, c.cache, batch or c.batch(), c.hq, scale=scale, window=window, decay=decay, **kw)
    torch.cuda.synchronize()
    s = 1.0 / np.sqrt(c.d) if scale is None else scale
    group = c.hq // c.hk
    for b, (r, n) in enumerate(c.seqs):
        q, k = c.q[c.start[b]:c.start[b + 1]], c.stored("k", b)
        added = serving.weights(q, k, n, group, s, window)
        kept = np.float32(before) * np.float32(decay) * (np.arange(n) < n - r)
        got = score_of(c, score, b)
        tol = weight_tolerance(q, k, s, group, r * group) * added + 2 * U * (kept + added) + 1e-30
        err = np.abs(got - (kept + added))
        assert np.all(err <= tol), f"sequence {b} {r, n}: worst err/tol {np.max(err / tol):.3g}"
    used = np.zeros(tuple(c.cache.k.shape[:3]), dtype=bool)
    for b, (_, n) in enumerate(c.seqs):
        j = np.arange(n)
        used[c.table[b, j // c.page], :, j % c.page] = True
    left = score.cpu().numpy()[~used]
    assert np.all(left == before), "a slot of no token was written"
    assert c.spl.spl_get_device_status() == c.spl.SPL_OK
    return score


WEIGHS = {"one": [(1, 1)], "odd": [(1, 299)], "ragged": [(1, 5), (1, 1000), (0, 17), (1, 128), (0, 0), (1, 1)],
          "drafts": [(5, 261), (3, 3), (1, 700), (4, 64)], "chunks": [(37, 37), (130, 333), (1, 90), (64, 64)],
          "prompt": [(300, 300), (129, 640)]}


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("heads", [(24, 8, 128), (8, 2, 64), (3, 3, 128), (7, 1, 64), (16, 1, 128)], ids=str)
@pytest.mark.parametrize("name", WEIGHS)
@KERNELS
def test_weigh(spl, kernel, name, heads, fmt):
    c = kernel(Case(spl, WEIGHS[name], heads, fmt, 16 if name == "ragged" else 64, seed=len(name)))
    c.fill()
    check_weights(c, decay=0.5)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("page", [16, 32, 128, 256])
@pytest.mark.parametrize("window", [0, 1, 63, 129, 1000])
@KERNELS
def test_weigh_pages_and_windows(spl, kernel, page, window, fmt):
    c = kernel(Case(spl, [(3, 300), (20, 257), (1, page), (150, 150 + page)], (6, 2, 128), fmt, page, seed=page))
    c.fill()
    check_weights(c, window=window, decay=0.0)


@pytest.mark.parametrize("rows", [1, 40, 200])
@pytest.mark.parametrize("fmt", ["f16", "i8"])
@KERNELS
def test_weigh_sharp_and_flat(spl, kernel, rows, fmt):
    for std, scale in ((6.0, None), (1.0, 0.0), (1.0, -0.3), (2.0, 1.0)):
        c = kernel(Case(spl, [(rows, 777)], (4, 1, 64), fmt, 64, seed=rows, std=std))
        c.fill()
        check_weights(c, scale=scale)


@pytest.mark.parametrize("rows", [3, 140])
@pytest.mark.parametrize("fmt", ["f16", "i8"])
@KERNELS
def test_weigh_new_tokens_start_from_nothing(spl, kernel, rows, fmt):
    """What a new token's slot held, NaN or not, does not count; without rows the scores only decay; a sequence shorter
    than its rows."""
    c = kernel(Case(spl, [(rows, 200), (rows, 2), (0, 90)], (4, 2, 128), fmt, 16, seed=3))
    c.fill()
    check_weights(c, before=0.75)
    score = scores_for(c)
    q = torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV)
    spl.spl_kv_weigh(score, q, c.cache, c.batch(), c.hq)
    got = score_of(c, score, 0)
    assert np.isnan(got[:, :200 - rows]).all() and np.isfinite(got[:, 200 - rows:]).all()
    assert np.isfinite(score_of(c, score, 1)).all() and np.isnan(score_of(c, score, 2)).all()


@pytest.mark.parametrize("rows", [2, 48, 200])
@pytest.mark.parametrize("fmt", ["f16", "i8"])
@KERNELS
def test_weigh_nan_reaches_only_what_its_rows_see(spl, kernel, rows, fmt):
    """A NaN in a later token's key: rows that see it give NaN to what they see, in its head alone."""
    c = kernel(Case(spl, [(rows, 100 + rows), (1, 50)], (4, 2, 64), fmt, 16, seed=rows))
    c.k[0][100 + rows // 2, 1, 3] = np.nan
    c.fill()
    score = scores_for(c, 0.0)
    spl.spl_kv_weigh(score, torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV), c.cache, c.batch(), 4)
    got = score_of(c, score, 0)
    assert np.isfinite(got[0]).all() and np.isnan(got[1]).all()
    assert np.isfinite(score_of(c, score, 1)).all()


@KERNELS
@pytest.mark.parametrize("fmt", ["f16", "i8"])
def test_weigh_pages_outside_the_pool_and_lengths(spl, fmt, kernel):
    for rows in (1, 40, 150):
        c = kernel(Case(spl, [(rows, 200), (rows, 164)], (4, 2, 64), fmt, 16, seed=4))
        c.fill()
        q = torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV)
        c.table[0, 3], c.table[0, 6] = -5, 1 << 30
        score = scores_for(c, 0.0)
        spl.spl_kv_weigh(score, q, c.cache, c.batch(), 4)
        assert spl.spl_get_device_status() == spl.SPL_EINVAL
        there = np.array([j for j in range(200) if j // 16 not in (3, 6)])
        page = c.table[0, there // 16]
        got = score.cpu().numpy()[page, :, there % 16].T
        want = np.zeros((2, 200))
        for i in range(rows):
            keys = there[there <= 200 - rows + i]
            want[:, keys] += serving.weights(c.q[i:i + 1], c.stored("k", 0)[keys], len(keys), 2, 0.125)
        assert np.allclose(got, want[:, there], rtol=1e-5, atol=1e-12)
        batch = c.batch()
        batch.kv_len.copy_(i32([-3, 164]))
        score = scores_for(c, 0.25)
        spl.spl_kv_weigh(score, q, c.cache, batch, 4)
        assert spl.spl_get_device_status() == spl.SPL_EINVAL
        assert bool((score[torch.as_tensor(page).long().to(DEV)] == 0.25).all())
        batch.kv_len.copy_(i32([1 << 30, 164]))
        spl.spl_kv_weigh(score, q, c.cache, batch, 4)
        assert spl.spl_get_device_status() == spl.SPL_EINVAL


@pytest.mark.parametrize("rows", [1, 90, 260])
def test_weigh_is_deterministic_in_graphs_and_on_streams(spl, rows):
    """The same bits again; a captured call follows the lengths; calls follow their stream."""
    c = Case(spl, [(rows, 900), (rows, 1500)], (8, 2, 128), "f16", 64, seed=1)
    c.fill()
    first = check_weights(c)
    q = torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV)
    batch = c.batch()
    ws = spl.workspace(spl.spl_kv_weigh_workspace_bytes(c.cache, batch, c.hq))
    score = scores_for(c, 0.75)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(10_000_000)
        late = q.clone()
        spl.spl_kv_weigh(score, late, c.cache, batch, 8, workspace=ws)
    s.synchronize()
    assert torch.equal(score, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spl.spl_kv_weigh(score, q, c.cache, batch, 8, workspace=ws)
    ws.fill_(255)  # any contents, and the counters' place is not touched
    for lens in ([900, 1500], [rows, rows + 400], [900, 0]):
        batch.kv_len.copy_(i32(lens))
        score.fill_(0.75)
        graph.replay()
        torch.cuda.synchronize()
        for b, n in enumerate(lens):
            added = serving.weights(c.q[c.start[b]:c.start[b + 1]], c.stored("k", b)[:n], n, 4, 128 ** -0.5)
            got = score_of(c, score, b)[:, :n]
            want = added + 0.75 * (np.arange(n) < n - rows)
            assert np.allclose(got, want, rtol=1e-5, atol=0)
    assert spl.spl_get_device_status() == spl.SPL_OK
    assert bool((ws[:65536] == 255).all())


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("scale", [None, 0.0, -0.25, 3.0], ids=str)
@pytest.mark.parametrize("heads", [(8, 2, 128), (7, 1, 64)], ids=str)
@KERNELS
def test_weigh_rows_of_any_size(spl, kernel, heads, scale, fmt):
    """Rows that differ by powers of two, by far, or are zero: each keeps its own precision."""
    c = kernel(Case(spl, [(200, 600), (40, 40), (33, 500)], heads, fmt, 32, seed=8))
    c.fill()
    g = np.random.default_rng(9)
    for b, sizes in enumerate(([0, -1, -6, -12, -13, -40], [0], [-200, -2])):
        rows = slice(c.start[b], c.start[b + 1])
        c.q[rows] = np.ldexp(c.q[rows], g.choice(sizes, size=c.q[rows].shape[:2])[..., None])
        c.q[rows][g.random(c.q[rows].shape[:2]) < 0.05] = 0.0
    check_weights(c, scale=scale, decay=0.5)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), 3e38], ids=str)
@pytest.mark.parametrize("fmt", ["f16", "i8"])
@KERNELS
def test_weigh_rows_of_other_sequences(spl, kernel, fmt, value):
    """What the rows next to a sequence's are does not reach it, to the bit."""
    c = kernel(Case(spl, [(100, 700), (150, 300), (40, 900)], (4, 2, 64), fmt, 32, seed=10))
    c.fill()
    want = [score_of(c, check_weights(c), b) for b in (0, 2)]
    q = torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV)
    q[c.start[1]:c.start[2]] = value
    score = scores_for(c, 0.75)
    spl.spl_kv_weigh(score, q, c.cache, c.batch(), c.hq)
    for b, was in zip((0, 2), want):
        assert np.array_equal(score_of(c, score, b), was)
    assert spl.spl_get_device_status() == spl.SPL_OK


# Few heads and many rows: the rows of a key are shared out, and the last of their parts to end adds all up.  Tolerance: a sum's
# additions, one a part and half more, are no more than its rows.
PARTS = {"one": [(1500, 1600)], "itself": [(700, 700)], "past": [(600, 3000)],
         "ragged": [(700, 900), (0, 5), (1, 1300), (260, 260), (0, 0)]}


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("window", [0, 300])
@pytest.mark.parametrize("heads", [(7, 1, 64), (14, 2, 64), (4, 1, 128), (1, 1, 128)], ids=str)
@pytest.mark.parametrize("name", PARTS)
def test_weigh_rows_in_parts(spl, name, heads, window, fmt):
    c = many(Case(spl, PARTS[name], heads, fmt, 32, seed=len(name)))
    c.fill()
    check_weights(c, window=window, decay=0.5)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
def test_weigh_rows_in_parts_again(spl, fmt):
    """The same bits whichever part ends last, over any contents of the workspace; two graphs on one workspace; a replayed call
    after the lengths have changed, where a part may have no rows."""
    c = many(Case(spl, [(900, 1000), (300, 2000)], (4, 1, 64), fmt, 32, seed=3))
    c.fill()
    first = check_weights(c)
    q = torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV)
    batch = c.batch()
    ws = spl.workspace(spl.spl_kv_weigh_workspace_bytes(c.cache, batch, c.hq))
    score = scores_for(c, 0.75)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            spl.spl_kv_weigh(score, q, c.cache, batch, c.hq, workspace=ws)
    for turn in range(20):
        if turn % 5 == 0:
            ws.fill_(255)
        score.fill_(0.75)
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(raw(score), raw(first))
    for lens in ([900, 300], [900, 0], [0, 300], [1000, 300]):
        batch.kv_len.copy_(i32(lens))
        score.fill_(0.75)
        graphs[0].replay()
        torch.cuda.synchronize()
        for b, (n, rows) in enumerate(zip(lens, (900, 300))):
            own = c.q[c.start[b]:c.start[b + 1]]
            k = c.stored("k", b)[:n]
            added = serving.weights(own, k, n, 4, 64 ** -0.5) if n else np.zeros((1, 0))
            kept = 0.75 * (np.arange(n) < n - rows)
            tol = weight_tolerance(own, k, 64 ** -0.5, 4, rows * 4) * added + 2 * U * (kept + added) + 1e-30
            assert np.all(np.abs(score_of(c, score, b)[:, :n] - (kept + added)) <= tol)
    assert spl.spl_get_device_status() == spl.SPL_OK


# ---------------------------------------------------------------------------------- eviction
def check_evict(c, score, keep, recent, fresh=False, alias=False):
    """Against the definition, to the bit; scores [pages, heads, page] on the device."""
    spl, page = c.spl, c.page
    before = {n: t.clone() for n, t in (("k", c.cache.k), ("v", c.cache.v), ("ks", c.cache.k_scale), ("vs", c.cache.v_scale),
                                        ("score", score)) if t is not None}
    batch = c.batch()
    table = c.table
    if fresh:  # pages that no sequence has
        taken = set(int(p) for b, (_, n) in enumerate(c.seqs) for p in c.table[b, :-(-n // page)])
        free = [p for p in range(c.cache.pages) if p not in taken]
        table = np.full_like(c.table, c.cache.pages + 3)
        for b, (_, n) in enumerate(c.seqs):
            for i in range(-(-min(n, keep) // page)):
                table[b, i] = free.pop()
    out_len = batch.kv_len if alias else i32([-1] * len(c.seqs))
    spl.spl_kv_evict(c.cache, score, batch, keep, recent, out_len, out_table=torch.as_tensor(table).to(DEV) if fresh else None)
    assert spl.spl_get_device_status() == spl.SPL_OK
    assert out_len.tolist() == [min(n, keep) for _, n in c.seqs]
    after = {"k": c.cache.k, "v": c.cache.v, "ks": c.cache.k_scale, "vs": c.cache.v_scale, "score": score}
    old = before["score"].cpu().numpy()
    moves = []
    for b, (_, n) in enumerate(c.seqs):
        j = np.arange(n)
        for h in range(c.hk):
            stay = np.array(serving.evict(old[c.table[b, j // page], h, j % page], keep, recent), dtype=np.int64)
            to = np.arange(len(stay))
            moves.append((c.table[b, stay // page], h, stay % page, table[b, to // page], to % page))
    source = [np.concatenate([np.broadcast_to(m[i], m[0].shape) for m in moves]) for i in (0, 1, 2)]
    target = [np.concatenate([np.broadcast_to(m[i], m[0].shape) for m in moves]) for i in (3, 1, 4)]
    source, target = (tuple(torch.as_tensor(np.ascontiguousarray(i)).long().to(DEV) for i in w) for w in (source, target))
    for name, t in before.items():
        want = t.clone()
        want[target] = t[source]
        got = after[name]
        assert torch.equal(raw(got), raw(want)), name


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("heads", [(8, 8, 128), (2, 2, 64), (9, 9, 64)], ids=str)
@pytest.mark.parametrize("keep,recent", [(0, 0), (1, 0), (1, 1), (16, 5), (100, 0), (100, 100), (257, 31), (999, 500), (5000, 9)])
def test_evict(spl, keep, recent, heads, fmt):
    g = np.random.default_rng(keep + recent)
    for fresh in (False, True):
        c = Case(spl, [(1, 1000), (0, 100), (0, 0), (1, 1), (5, 258), (1, 4100)], heads, fmt, 16, seed=keep, spare=400)
        c.fill()
        score = torch.as_tensor(g.exponential(size=tuple(c.cache.k.shape[:3])).astype(np.float32)).to(DEV)
        check_evict(c, score, keep, recent, fresh, alias=keep == 16)


@pytest.mark.parametrize("page", [16, 64, 256])
def test_evict_ties_and_special_scores(spl, page):
    """Few different scores, both zeros, denormal, infinite, negative and NaN ones: the earliest of equals, NaN last."""
    g = np.random.default_rng(page)
    values = np.array([0.0, -0.0, 1.0, 1.0000001, np.inf, -np.inf, np.nan, -1.0, 1e-42, 2.0], dtype=np.float32)
    for pool in (values, values[:2], values[6:7], values[2:4]):
        for keep, recent in ((700, 10), (64, 64), (33, 0)):
            c = Case(spl, [(1, 1500), (1, 701)], (2, 2, 64), "f16", page, seed=page)
            c.fill()
            score = torch.as_tensor(g.choice(pool, tuple(c.cache.k.shape[:3]))).to(DEV)
            check_evict(c, score, keep, recent)


@pytest.mark.parametrize("early", [24575, 24576, 24577, 30000, 60001])
def test_evict_lengths_around_what_shared_memory_holds(spl, early):
    g = np.random.default_rng(early)
    c = Case(spl, [(1, early + 100)], (2, 2, 64), "i8", 64, seed=1)
    c.fill()
    score = torch.as_tensor(np.round(g.exponential(size=tuple(c.cache.k.shape[:3])) * 1000).astype(np.float32)).to(DEV)
    check_evict(c, score, early // 2, 100)


def test_evict_again_and_again(spl):
    """A sequence that is cut, grows and is cut again: positions count from the front each time."""
    c = Case(spl, [(1, 400), (1, 300)], (4, 4, 64), "f16", 16, seed=5)
    c.fill()
    g = np.random.default_rng(1)
    for keep in (350, 200, 64):
        score = torch.as_tensor(g.random(tuple(c.cache.k.shape[:3])).astype(np.float32)).to(DEV)
        check_evict(c, score, keep, 16)
        c.seqs = [(1, min(n, keep)) for _, n in c.seqs]


def test_evict_pages_outside_the_pool_and_lengths(spl):
    c = Case(spl, [(1, 200), (1, 150)], (2, 2, 64), "f16", 16, seed=5)
    c.fill()
    score = torch.rand(tuple(c.cache.k.shape[:3]), device=DEV) + 1.0
    batch = c.batch()
    batch.page_table[0, 2] = -1
    before = c.cache.k.clone()
    out = i32([7, 7])
    spl.spl_kv_evict(c.cache, score, batch, 150, 10, out)
    assert spl.spl_get_device_status() == spl.SPL_EINVAL
    assert out.tolist() == [150, 150]
    other = torch.as_tensor(c.table[1, :10]).long().to(DEV)
    assert torch.equal(bits(c.cache.k[other]), bits(before[other]))
    batch = c.batch()
    for n, want in ((-5, 0), (1 << 30, 100)):
        batch.kv_len.copy_(i32([150, n]))
        spl.spl_kv_evict(c.cache, score, batch, 100, 10, out)
        assert spl.spl_get_device_status() == spl.SPL_EINVAL and out.tolist() == [100, want]


# ---------------------------------------------------------------------------------- together
@pytest.mark.parametrize("fmt", ["f16", "i8"])
def test_a_step_over_a_bounded_cache(spl, fmt):
    """Append a tree, attend, verify, keep the path, weigh the kept rows, evict: what the cache then holds are the tokens
    that the definitions keep, and attention over it is that of those tokens."""
    g = np.random.default_rng(11)
    seqs = [(10, 70), (10, 45), (10, 30)]
    c = Case(spl, seqs, (4, 2, 64), fmt, 16, seed=12)
    c.fill()
    parents = [random_tree(g, 10) for _ in seqs]
    masks = [masks_of(p) for p in parents]
    check_tree(c, masks)
    p, x, _, e = tree_draws(13, [10] * 3, 300, 6)
    for b in range(3):  # the same trees for the target's probabilities
        p[b] = np.full((10, 300), 1e-3, dtype=np.float32)
        for i in range(1, 10):
            p[b][parents[b][i], x[b][i]] += 1.0
    accepted, path, _ = call_verify_tree(spl, p, x, parents, e)
    spl.spl_kv_keep_path(c.cache, c.batch(), i32(path), i32(accepted))
    stay, lens = [], []
    for b, (r, n) in enumerate(seqs):
        stay.append(list(range(n - r + 1)) + [n - r + i for i in path[b][:accepted[b]]])
        lens.append(len(stay[b]))
        c.k[b], c.v[b] = c.k[b][stay[b]], c.v[b][stay[b]]
    rows = [a + 1 for a in accepted]
    c.q = np.concatenate([c.q[[c.start[b]] + [c.start[b] + i for i in path[b][:accepted[b]]]] for b in range(3)])
    c.seqs, c.rows = list(zip(rows, lens)), sum(rows)
    c.start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    score = check_weights(c)
    keep = 32
    check_evict(c, score.clone(), keep, 8)
    assert spl.spl_get_device_status() == spl.SPL_OK


def test_one_workspace_for_all(spl):
    """Attention, weights and eviction in turn on one workspace, with a product's and graphs': the same bits every time, and
    the arrival counters stay zero."""
    a = Case(spl, [(1, 900), (1, 1500)], (8, 2, 128), "f16", 64, seed=1)
    b = many(Case(spl, [(130, 500), (60, 700)], (4, 2, 64), "i8", 16, seed=2))
    for c in (a, b):
        c.fill()
    keep = 400
    ws = spl.workspace(max(max(spl.spl_paged_attention_workspace_bytes(c.cache, c.batch(), c.hq),
                               spl.spl_kv_weigh_workspace_bytes(c.cache, c.batch(), c.hq),
                               spl.spl_kv_evict_workspace_bytes(c.cache, c.batch(), keep)) for c in (a, b)))
    qs = [torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV) for c in (a, b)]
    batches = [c.batch() for c in (a, b)]
    outs = [torch.empty_like(q) for q in qs]
    scores = [scores_for(c) for c in (a, b)]
    lens = [i32([0, 0]) for _ in range(2)]

    def step(i, c):
        scores[i].fill_(0.5)
        spl.spl_paged_attention(outs[i], qs[i], c.cache, batches[i], c.hq, workspace=ws)
        spl.spl_kv_weigh(scores[i], qs[i], c.cache, batches[i], c.hq, workspace=ws)
        return outs[i], scores[i]

    want = []
    for i, c in enumerate((a, b)):
        want.append([t.clone() for t in step(i, c)])
    graphs = []
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for i, c in enumerate((a, b)):
            step(i, c)
    s.synchronize()
    for i, c in enumerate((a, b)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(i, c)
    for turn in range(3):
        for i in (0, 1, 1, 0):
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want[i][0]) and torch.equal(raw(scores[i]), raw(want[i][1]))
    for i, c in enumerate((a, b)):  # (moves the caches' tokens: last)
        spl.spl_kv_evict(c.cache, scores[i], batches[i], keep, 16, lens[i], workspace=ws)
        assert lens[i].tolist() == [keep, keep]
    assert int(ws[:65536].count_nonzero()) == 0
    assert spl.spl_get_device_status() == spl.SPL_OK


@pytest.mark.parametrize("fmt", ["f16", "i8"])
def test_offsets_past_32_bits(spl, fmt):
    """Tokens on the last pages of a pool of more than 4 GB of keys: the bits of a small pool's."""
    seqs, heads, page = [(20, 300), (1, 150), (40, 90)], (4, 2, 64), 256
    small = Case(spl, seqs, heads, fmt, page, seed=21)
    small.fill()
    big = Case(spl, seqs, heads, fmt, page, seed=21)
    pages = (9 << 28) // (2 * page * 64)  # 2.4e9 elements
    big.cache = spl.KVCache.empty(pages, 2, 64, page, fmt)
    big.poison()
    big.table = np.where(big.table < small.cache.pages, big.table + pages - small.cache.pages, pages + 7).astype(np.int32)
    big.fill()
    last = slice(pages - small.cache.pages, pages)
    g = np.random.default_rng(2)
    masks = [masks_of(random_tree(g, r)) for r, _ in seqs]
    score = torch.rand(tuple(small.cache.k.shape[:3]), device=DEV)
    wide = torch.empty(tuple(big.cache.k.shape[:3]), device=DEV)
    wide[last] = score
    q = torch.as_tensor(small.q.reshape(small.rows, -1)).to(DEV)
    for kernel in (few, many):
        assert np.array_equal(attend_tree(kernel(small), masks, 2), attend_tree(kernel(big), masks, 2))
        spl.spl_kv_weigh(score, q, small.cache, small.batch(), 4)
        spl.spl_kv_weigh(wide, q, big.cache, big.batch(), 4)
        assert torch.equal(raw(wide[last]), raw(score))
    path, accepted, lens = i32([[1, 4, 9], [-1, -1, -1], [3, 7, 39]]), i32([3, 0, 3]), i32([0, 0, 0])
    for c, sc in ((small, score), (big, wide)):
        spl.spl_kv_keep_path(c.cache, c.batch(), path, accepted, score=sc)
        spl.spl_kv_evict(c.cache, sc, c.batch(), 100, 10, lens)
    used = sorted(set(int(p) for b, (_, n) in enumerate(seqs) for p in small.table[b, :-(-n // page)]))
    for name in ("k", "v", "k_scale", "v_scale"):
        x, y = getattr(small.cache, name), getattr(big.cache, name)
        if x is not None:
            assert torch.equal(raw(y[last][used]), raw(x[used])), name
    assert torch.equal(raw(wide[last][used]), raw(score[used]))
    assert spl.spl_get_device_status() == spl.SPL_OK
    del big, wide
    torch.cuda.empty_cache()


def test_decisions_follow_their_stream(spl):
    """Probabilities and trees made on a stream that is still busy, an eviction and a path behind them in a graph."""
    p, x, parents, e = tree_draws(8, [12, 5], 5003, 5)
    want = [serving.verify_tree(p[b], x[b], parents[b], e[b]) for b in range(2)]
    c = Case(spl, [(12, 60), (5, 40)], (2, 2, 64), "f16", 16, seed=3)
    c.fill()
    before = c.cache.k.clone()
    flat = lambda parts, t: torch.as_tensor(np.concatenate(parts).astype(t)).to(DEV)  # noqa: E731
    P, E, X, up = flat(p, np.float32), torch.as_tensor(e.reshape(-1, 5003)).to(DEV), flat(x, np.int32), flat(parents, np.int32)
    accepted, token, path = i32([0, 0]), i32([0, 0]), i32([[0] * 5] * 2)
    batch, s = c.batch(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        late = P.clone()
        spl.spl_verify_tree(accepted, path, token, late, X, up, E, batch.row_start)
        spl.spl_kv_keep_path(c.cache, batch, path, accepted)
    s.synchronize()
    assert accepted.tolist() == [len(w) for w, _ in want] and token.tolist() == [t for _, t in want]
    moved = c.cache.k.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spl.spl_verify_tree(accepted, path, token, P, X, up, E, batch.row_start)
        spl.spl_kv_keep_path(c.cache, batch, path, accepted)
    for _ in range(2):
        c.cache.k.copy_(before)
        accepted.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(raw(c.cache.k), raw(moved)) and accepted.tolist() == [len(w) for w, _ in want]
    assert spl.spl_get_device_status() == spl.SPL_OK


@pytest.mark.parametrize("fmt", ["f16", "i8"])
def test_rows_behind_the_last_sequence(spl, fmt):
    """A padded batch: rows of no sequence, NaN in theirs, are left as they were and reach nobody."""
    g = np.random.default_rng(3)
    for kernel in (few, many):
        c = kernel(Case(spl, [(9, 200), (40, 90), (0, 33)], (4, 2, 128), fmt, 16, seed=14))
        c.fill()
        masks = [masks_of(random_tree(g, r)) for r, _ in c.seqs]
        want, score = attend_tree(c, masks, 2), check_weights(c)
        extra, batch = 13, c.batch()
        padded = spl.KVBatch(batch.row_start, batch.kv_len, batch.page_table, c.rows + extra, 1 if kernel is few else 1 << 24)
        q = torch.full((c.rows + extra, 4 * 128), float("nan"), device=DEV)
        q[:c.rows] = torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV)
        seen = torch.full((c.rows + extra, 2), -1, dtype=torch.int32, device=DEV)
        seen[:c.rows] = words_of(sum(masks, []), 2)
        out = torch.full_like(q, 7.0)
        spl.spl_tree_attention(out, q, c.cache, padded, seen, 4)
        assert np.array_equal(out[:c.rows].cpu().numpy().reshape(want.shape), want) and bool((out[c.rows:] == 7.0).all())
        again = scores_for(c, 0.75)
        spl.spl_kv_weigh(again, q, c.cache, padded, 4)
        assert torch.equal(raw(again), raw(score))
        assert spl.spl_get_device_status() == spl.SPL_OK


@pytest.mark.parametrize("kernel", [few, many], ids=["few", "many"])
def test_weigh_as_many_sequences_as_there_may_be(spl, kernel):
    g = np.random.default_rng(7)
    seqs = [(int(r), int(r + n)) for r, n in zip(g.integers(0, 3, 4096), g.integers(0, 40, 4096))]
    seqs[0] = seqs[-1] = (40, 300)
    c = kernel(Case(spl, seqs, (4, 2, 64), "f16", 16, seed=7))
    c.fill()
    check_weights(c, decay=0.5)


def test_evict_as_many_sequences_as_there_may_be(spl):
    g = np.random.default_rng(8)
    seqs = [(0, int(n)) for n in g.integers(0, 60, 4096)]
    c = Case(spl, seqs, (2, 2, 64), "i8", 16, seed=8)
    c.fill()
    score = torch.as_tensor(g.random(tuple(c.cache.k.shape[:3])).astype(np.float32)).to(DEV)
    check_evict(c, score, 20, 4, alias=True)
