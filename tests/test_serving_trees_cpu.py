"""Refusals and empty calls of tree attention, tree verification, attention weights and eviction, which need no GPU, and the
oracle against closed forms."""

import ctypes

import numpy as np
import pytest

from oracle import serving
from test_serving_cpu import BATCHES, CACHES, base, batch_of, cache_of, shifted, spl  # noqa: F401


def every(spl, cache, batch, p):  # noqa: F811
    """The operators' answers to one cache and batch."""
    L = spl.lib()
    c, b = (ctypes.byref(x) if x is not None else None for x in (cache, batch))
    return (L.spl_tree_attention(p, 256, p, 256, c, b, p, 1, 2, 4, 1.0, 0, p, 1 << 40, None),
            L.spl_kv_weigh(p, p, 256, c, b, 2, 4, 1.0, 0, 1.0, p, 1 << 40, None),
            L.spl_kv_evict(c, p, b, 4, 2, None, p, p, 1 << 40, None),
            L.spl_kv_keep_path(c, p, b, 2, p, 2, p, 2, None))


@pytest.mark.parametrize("fields,error", CACHES, ids=str)
def test_caches_that_are_refused(spl, base, fields, error):  # noqa: F811
    want = getattr(spl, "SPL_" + error)
    assert every(spl, cache_of(spl, base, **shifted(fields, base)), batch_of(spl, base), base) == (want,) * 4


@pytest.mark.parametrize("fields,error", BATCHES, ids=str)
def test_batches_that_are_refused(spl, base, fields, error):  # noqa: F811
    want = getattr(spl, "SPL_" + error)
    assert every(spl, cache_of(spl, base), batch_of(spl, base, **shifted(fields, base)), base) == (want,) * 4


def test_null_structs_and_empty_calls(spl, base):  # noqa: F811
    L, c, b = spl.lib(), cache_of(spl, base), batch_of(spl, base)
    assert every(spl, None, b, base) == (spl.SPL_EINVAL,) * 4
    assert every(spl, c, None, base) == (spl.SPL_EINVAL,) * 4
    c, b, none = ctypes.byref(c), ctypes.byref(b), ctypes.byref(batch_of(spl, None, seqs=0, max_pages=0))
    for batch, rows in ((b, 0), (none, 0)):
        assert L.spl_tree_attention(None, 0, None, 0, c, batch, None, 0, rows, 4, 1.0, 0, None, 0, None) == spl.SPL_OK
        assert L.spl_kv_keep_path(c, None, batch, rows, None, 0, None, 3, None) == spl.SPL_OK
    assert L.spl_kv_weigh(None, None, 0, c, none, 0, 4, 1.0, 0, 1.0, None, 0, None) == spl.SPL_OK
    assert L.spl_kv_evict(c, None, none, 4, 2, None, None, None, 0, None) == spl.SPL_OK
    assert L.spl_kv_keep_path(c, None, b, 2, None, 0, None, 0, None) == spl.SPL_OK
    assert L.spl_verify_tree(*[None] * 2, 0, None, None, 0, None, None, None, 0, None, 0, 0, 1, 9, None) == spl.SPL_OK


def test_tree_attention_that_is_refused(spl, base):  # noqa: F811
    L, c, b = spl.lib(), ctypes.byref(cache_of(spl, base)), ctypes.byref(batch_of(spl, base))
    good = dict(out=base, ldo=256, Q=base, ldq=256, seen=base, words=1, rows=2, heads=4, scale=1.0, window=0, ws=base,
                size=1 << 40)

    def call(**kw):
        a = {**good, **kw}
        return L.spl_tree_attention(a["out"], a["ldo"], a["Q"], a["ldq"], c, b, a["seen"], a["words"], a["rows"], a["heads"],
                                    a["scale"], a["window"], a["ws"], a["size"], None)
    for kw in ({"out": None}, {"Q": None}, {"seen": None}, {"words": -1}, {"ldo": 252}, {"ldq": -256}, {"rows": -1},
               {"heads": 3}, {"heads": 0}, {"scale": float("nan")}, {"scale": float("inf")}, {"window": -1}):
        assert call(**kw) == spl.SPL_EINVAL, kw
    for kw in ({"rows": 1 << 60}, {"rows": 1 << 31}, {"heads": 2 * 1025}):
        assert call(**kw) == spl.SPL_ESHAPE, kw
    for kw in ({"out": base + 4}, {"Q": base + 8}, {"seen": base + 2}, {"ldo": 258}, {"ldq": 257}, {"ws": base + 8}):
        assert call(**kw) == spl.SPL_EALIGN, kw
    need = L.spl_paged_attention_workspace_bytes(c, b, 2, 4)
    assert call(size=need - 1) == spl.SPL_EWORKSPACE and call(ws=None) == spl.SPL_EWORKSPACE


def test_weights_that_are_refused(spl, base):  # noqa: F811
    L, c, b = spl.lib(), ctypes.byref(cache_of(spl, base)), ctypes.byref(batch_of(spl, base))
    good = dict(score=base, Q=base, ldq=256, rows=2, heads=4, scale=1.0, window=0, decay=1.0, ws=base, size=1 << 40)

    def call(**kw):
        a = {**good, **kw}
        return L.spl_kv_weigh(a["score"], a["Q"], a["ldq"], c, b, a["rows"], a["heads"], a["scale"], a["window"], a["decay"],
                              a["ws"], a["size"], None)
    for kw in ({"score": None}, {"Q": None}, {"ldq": 252}, {"ldq": -4}, {"rows": -1}, {"heads": 3}, {"heads": 0},
               {"scale": float("nan")}, {"window": -1}, {"decay": -0.1}, {"decay": 1.5}, {"decay": float("nan")}):
        assert call(**kw) == spl.SPL_EINVAL, kw
    for kw in ({"rows": 1 << 60}, {"rows": 1 << 31}, {"heads": 2 * 1025}):
        assert call(**kw) == spl.SPL_ESHAPE, kw
    for kw in ({"score": base + 2}, {"Q": base + 8}, {"ldq": 257}, {"ws": base + 8}):
        assert call(**kw) == spl.SPL_EALIGN, kw
    need = L.spl_kv_weigh_workspace_bytes(c, b, 2, 4)
    assert need > 0 and call(size=need - 1) == spl.SPL_EWORKSPACE and call(ws=None) == spl.SPL_EWORKSPACE
    assert L.spl_kv_weigh_workspace_bytes(c, b, 2, 3) == 0


def test_evictions_that_are_refused(spl, base):  # noqa: F811
    L, c, b = spl.lib(), ctypes.byref(cache_of(spl, base)), ctypes.byref(batch_of(spl, base))
    good = dict(score=base, keep=8, recent=2, table=None, out=base, ws=base, size=1 << 40)

    def call(**kw):
        a = {**good, **kw}
        return L.spl_kv_evict(c, a["score"], b, a["keep"], a["recent"], a["table"], a["out"], a["ws"], a["size"], None)
    for kw in ({"score": None}, {"out": None}, {"keep": -1}, {"recent": -1}, {"recent": 9}):
        assert call(**kw) == spl.SPL_EINVAL, kw
    for kw in ({"score": base + 2}, {"out": base + 1}, {"table": base + 2}, {"ws": base + 8}):
        assert call(**kw) == spl.SPL_EALIGN, kw
    need = L.spl_kv_evict_workspace_bytes(c, b, 8)
    assert need > 0 and call(size=need - 1) == spl.SPL_EWORKSPACE and call(ws=None) == spl.SPL_EWORKSPACE
    assert L.spl_kv_evict_workspace_bytes(c, b, -1) == 0
    # no more places than the table has room for
    assert L.spl_kv_evict_workspace_bytes(c, b, 1 << 60) == L.spl_kv_evict_workspace_bytes(c, b, 32)


def test_paths_that_are_refused(spl, base):  # noqa: F811
    L, c, b = spl.lib(), ctypes.byref(cache_of(spl, base)), ctypes.byref(batch_of(spl, base))
    call = lambda score=base, rows=2, path=base, ld=3, accepted=base, levels=3: L.spl_kv_keep_path(  # noqa: E731
        c, score, b, rows, path, ld, accepted, levels, None)
    for kw in ({"path": None}, {"accepted": None}, {"ld": 2}, {"ld": -3}, {"levels": -1}, {"rows": -1}):
        assert call(**kw) == spl.SPL_EINVAL, kw
    for kw in ({"rows": 1 << 31}, {"levels": 1 << 31, "ld": 1 << 32}):
        assert call(**kw) == spl.SPL_ESHAPE, kw
    for kw in ({"score": base + 1}, {"path": base + 2}, {"accepted": base + 3}):
        assert call(**kw) == spl.SPL_EALIGN, kw


def test_tree_verification_that_is_refused(spl, base):  # noqa: F811
    L = spl.lib()
    names = "accepted path ldpath token P ldp x parent e lde row_start rows seqs levels vocab".split()
    good = dict(zip(names, (base, base, 4, base, base, 8, base, base, base, 8, base, 3, 2, 4, 8)))
    call = lambda **kw: L.spl_verify_tree(*{**good, **kw}.values(), None)  # noqa: E731
    for n in [n for n in names if good[n] == base]:
        assert call(**{n: None}) == spl.SPL_EINVAL, n
        assert call(**{n: base + 2}) == spl.SPL_EALIGN, n
    for kw in ({"vocab": 0}, {"vocab": -1}, {"ldp": 7}, {"lde": 7}, {"ldpath": 3}, {"rows": -1}, {"seqs": -1}, {"levels": 0},
               {"levels": -1}):
        assert call(**kw) == spl.SPL_EINVAL, kw
    big = {"ldp": 1 << 32, "lde": 1 << 32}
    for kw in ({"seqs": 4097}, {"rows": 1 << 31}, {"levels": 1 << 31, "ldpath": 1 << 32}, {"vocab": 1 << 31, **big}):
        assert call(**kw) == spl.SPL_ESHAPE, kw


# ---------------------------------------------------------------------------------- the oracle
def test_oracle_trees():
    """Two branches behind two tokens: each row averages the context and its own branch; the window takes the last."""
    masks = [0b1, 0b11, 0b101, 0b1011]
    assert serving.tree_keys(masks[3], 2, 6, 0).tolist() == [0, 1, 2, 3, 5]
    assert serving.tree_keys(masks[3], 2, 6, 2).tolist() == [3, 5] and serving.tree_keys(0, 2, 6, 0).tolist() == [0, 1]
    v = np.arange(6.0)[:, None, None] * np.ones((1, 1, 4))
    out, _ = serving.tree_attention(np.zeros((4, 1, 4)), np.ones((6, 1, 4)), v, masks, 2, 1, 1.0)
    assert np.allclose(out[:, 0, 0], [1.0, 1.5, 7 / 4, 11 / 5])
    chain = [(1 << i + 1) - 1 for i in range(4)]
    g = np.random.default_rng(0)
    q, k, v = g.standard_normal((4, 2, 8)), g.standard_normal((9, 1, 8)), g.standard_normal((9, 1, 8))
    for window in (0, 3):
        assert np.allclose(serving.tree_attention(q, k, v, chain, 5, 2, 0.3, window)[0],
                           serving.attention(q, k, v, 9, 2, 0.3, window)[0])


def test_oracle_weights_and_eviction():
    """Equal scores share a row's weight of 1; a row's weights sum to 1; the heaviest and the latest stay."""
    w = serving.weights(np.zeros((2, 1, 4)), np.ones((3, 1, 4)), 3, 1, 1.0)
    assert np.allclose(w, [[1 / 2 + 1 / 3, 1 / 2 + 1 / 3, 1 / 3]])
    g = np.random.default_rng(1)
    w = serving.weights(g.standard_normal((4, 6, 8)), g.standard_normal((9, 2, 8)), 9, 3, 1.0, window=4)
    assert np.allclose(w.sum(1), 4 * 3)
    assert serving.evict([5, 1, 5, 9, 0, 0], 4, 1) == [0, 2, 3, 5]
    assert serving.evict([5, np.nan, -np.inf, 5], 3, 0) == [0, 2, 3] and serving.evict([1, 2], 2, 1) == [0, 1]
    assert serving.evict([1, 2, 3], 1, 1) == [2] and serving.evict([1, 2, 3], 0, 0) == []


def test_oracle_tree_verification_keeps_the_target_distribution():
    """Whatever the drafts, the first token is the race's winner: its distribution is p, here by enumeration of which
    entry's exponential is smallest in proportion."""
    p = np.array([[0.5, 0.3, 0.2], [0.1, 0.8, 0.1], [1.0, 0, 0]])
    path, token = serving.verify_tree(p, [0, 1, 2], [-1, 0, 0], np.array([[1, 0.5, 1], [1, 1, 1.0]]))
    assert path == [1] and token == 1
    path, token = serving.verify_tree(p, [0, 1, 2], [-1, 0, 0], np.array([[0.1, 1, 1], [1, 1, 1.0]]))
    assert path == [] and token == 0
    g = np.random.default_rng(2)
    e = g.exponential(size=(40000, 3))
    won = np.argmax(p[0] / e, axis=1)
    share = np.bincount(won, minlength=3) / len(won)
    assert np.all(np.abs(share - p[0]) < 5 * np.sqrt(p[0] * (1 - p[0]) / len(won)))


# ---------------------------------------------------------------------------------- serving.py
def test_the_shape_of_a_tree():
    from paper_2609_15039_gb300 import serving as example
    t = example.Tree([3, 2])
    assert (t.nodes, t.levels, t.first) == (10, 3, [0, 1, 4, 10])
    assert t.parents == [-1, 0, 0, 0, 1, 1, 2, 2, 3, 3]
    assert t.seen[:, 0].tolist() == [1, 3, 5, 9, 19, 35, 69, 133, 265, 521]
    t = example.Tree([1] * 40)  # a chain: the bits of all before, over two words
    assert t.seen.shape == (41, 2) and t.seen[40].tolist() == [-1, 511] and t.seen[31].tolist() == [-1, 0]
    assert example.Tree([]).nodes == 1
    with pytest.raises(ValueError):
        example.Tree([2, 0])


def test_generation_that_is_refused(monkeypatch):
    from paper_2609_15039_gb300 import serving as example
    for call in (lambda: example.generate_tree(None, None, None, [[1], []], [2], 1),
                 lambda: example.generate_bounded(None, None, [[]], 1, 4, 1),
                 lambda: example.generate_bounded(None, None, [[1]], 1, 4, 5),
                 lambda: example.generate_bounded(None, None, [[1]], 1, 4, -1)):
        with pytest.raises(ValueError):
            call()


def test_a_trees_rows_are_not_weighed():
    from paper_2609_15039_gb300 import serving as example
    with pytest.raises(ValueError, match="tree"):
        example.CachedDecoder.forward(None, None, None, seen=1, weigh=True)


def test_the_slots_of_new_tokens():
    """By sequences without rows, rows before the first position or past the table, and pages outside the pool."""
    from types import SimpleNamespace

    import torch

    from paper_2609_15039_gb300 import serving as example
    batch = SimpleNamespace(row_start=torch.tensor([0, 3, 3, 5, 9, 11]), kv_len=torch.tensor([18, 7, 1, 34, 17]),
                            page_table=torch.tensor([[4, 2], [0, 0], [1, 0], [3, 5], [0, 6]]))
    page, place = example.slots(batch, SimpleNamespace(page_size=16, pages=6))
    assert page.tolist() == [4, 2, 2] + [1] + [5, 5] + [0]
    assert place.tolist() == [15, 0, 1] + [0] + [14, 15] + [15]


def test_a_bound_and_a_tree_are_not_one_command(monkeypatch, capsys):
    from paper_2609_15039_gb300 import serving as example

    def begun(*a, **k):
        raise AssertionError("the command began")
    monkeypatch.setattr(example, "synthetic", begun)
    with pytest.raises(SystemExit) as end:
        example.main(["--keep", "40", "--tree", "3,2"])
    assert end.value.code == 2 and "--tree" in capsys.readouterr().err


def test_a_bound_on_the_rows_that_bounds_nothing(spl, base):  # noqa: F811
    """max_rows may be any number that is enough: the largest chooses the kernels of many rows like any other large one."""
    L = spl.lib()
    for group in (1, 2, 3, 1024):
        for size in (L.spl_kv_weigh_workspace_bytes, L.spl_paged_attention_workspace_bytes):
            for d in (64, 128):
                # (a table wide enough for the choice of kernel to go by the rows)
                c = ctypes.byref(cache_of(spl, base, head_dim=d, pages=1 << 16))
                need = [size(c, ctypes.byref(batch_of(spl, base, max_rows=most, max_pages=1 << 16)), 30, 2 * group)
                        for most in (1 << 24, 1 << 61, (1 << 63) - 1)]
                assert need[0] > 0 and need[1:] == need[:1] * 2, (group, d, need)
