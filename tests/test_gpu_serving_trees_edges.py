"""Attention weights and trees at the edges of their contracts: lengths past the page table, rows and keys that are not finite."""

import numpy as np
import pytest
import torch

from oracle import serving
from test_gpu_serving import DEV, U, Case, i32, many, tolerance
from test_gpu_serving_trees import KERNELS, attend_tree, masks_of, random_tree, score_of, scores_for, weight_tolerance

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def spl():
    from paper_2609_15039_gb300 import spl as binding
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    binding.lib()
    return binding


def queries(c):
    return torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("page", [64, 256])
@pytest.mark.parametrize("over", [0, 2])
@pytest.mark.parametrize("past", [50, 700])
@pytest.mark.parametrize("window", [0, 1, 100])
@KERNELS
def test_weigh_lengths_past_a_table_of_whole_tiles(spl, kernel, window, past, over, page, fmt):
    """A length past the table whose room is a whole number of tiles of keys: its rows see what is there, or nothing; the other
    sequences' scores keep their bits, and nothing is written behind the workspace."""
    room = 512
    c = kernel(Case(spl, [(3, room), (2, 300), (3, room)], (4, 2, 64), fmt, page, seed=past))
    c.table = np.ascontiguousarray(c.table[:, :room // page])
    c.fill()
    batch, q = c.batch(), queries(c)
    size = spl.spl_kv_weigh_workspace_bytes(c.cache, batch, c.hq)
    memory = torch.full((size + 65536,), 0xa5, dtype=torch.uint8, device=DEV)

    def weigh(lens):
        batch.kv_len.copy_(i32(lens))
        score = scores_for(c, 0.75)
        spl.spl_kv_weigh(score, q, c.cache, batch, c.hq, window=window, workspace=memory[:size])
        torch.cuda.synchronize()
        assert bool((memory[size:] == 0xa5).all())
        return score

    lens = [n for _, n in c.seqs]
    clean = weigh(lens)
    assert spl.spl_get_device_status() == spl.SPL_OK
    lens[over] = room + past
    score = weigh(lens)
    assert spl.spl_get_device_status() == spl.SPL_EINVAL
    for b in {0, 1, 2} - {over}:
        assert np.array_equal(score_of(c, score, b), score_of(c, clean, b))
    rows, k = c.q[c.start[over]:c.start[over + 1]], c.stored("k", over)
    added = np.zeros((c.hk, room))
    for i in range(3):
        lo, hi = serving.visible(room + past - 3 + i, room, window)
        if lo < hi:
            added[:, lo:hi] += serving.weights(rows[i:i + 1], k[lo:hi], hi - lo, 2, 0.125)
    err = np.abs(score_of(c, score, over) - (0.75 + added))  # (all of them are before the rows)
    assert np.all(err <= weight_tolerance(rows, k, 0.125, 2, 6) * added + 2 * U * (0.75 + added))
    used = np.zeros(tuple(score.shape), dtype=bool)
    for b, (_, n) in enumerate(c.seqs):
        j = np.arange(n)
        used[c.table[b, j // page], :, j % page] = True
    assert np.all(score.cpu().numpy()[~used] == 0.75)


@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=str)
@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("length", [200, 201, 202, 203])
@pytest.mark.parametrize("window", [1, 2, 63, 64])
@KERNELS
def test_weigh_a_nan_row_leaves_what_is_before_its_window(spl, kernel, window, length, fmt, value):
    c = kernel(Case(spl, [(1, length)], (4, 2, 64), fmt, 16, seed=window))
    c.fill()
    c.q[0, 2, 3] = value
    score = scores_for(c, 0.75)
    spl.spl_kv_weigh(score, queries(c), c.cache, c.batch(), c.hq, window=window)
    got = score_of(c, score, 0)
    assert np.all(got[:, :length - window] == 0.75)
    assert np.isfinite(got[0]).all() and np.isnan(got[1, length - window:]).all()
    assert spl.spl_get_device_status() == spl.SPL_OK


@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=str)
@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("context", [100, 101, 102, 103])
@KERNELS
def test_weigh_a_nan_row_leaves_what_is_behind_it(spl, kernel, context, fmt, value):
    """The tokens that only later rows see, in the same four keys or not, get their weights."""
    c = kernel(Case(spl, [(9, context + 9)], (4, 2, 64), fmt, 16, seed=context))
    c.fill()
    c.q[1, 2, 3] = value
    score = scores_for(c, 0.75)
    spl.spl_kv_weigh(score, queries(c), c.cache, c.batch(), c.hq)
    got = score_of(c, score, 0)
    assert np.isfinite(got[0]).all() and np.isnan(got[1, :context + 2]).all()
    k = c.stored("k", 0)
    added = serving.weights(c.q[2:], k, context + 9, 2, 0.125)[1, context + 2:]
    err = np.abs(got[1, context + 2:] - added)  # (new tokens: they start from 0)
    assert np.all(err <= weight_tolerance(c.q[2:], k, 0.125, 2, 18) * added + 2 * U * added)
    assert spl.spl_get_device_status() == spl.SPL_OK


@pytest.mark.parametrize("value", [float("inf"), float("-inf")], ids=str)
@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("at", [5, 131, 290])
@pytest.mark.parametrize("window", [0, 40, 300])
@KERNELS
def test_weigh_infinite_keys(spl, kernel, window, at, fmt, value):
    """A stored infinity (of an 8-bit vector: its scale), whichever way the halves of a query row point: the rows that see it give
    NaN to what they see, in its head alone; those that do not are as without it, to the bit."""
    seqs = [(1, 300 + b) for b in range(24)]
    c = kernel(Case(spl, seqs, (4, 2, 64), fmt, 16, seed=at))
    c.fill()
    clean = scores_for(c, 0.75)
    spl.spl_kv_weigh(clean, queries(c), c.cache, c.batch(), c.hq, window=window)
    for b in range(0, len(seqs), 2):  # (every other sequence)
        page, place = int(c.table[b, at // 16]), at % 16
        if fmt == "f16":
            c.cache.k[page, 1, place, b % 64] = value
        else:
            c.cache.k_scale[page, 1, place] = value
    score = scores_for(c, 0.75)
    spl.spl_kv_weigh(score, queries(c), c.cache, c.batch(), c.hq, window=window)
    for b, (_, n) in enumerate(seqs):
        got, was = score_of(c, score, b), score_of(c, clean, b)
        lo = max(0, n - window) if window else 0
        assert np.array_equal(got[0], was[0])
        if b % 2 == 0 and at >= lo:
            assert np.array_equal(got[1, :lo], was[1, :lo]) and np.isnan(got[1, lo:]).all()
        else:
            assert np.array_equal(got[1], was[1])
    assert spl.spl_get_device_status() == spl.SPL_OK


@pytest.mark.parametrize("value", [float("inf"), float("-inf")], ids=str)
@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("at", [20, 400, 610])
@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 2, 128)], ids=str)
@KERNELS
def test_weigh_infinite_keys_of_many_rows(spl, kernel, heads, at, fmt, value):
    """The rows that see the key give NaN to all that they see: without a window the last one's is everything, with one what the
    others see stays, to the bit, and so do other sequences and heads."""
    c = kernel(Case(spl, [(200, 700), (150, 300)], heads, fmt, 32, seed=at))
    c.fill()
    clean = [scores_for(c, 0.75) for _ in range(2)]
    score = [scores_for(c, 0.75) for _ in range(2)]
    for s, window in zip(clean, (0, 100)):
        spl.spl_kv_weigh(s, queries(c), c.cache, c.batch(), c.hq, window=window)
    page, place = int(c.table[0, at // 32]), at % 32
    if fmt == "f16":
        c.cache.k[page, 1, place, 7] = value
    else:
        c.cache.k_scale[page, 1, place] = value
    for s, window in zip(score, (0, 100)):
        spl.spl_kv_weigh(s, queries(c), c.cache, c.batch(), c.hq, window=window)
    # rows from max(at, 500) on see it, those up to at + 99 with the window
    first, last = max(at, 500), min(699, at + 99)
    for s, was, lo, hi in zip(score, clean, (0, first - 99 if first <= last else 700), (700, last + 1)):
        got, want = score_of(c, s, 0), score_of(c, was, 0)
        assert np.array_equal(score_of(c, s, 1), score_of(c, was, 1)) and np.array_equal(got[0], want[0])
        assert np.isnan(got[1, lo:hi]).all() and np.array_equal(got[1, :lo], want[1, :lo])
        assert lo > hi or np.array_equal(got[1, hi:], want[1, hi:])
    assert spl.spl_get_device_status() == spl.SPL_OK


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("past", [0, 3, 5, 40, 400])
@pytest.mark.parametrize("window", [1, 5, 40, 63, 64, 100])
def test_tree_attention_windows_of_lengths_past_the_table(spl, window, past, fmt):
    """A window takes the last keys that a row sees, which end with the table where the length does not."""
    g = np.random.default_rng(past)
    room = 64
    for kernel in (lambda c: c, many):
        c = kernel(Case(spl, [(5, room), (3, 40)], (4, 2, 64), fmt, 16, seed=window))
        c.table = np.ascontiguousarray(c.table[:, :room // 16])
        c.fill()
        masks = [masks_of(random_tree(g, r)) for r, _ in c.seqs]
        batch = c.batch()
        c.batch = lambda all_rows=False, batch=batch: batch
        batch.kv_len.copy_(i32([room + past, 40]))
        got = attend_tree(c, masks, 1, window=window)
        assert spl.spl_get_device_status() == (spl.SPL_EINVAL if past else spl.SPL_OK)
        for b, context in enumerate((room + past - 5, 37)):
            q, k, v = c.q[c.start[b]:c.start[b + 1]], c.stored("k", b), c.stored("v", b)
            ref, mass = serving.tree_attention(q, k, v, masks[b], context, 2, 0.125, window)
            tol = tolerance(q, k, 0.125, len(k), 2, mass) + 2.0 ** -32 * len(k) * np.max(np.abs(v))
            err = np.abs(got[c.start[b]:c.start[b + 1]].astype(np.float64) - ref)
            assert np.all(err <= tol), f"sequence {b}: worst err/tol {np.max(err / tol):.3g}"


@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=str)
@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 2, 128)], ids=str)
@KERNELS
def test_weigh_a_nan_row_among_many(spl, kernel, heads, fmt, value):
    """Over several ranges of keys and tiles of rows: what the row does not see is as without it, to the bit."""
    c = kernel(Case(spl, [(40, 90), (300, 5000), (0, 300)], heads, fmt, 64, seed=1))
    c.fill()
    clean = scores_for(c, 0.75)
    spl.spl_kv_weigh(clean, queries(c), c.cache, c.batch(), c.hq, window=700, decay=0.5)
    c.q[40 + 100, c.hq // 2, 5] = value
    score = scores_for(c, 0.75)
    spl.spl_kv_weigh(score, queries(c), c.cache, c.batch(), c.hq, window=700, decay=0.5)
    lo, hi = serving.visible(4800, 5000, 700)
    for b in (0, 2):
        assert np.array_equal(score_of(c, score, b), score_of(c, clean, b))
    got, want = score_of(c, score, 1), score_of(c, clean, 1)
    assert np.isnan(got[1, lo:hi]).all() and np.array_equal(got[0], want[0])
    assert np.array_equal(got[1, :lo], want[1, :lo]) and np.array_equal(got[1, hi:], want[1, hi:])
    assert spl.spl_get_device_status() == spl.SPL_OK
