"""The paged cache, attention over it and the verification of drafts, on the GPU against 64 bits."""

import numpy as np
import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


@pytest.fixture(scope="module")
def spl():
    from paper_2609_15039_gb300 import spl as binding
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    binding.lib()
    return binding


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Case:
    """A batch of sequences (new rows, length) on shuffled pages, every slot outside the tokens poisoned with NaN."""

    def __init__(self, spl, seqs, heads, fmt, page, seed, std=1.0, spare=2):
        self.spl, self.seqs, self.fmt, self.page = spl, seqs, fmt, page
        self.hq, self.hk, self.d = heads
        g = np.random.default_rng(seed)
        need = [-(-n // page) for _, n in seqs]
        pages = sum(need) + spare
        order = g.permutation(pages)[:sum(need)]
        self.table = np.full((len(seqs), max(need + [1]) + 1), pages + 7, dtype=np.int32)  # ids past the pool
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = order[at:at + m]
            at += m
        self.rows = sum(r for r, _ in seqs)
        self.start = np.concatenate([[0], np.cumsum([r for r, _ in seqs])]).astype(np.int32)
        self.k = [g.standard_normal((n, self.hk, self.d)).astype(np.float32) * std for _, n in seqs]
        self.v = [(g.standard_normal((n, self.hk, self.d)) + 0.25).astype(np.float32) for _, n in seqs]
        self.q = g.standard_normal((self.rows, self.hq, self.d)).astype(np.float32) * std
        self.cache = spl.KVCache.empty(pages, self.hk, self.d, page, fmt)
        self.poison()

    def poison(self):
        if self.fmt == "f16":
            self.cache.k.fill_(float("nan"))
            self.cache.v.fill_(float("nan"))
        else:
            self.cache.k.fill_(-128)
            self.cache.v.fill_(127)
            self.cache.k_scale.fill_(float("nan"))
            self.cache.v_scale.fill_(float("inf"))

    def batch(self, all_rows=False):
        """The batch of the new rows, or of every token as a new row."""
        lens = [n for _, n in self.seqs]
        start = np.concatenate([[0], np.cumsum(lens)]) if all_rows else self.start
        rows = sum(lens) if all_rows else self.rows
        most = max([r for r, _ in self.seqs] + [1])
        return self.spl.KVBatch(i32(start.tolist()), i32(lens), torch.as_tensor(self.table).to(DEV), rows,
                                max(lens) if all_rows else most)

    def fill(self):
        cat = lambda parts: torch.as_tensor(np.concatenate(parts).reshape(-1, self.hk * self.d)).to(DEV)  # noqa: E731
        self.spl.spl_kv_append(self.cache, self.batch(True), cat(self.k), cat(self.v))

    def stored(self, which, b):
        """fp32 values that the cache holds of sequence b, from the definition."""
        x = (self.k if which == "k" else self.v)[b]
        if self.fmt == "f16":
            return serving.quantize_f16(x).astype(np.float32)
        code, scale = serving.quantize_i8(x)
        return (code.astype(np.float32) * scale[..., None]).astype(np.float32)

    def attend(self, window=0, scale=None, workspace=None, q=None):
        out = torch.full((self.rows, self.hq * self.d), float("nan"), device=DEV)
        q = torch.as_tensor(self.q.reshape(self.rows, -1)).to(DEV) if q is None else q
        self.spl.spl_paged_attention(out, q, self.cache, self.batch(), self.hq, scale=scale, window=window,
                                     workspace=workspace)
        torch.cuda.synchronize()
        return out.cpu().numpy().reshape(self.rows, self.hq, self.d)

    def check(self, window=0, scale=None, **kw):
        got = self.attend(window, scale, **kw)
        s = 1.0 / np.sqrt(self.d) if scale is None else scale
        num = den = 0.0
        for b, (r, n) in enumerate(self.seqs):
            k, v = self.stored("k", b), self.stored("v", b)
            q = self.q[self.start[b]:self.start[b + 1]]
            ref, mass = serving.attention(q, k, v, n, self.hq // self.hk, s, window)
            mine = got[self.start[b]:self.start[b + 1]]
            tol = tolerance(q, k, s, n, self.hq // self.hk, mass)
            err = np.abs(mine.astype(np.float64) - ref)
            assert not np.isnan(mine).any(), f"sequence {b}: NaN"
            assert np.all(err <= tol), f"sequence {b} {r, n}: worst err/tol {np.max(err / np.maximum(tol, 1e-300)):.3g}"
            num += float(np.sum((mine - ref) ** 2))
            den += float(np.sum(ref ** 2))
        assert num <= (1e-5 ** 2) * den, f"relative error {np.sqrt(num / max(den, 1e-300)):.3g}"
        assert self.spl.spl_get_device_status() == self.spl.SPL_OK
        return got


def tolerance(q, k, scale, n, group, mass):
    """Elementwise bound.  A score is a sum of `dim` terms of which q's split loses 2^-22 and each of the dim / 16
    accumulations (twice, for the two halves) at most 2^-23 of the sum of sizes S: its error is at most
    (2^-22 + (dim / 8) 2^-23) S, and a few ulp from the scaling.  That, an exp of 2^-21, a probability's split of 2^-22
    and the accumulation of the n / 16 key steps (2^-23 each, twice) are relative to sum_j p_j |v_j|; the total has
    the same, and three roundings follow."""
    if n == 0 or q.shape[0] == 0:
        return np.zeros_like(mass)
    dim = q.shape[-1]
    size = abs(scale) * np.max(np.einsum("ihd,jhd->ihj", np.abs(q).astype(np.float64),
                                         np.repeat(np.abs(k).astype(np.float64), group, axis=1)), axis=2)
    score = (2.0 ** -22 + dim / 8 * 2.0 ** -23 + 4 * U) * size
    rel = 2 * (score + 2.0 ** -21) + 2.0 ** -22 + (n / 8 + 16) * 2.0 ** -23 + 4 * U
    return rel[..., None] * mass + 1e-30


HEADS = [(24, 8, 128), (8, 2, 64), (3, 3, 128), (7, 1, 64), (16, 1, 128)]
BATCHES = {
    "one": [(1, 1)], "two": [(1, 2)], "page": [(1, 64)], "past_page": [(1, 65)], "odd": [(1, 299)],
    "ragged": [(1, 5), (1, 1000), (0, 17), (1, 128), (0, 0), (1, 1)],
    "drafts": [(5, 261), (3, 3), (1, 700), (4, 64)],
    "chunks": [(37, 37), (130, 333), (1, 90), (64, 64)],
}


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("name", BATCHES)
def test_attention(spl, name, heads, fmt):
    c = Case(spl, BATCHES[name], heads, fmt, 16 if name == "ragged" else 64, seed=len(name))
    c.fill()
    c.check()


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_attention_page_sizes(spl, page, fmt):
    c = Case(spl, [(3, 300), (20, 257), (1, page), (150, 150 + page)], (6, 2, 128), fmt, page, seed=page)
    c.fill()
    c.check()


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("window", [1, 2, 63, 64, 129, 1000])
def test_attention_window(spl, window, fmt):
    c = Case(spl, [(1, 500), (9, 300), (140, 400), (70, 70)], (4, 2, 64), fmt, 32, seed=window)
    c.fill()
    c.check(window=window)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
def test_rows_without_keys_are_zero(spl, fmt):
    """A sequence shorter than its rows: the first stand before position 0 and see nothing."""
    c = Case(spl, [(6, 2), (1, 0), (140, 3)], (4, 2, 128), fmt, 16, seed=3)
    c.fill()  # writes the tokens that exist
    got = c.check()
    assert np.all(got[:4] == 0) and np.all(got[6] == 0) and np.all(got[7:7 + 137] == 0)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("rows", [1, 40])
def test_attention_sharp_and_flat(spl, rows, fmt):
    """Scores that single out one key, and scores that are all equal; other scales, a negative one among them."""
    for std, scale in ((6.0, None), (1.0, 0.0), (1.0, -0.3), (2.0, 1.0)):
        c = Case(spl, [(rows, 777)], (4, 1, 64), fmt, 64, seed=rows, std=std)
        c.fill()
        c.check(scale=scale)


@pytest.mark.parametrize("rows", [2, 5, 48, 200])
@pytest.mark.parametrize("which", ["k", "v"])
def test_nan_reaches_only_rows_that_see_it(spl, which, rows):
    """A NaN in a later token of the chunk: earlier rows are as without it, later ones are NaN."""
    for fmt in ("f16", "i8"):
        c = Case(spl, [(rows, 100 + rows)], (4, 2, 64), fmt, 16, seed=rows)
        c.fill()
        clean = c.check()
        at = rows // 2
        x = getattr(c, which)[0]
        x[100 + at, 1, 3] = np.nan
        c.fill()
        got = c.attend()
        assert np.array_equal(got[:at], clean[:at])
        assert np.array_equal(got[:, :2], clean[:, :2])  # the other key head's rows
        assert np.isnan(got[at:, 2:]).any(axis=2).all()


def test_attention_reads_and_writes_strided_rows(spl):
    c = Case(spl, [(3, 50), (60, 61)], (6, 2, 64), "f16", 16, seed=8)
    c.fill()
    want = c.check()
    wide = torch.full((c.rows, 1000), 7.0, device=DEV)
    wide[:, 8:8 + 384] = torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV)
    out = torch.full((c.rows, 516), 5.0, device=DEV)
    spl.spl_paged_attention(out[:, 64:448], wide[:, 8:392], c.cache, c.batch(), 6)
    assert np.array_equal(out[:, 64:448].cpu().numpy().reshape(want.shape), want)
    assert bool((out[:, :64] == 5).all()) and bool((out[:, 448:] == 5).all())


@pytest.mark.parametrize("rows", [1, 60])
def test_attention_is_deterministic_and_leaves_the_workspace_clean(spl, rows):
    """Same bits again on one workspace, shared with other shapes; the arrival counters end at zero."""
    a = Case(spl, [(rows, 3000), (rows, 100)], (8, 2, 128), "f16", 64, seed=1)
    b = Case(spl, [(1, 40)], (4, 4, 64), "i8", 16, seed=2)
    for c in (a, b):
        c.fill()
    ws = spl.workspace(max(spl.spl_paged_attention_workspace_bytes(c.cache, c.batch(), c.hq) for c in (a, b)))
    first = a.attend(workspace=ws)
    for _ in range(3):
        b.check(workspace=ws)
        assert np.array_equal(a.attend(workspace=ws), first)
    assert int(ws[:65536].count_nonzero()) == 0


def test_attention_in_a_graph_follows_the_lengths(spl):
    """A captured decode step is replayed as its sequences grow: lengths and tables are read on the device."""
    c = Case(spl, [(1, 90), (1, 31)], (4, 2, 64), "f16", 16, seed=5)
    c.fill()
    batch = c.batch()
    q = torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV)
    out = torch.zeros((c.rows, 4 * 64), device=DEV)
    ws = spl.workspace(spl.spl_paged_attention_workspace_bytes(c.cache, batch, 4))
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        spl.spl_paged_attention(out, q, c.cache, batch, 4, workspace=ws)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spl.spl_paged_attention(out, q, c.cache, batch, 4, workspace=ws)
    for lens in ([90, 31], [40, 1], [90, 0]):
        batch.kv_len.copy_(i32(lens))
        graph.replay()
        torch.cuda.synchronize()
        for b, n in enumerate(lens):
            ref, _ = serving.attention(c.q[b:b + 1], c.stored("k", b)[:n], c.stored("v", b)[:n], n, 2, 0.125)
            assert np.allclose(out[b].cpu().numpy().reshape(4, 64), ref[0], rtol=0, atol=1e-5)


def test_ids_outside_the_pool_are_reported_and_not_followed(spl):
    for rows in (1, 40):
        c = Case(spl, [(rows, 200), (rows, 64)], (4, 2, 64), "f16", 16, seed=4)
        c.fill()
        good = c.check()
        keep = c.table.copy()
        c.table[0, 3] = -5
        c.table[0, 6] = 1 << 30
        bad = c.attend()
        assert spl.spl_get_device_status() == spl.SPL_EINVAL
        assert spl.spl_get_device_status() == spl.SPL_OK
        assert np.array_equal(bad[rows:], good[rows:]) and np.isfinite(bad).all()
        c.table = keep
        batch = c.batch()
        batch.kv_len.copy_(i32([1 << 30, 64]))  # past the table: its tokens end where the table does
        x = torch.zeros((c.rows, 2 * 64), device=DEV)
        spl.spl_kv_append(c.cache, batch, x, x)
        assert spl.spl_get_device_status() == spl.SPL_EINVAL


# ---------------------------------------------------------------------------------- the cache itself
@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("heads", [(8, 8, 128), (2, 2, 64), (1, 1, 128), (9, 9, 64), (20, 20, 128)], ids=str)
def test_append_and_read_back_exactly(spl, heads, fmt):
    c = Case(spl, [(1, 1), (0, 40), (17, 200), (64, 64), (0, 0), (1, 33)], heads, fmt, 16, seed=11)
    for x in c.k + c.v:
        if x.size:
            x[0, 0] = 0.0  # a zero vector
            x[-1, -1] *= 1e30 if fmt == "i8" else 1e6
    c.fill()
    lens = [n for _, n in c.seqs]
    start = np.concatenate([[0], np.cumsum(lens)])
    width = c.hk * c.d
    K = torch.full((int(start[-1]) + 3, width), 3.0, device=DEV)
    V = torch.full_like(K, 3.0)
    spl.spl_kv_read(K, V, c.cache, c.batch(), i32(start.tolist()))
    for got, which in ((K, "k"), (V, "v")):
        want = np.concatenate([c.stored(which, b) for b in range(len(lens))]).reshape(-1, width)
        assert np.array_equal(got[:-3].cpu().numpy(), want)
        assert bool((got[-3:] == 3.0).all())  # rows of no token
    assert spl.spl_get_device_status() == spl.SPL_OK
    # untouched: the pages of no sequence
    used = set(int(p) for b, n in enumerate(lens) for p in c.table[b, :-(-n // 16)])
    free = [p for p in range(c.cache.pages) if p not in used]
    x = c.cache.k[free].float()
    assert bool((x.isnan() if fmt == "f16" else x == -128).all())


def test_append_writes_only_the_new_rows(spl):
    c = Case(spl, [(2, 50), (1, 7)], (2, 2, 64), "i8", 16, seed=12)
    rows = torch.randn((c.rows, 300), device=DEV)
    spl.spl_kv_append(c.cache, c.batch(), rows[:, 4:132], rows[:, 136:264])
    code, scale = serving.quantize_i8(rows[:, 4:132].cpu().numpy().reshape(-1, 2, 64))
    want = np.full(tuple(c.cache.k.shape), -128, dtype=np.int8)
    for r, (b, pos) in enumerate([(0, 48), (0, 49), (1, 6)]):
        want[c.table[b, pos // 16], :, pos % 16] = code[r]
    assert np.array_equal(c.cache.k.cpu().numpy(), want)
    assert int(c.cache.k_scale.isfinite().sum()) == 3 * 2


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_special_values_in_the_cache(spl, bad):
    for fmt in ("f16", "i8"):
        c = Case(spl, [(1, 3)], (2, 2, 64), fmt, 16, seed=13)
        c.k[0][1, 1, 5] = bad
        c.fill()
        K, V = torch.zeros((3, 128), device=DEV), torch.zeros((3, 128), device=DEV)
        spl.spl_kv_read(K, V, c.cache, c.batch(), i32([0, 3]))
        got = K.cpu().numpy().reshape(3, 2, 64)
        want = c.stored("k", 0)
        assert np.array_equal(got, want, equal_nan=True)
        if fmt == "i8":
            assert np.isnan(got[1, 1]).all()
        else:
            assert np.isnan(got[1, 1, 5]) if np.isnan(bad) else got[1, 1, 5] == np.sign(bad) * 65504


# ---------------------------------------------------------------------------------- drafts
def draws(seed, counts, vocab, sharp=2.5):
    g = np.random.default_rng(seed)
    soft = lambda z: (np.exp(z) / np.exp(z).sum(-1, keepdims=True)).astype(np.float32)  # noqa: E731
    rows, drafts = sum(k + 1 for k in counts), sum(counts)
    p = soft(g.standard_normal((rows, vocab)) * sharp)
    q = soft(g.standard_normal((max(drafts, 1), vocab)) * sharp)[:drafts]
    x = np.array([g.choice(vocab, p=r.astype(np.float64) / r.sum(dtype=np.float64)) for r in q], dtype=np.int32)
    return p, q, x, g.random(drafts, dtype=np.float32), g.exponential(size=(len(counts), vocab)).astype(np.float32)


def run_verify(spl, p, q, x, u, e, counts, pad=0):
    dev = lambda t: torch.as_tensor(np.ascontiguousarray(t)).to(DEV)  # noqa: E731

    def rows(t):
        wide = torch.full((t.shape[0], t.shape[1] + pad), 9.0, device=DEV)
        wide[:, :t.shape[1]] = dev(t)
        return wide[:, :t.shape[1]]

    n = len(counts)
    accepted, token = torch.full((n,), -9, dtype=torch.int32, device=DEV), i32([-9] * n)
    start = np.concatenate([[0], np.cumsum([k + 1 for k in counts])])
    dstart = np.concatenate([[0], np.cumsum(counts)])
    ws = spl.workspace(spl.spl_verify_drafts_workspace_bytes(n))
    for _ in range(2):
        spl.spl_verify_drafts(accepted, token, rows(p), rows(q), dev(x), dev(u), rows(e), i32(start.tolist()),
                              i32(dstart.tolist()), workspace=ws)
    assert int(ws.count_nonzero()) == 0
    return accepted.cpu().tolist(), token.cpu().tolist()


def expected(p, q, x, u, e, counts):
    out, r, d = [], 0, 0
    for b, k in enumerate(counts):
        out.append(serving.verify(p[r:r + k + 1], q[d:d + k], x[d:d + k], u[d:d + k], e[b]))
        r, d = r + k + 1, d + k
    return [a for a, _ in out], [t for _, t in out]


@pytest.mark.parametrize("vocab,pad", [(1, 0), (5, 3), (1000, 0), (1001, 0), (4099, 5), (32768, 4)])
@pytest.mark.parametrize("counts", [[0], [1], [3, 0, 8, 1], [40, 2]], ids=str)
def test_verify(spl, counts, vocab, pad):
    args = draws(vocab + len(counts), counts, vocab)
    if vocab == 1000:  # a target that the drafts follow: whole runs are accepted
        p, q, x, u, e = args
        r = d = 0
        for k in counts:
            q[d:d + k] = p[r:r + k]
            r, d = r + k + 1, d + k
        q = q.copy()
        x = np.array([int(np.argmax(row)) for row in q], dtype=np.int32)
        args = (p, q, x, u, e)
    assert run_verify(spl, *args, counts, pad) == expected(*args, counts)


def test_verify_edges(spl):
    vocab, counts = 64, [2, 2, 2, 2]
    p, q, x, u, e = draws(7, counts, vocab)
    q[0], x[0], u[0] = p[0], 5, 1.0 - 2.0 ** -24  # equal rows and u just below 1: accepted
    q[1], x[1], u[1] = p[1], 6, 0.5
    p[3, 9], x[2] = 0.0, 9                         # p = 0 at the draft: rejected
    q[4], u[4], x[4] = p[6] * 3, 0.999, 11         # p nowhere above q: the draw is from p
    p[9] = 0.25
    e[3] = 1.0
    x[6], q[6], u[6] = 1, p[9], 0.0                # then a draft outside the vocabulary
    x[7] = vocab
    p[10] = 0.0
    p[10, 40:50] = 0.1                             # ties: the lowest index
    q[7] = 0.0
    got = run_verify(spl, p, q, x, u, e, counts)
    assert got == expected(p, q, x, u, e, counts)
    assert got[0][0] == 2 and got[0][1] == 0 and got[0][2] == 0 and got[0][3] == 1
    assert got[1][3] == 40
    assert spl.spl_get_device_status() == spl.SPL_EINVAL  # the draft outside the vocabulary


def test_verify_sequences_without_rows(spl):
    p, q, x, u, e = draws(3, [2], 100)
    dev = lambda t: torch.as_tensor(t).to(DEV)  # noqa: E731
    accepted, token = i32([-9, -9, -9]), i32([-9, -9, -9])
    e3 = np.repeat(e, 3, axis=0)
    spl.spl_verify_drafts(accepted, token, dev(p), dev(q), dev(x), dev(u), dev(e3), i32([0, 0, 3, 3]),
                          i32([0, 0, 2, 2]))
    n, t = serving.verify(p, q, x, u, e[0])
    assert accepted.cpu().tolist() == [0, n, 0] and token.cpu().tolist() == [-1, t, -1]


def test_verify_draws_follow_the_target(spl):
    """The token after no drafts is a draw from p: frequencies of 4096 races within 5 standard deviations."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    n, vocab = 4096, 8
    p = torch.softmax(torch.arange(vocab, device=DEV) * 0.4, 0)[None].repeat(n, 1).contiguous()
    e = -torch.log1p(-torch.rand((n, vocab), generator=g, device=DEV)).clamp(max=-1e-30)
    e = e.clamp(min=1e-30)
    accepted, token = torch.empty(n, dtype=torch.int32, device=DEV), torch.empty(n, dtype=torch.int32, device=DEV)
    start = torch.arange(n + 1, dtype=torch.int32, device=DEV)
    zero = torch.zeros(n + 1, dtype=torch.int32, device=DEV)
    empty = torch.empty((0, vocab), device=DEV)
    spl.spl_verify_drafts(accepted, token, p, empty, torch.empty(0, dtype=torch.int32, device=DEV),
                          torch.empty(0, device=DEV), e, start, zero)
    freq = torch.bincount(token.long(), minlength=vocab).double().cpu() / n
    want = p[0].double().cpu()
    assert bool((freq - want).abs().le(5 * (want * (1 - want) / n).sqrt()).all())


# ---------------------------------------------------------------------------------- the kernel for many rows, at all sizes
def many(c):
    """The case with a bound on a chunk's rows that sends the call to the kernel for many rows, however few there are."""
    batch = c.batch
    c.batch = lambda all_rows=False: spl_batch_with_bound(c.spl, batch(all_rows))
    return c


def spl_batch_with_bound(spl, batch):
    return spl.KVBatch(batch.row_start, batch.kv_len, batch.page_table, batch.rows, 1 << 24)


def check_sample(c, samples, window=0, seed=0, scale=None):
    """As Case.check, for some rows and heads; a probability's low half may lose an absolute 2^-33 of the row's largest
    (hi rounded and lo rounded, each by 2^-25 of p's 2^9), which the n values that a row sees meet."""
    got = c.attend(window, scale)
    s = 1.0 / np.sqrt(c.d) if scale is None else scale
    g = np.random.default_rng(seed)
    group = c.hq // c.hk
    num = den = 0.0
    for b, (r, n) in enumerate(c.seqs):
        if r == 0:
            continue
        k, v = c.stored("k", b), c.stored("v", b)
        picks = {(0, 0), (r - 1, c.hq - 1)} | {(int(g.integers(r)), int(g.integers(c.hq))) for _ in range(samples)}
        for i, h in picks:
            kh = slice(h // group, h // group + 1)
            q = c.q[c.start[b] + i:c.start[b] + i + 1, h:h + 1]
            upto = max(0, min(n - r + i + 1, n))
            ref, mass = serving.attention(q, k[:upto, kh], v[:upto, kh], upto, 1, s, window)
            mine = got[c.start[b] + i, h]
            if upto == 0:
                assert np.all(mine == 0)
                continue
            tol = tolerance(q, k[:upto, kh], s, upto, 1, mass) + 2.0 ** -32 * upto * np.max(np.abs(v[:upto, kh]))
            err = np.abs(mine.astype(np.float64) - ref[0, 0])
            assert np.all(err <= tol[0, 0]), f"sequence {b} row {i} head {h}: {np.max(err / tol[0, 0]):.3g}"
            num += float(np.sum((mine - ref[0, 0]) ** 2))
            den += float(np.sum(ref ** 2))
    assert not np.isnan(got).any() and num <= (1e-5 ** 2) * den
    assert c.spl.spl_get_device_status() == c.spl.SPL_OK
    return got


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("name", BATCHES)
def test_many_rows(spl, name, heads, fmt):
    c = many(Case(spl, BATCHES[name], heads, fmt, 16 if name == "ragged" else 256, seed=len(name)))
    c.fill()
    check_sample(c, 12)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("page", [16, 64, 128, 256])
@pytest.mark.parametrize("window", [0, 1, 127, 128, 200, 1000])
def test_many_rows_window(spl, window, page, fmt):
    c = many(Case(spl, [(200, 900), (33, 1200), (130, 130), (150, 149 + page), (6, 2), (1, 0)], (4, 2, 64), fmt, page,
                  seed=window))
    c.fill()
    check_sample(c, 16, window)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("heads,rows,keys", [((32, 8, 128), 512, 3000), ((16, 16, 64), 300, 7001), ((8, 8, 128), 129, 9000)],
                         ids=str)
@pytest.mark.parametrize("window", [0, 2500])
def test_many_rows_long_pieces(spl, heads, rows, keys, window, fmt):
    """Pieces of many accumulation chains, tiles divided among several blocks, int8 scales that grow along the keys."""
    c = Case(spl, [(rows, keys), (2, 40)], heads, fmt, 64, seed=keys, std=2.0)
    c.v[0] *= np.exp2(np.linspace(-6, 6, keys)).astype(np.float32)[:, None, None]
    c.fill()
    check_sample(c, 24, window)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("std,scale", [(6.0, None), (1.0, 0.0), (1.0, -0.3), (2.0, 1.0)])
def test_many_rows_sharp_and_flat(spl, std, scale, fmt):
    c = many(Case(spl, [(40, 777), (300, 1500)], (4, 1, 64), fmt, 64, seed=17, std=std))
    c.fill()
    check_sample(c, 30, scale=scale)


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("rows", [5, 48, 200, 400])
@pytest.mark.parametrize("which", ["k", "v"])
def test_many_rows_nan_reaches_only_rows_that_see_it(spl, which, rows, page):
    for fmt in ("f16", "i8"):
        for bad in (np.nan, np.inf):
            c = many(Case(spl, [(rows, 100 + rows)], (4, 2, 64), fmt, page, seed=rows))
            c.fill()
            clean = check_sample(c, 4)
            at = rows // 2
            getattr(c, which)[0][100 + at, 1, 3] = bad
            c.fill()
            got = c.attend()
            assert np.array_equal(got[:at], clean[:at])
            assert np.array_equal(got[:, :2], clean[:, :2])
            if fmt == "i8" or np.isnan(bad):  # (binary16 saturates an infinity)
                assert np.isnan(got[at:, 2:]).any(axis=2).all()


@pytest.mark.parametrize("fmt", ["f16", "i8"])
def test_many_rows_is_deterministic_and_leaves_the_workspace_clean(spl, fmt):
    a = many(Case(spl, [(300, 3000), (20, 100), (129, 2000)], (8, 2, 128), fmt, 64, seed=1))
    b = Case(spl, [(1, 40)], (4, 4, 64), "i8", 16, seed=2)
    for c in (a, b):
        c.fill()
    ws = spl.workspace(max(spl.spl_paged_attention_workspace_bytes(c.cache, c.batch(), c.hq) for c in (a, b)))
    first = a.attend(workspace=ws)
    for _ in range(3):
        b.check(workspace=ws)
        assert np.array_equal(a.attend(workspace=ws), first)
    assert int(ws[:65536].count_nonzero()) == 0
    # strided rows give the same bits
    wide = torch.full((a.rows, 8 * 128 + 12), 7.0, device=DEV)
    wide[:, 8:-4] = torch.as_tensor(a.q.reshape(a.rows, -1)).to(DEV)
    out = torch.full((a.rows, 8 * 128 + 4), 5.0, device=DEV)
    spl.spl_paged_attention(out[:, 4:], wide[:, 8:-4], a.cache, a.batch(), 8, workspace=ws)
    assert np.array_equal(out[:, 4:].cpu().numpy().reshape(first.shape), first) and bool((out[:, :4] == 5).all())


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("rows", [1, 5, 200])
def test_offsets_past_32_bits(spl, rows, fmt):
    """A pool whose elements and bytes pass 2^32: the sequences lie in its last pages."""
    page, heads = 256, (16, 8, 128)
    c = Case(spl, [(rows, 700), (rows, 300)], heads, fmt, page, seed=rows)
    pages = (1 << 32) // (8 * page * 128) + 40
    c.cache = spl.KVCache.empty(pages, 8, 128, page, fmt)
    c.poison()
    used = c.table < c.cache.pages - 40
    c.table[used] += pages - 40
    if rows == 200:
        many(c)
    c.fill()
    check_sample(c, 10)
    lens = [n for _, n in c.seqs]
    K = torch.zeros((sum(lens), 8 * 128), device=DEV)
    V = torch.zeros_like(K)
    spl.spl_kv_read(K, V, c.cache, c.batch(), i32([0, lens[0], sum(lens)]))
    for got, which in ((K, "k"), (V, "v")):
        want = np.concatenate([c.stored(which, b) for b in range(2)]).reshape(-1, 8 * 128)
        assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("rows", [1, 60, 300])
def test_calls_follow_the_stream_they_are_given(spl, rows):
    """Queries, cache and lengths made on a stream that is still busy, by argument and as the current stream."""
    c = Case(spl, [(rows, 600), (rows, 500)], (8, 2, 128), "i8", 64, seed=9)
    c.fill()
    if rows == 300:
        many(c)
    want = c.attend()
    K, V = (torch.as_tensor(np.concatenate([x[n - r:] for x, (r, n) in zip(xs, c.seqs)]).reshape(c.rows, -1)).to(DEV)
            for xs in (c.k, c.v))
    q = torch.as_tensor(c.q.reshape(c.rows, -1)).to(DEV)
    batch = c.batch()
    good = batch.kv_len.clone()
    torch.cuda.synchronize()
    for given in (False, True):
        s = torch.cuda.Stream()
        out, late = torch.zeros_like(q), torch.zeros_like(q)
        for b, (r, n) in enumerate(c.seqs):  # the new tokens' slots hold something else until the append
            for pos in range(n - r, n):
                c.cache.k[int(c.table[b, pos // 64]), :, pos % 64] = 0
        batch.kv_len.fill_(3)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)
            batch.kv_len.copy_(good)
            late.copy_(q)
            if not given:
                spl.spl_kv_append(c.cache, batch, K, V)
                spl.spl_paged_attention(out, late, c.cache, batch, c.hq)
        if given:
            spl.spl_kv_append(c.cache, batch, K, V, stream=s)
            spl.spl_paged_attention(out, late, c.cache, batch, c.hq, stream=s)
        s.synchronize()
        assert np.array_equal(out.cpu().numpy().reshape(want.shape), want)


def test_verify_on_another_stream_and_long_rows(spl):
    """Rows whose offsets pass 2^31 elements; probabilities made on a stream that is still busy."""
    vocab, rows = 151936, 14200
    P = torch.zeros((rows, vocab), device=DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    counts = [3, 2]
    p, q, x, u, e = draws(5, counts, vocab)
    dev = lambda t: torch.as_tensor(t).to(DEV)  # noqa: E731
    dp, dq, dx, du, de = dev(p), dev(q), dev(x), dev(u), dev(e)
    accepted, token = i32([-9, -9, -9]), i32([-9, -9, -9])
    de = torch.cat([de[:1], de])
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        P[rows - 7:].copy_(dp)
        spl.spl_verify_drafts(accepted, token, P, dq, dx, du, de, i32([0, rows - 7, rows - 3, rows]), i32([0, 0, 3, 5]))
    s.synchronize()
    want = expected(p, q, x, u, np.concatenate([e[:1], e])[1:], counts)
    assert accepted.cpu().tolist()[1:] == want[0] and token.cpu().tolist()[1:] == want[1]


@pytest.mark.parametrize("vocab,pad", [(997, 0), (4096, 0), (70001, 3)])
@pytest.mark.parametrize("kind", ["near", "extreme"])
def test_verify_chooses_the_rounded_quotient(spl, kind, vocab, pad):
    """The draw is the largest fl32(w / e), the lowest index of equal ones: quotients that differ by few ulp or not at
    all, and random numbers and weights at the ends of the range (zero, subnormal, infinite, NaN)."""
    g = np.random.default_rng(vocab)
    n = 24
    if kind == "near":
        e = (1.0 + g.integers(0, 64, (n, vocab)) * 2.0 ** -20).astype(np.float32)
        p = (e * np.float32(0.37) * (1 + g.integers(-2, 3, (n, vocab)) * 2.0 ** -23)).astype(np.float32)
    else:
        ends = np.array([0.0, 1e-45, 1e-39, 1.2e-38, 1e-30, 1e-3, 0.5, 1.0, 3.0, 1e20, 1e37, 3e38, np.inf, np.nan], np.float32)
        e = ends[g.integers(0, len(ends), (n, vocab))]
        p = ends[g.integers(0, 9, (n, vocab))]
        e[: n // 2] = np.where(e[: n // 2] < 1e-3, np.float32(1.0), e[: n // 2])  # without overflow and 0 / 0
        p[: n // 4] *= np.float32(1e-38)
    with np.errstate(all="ignore"):
        r = (p / e).astype(np.float32)
    want = np.argmax(np.where(r >= 0, r, -1), axis=1)
    got = run_verify(spl, p, np.zeros((0, vocab), np.float32), np.zeros(0, np.int32), np.zeros(0, np.float32), e, [0] * n, pad)
    assert got == ([0] * n, want.tolist())


@pytest.mark.parametrize("heads", [(8, 8, 128), (3, 3, 64)], ids=str)
def test_int8_codes_are_the_rounded_quotients(spl, heads):
    """Values on and next to the middles of two codes, vectors at the ends of the range."""
    c = Case(spl, [(1, 700)], heads, "i8", 16, seed=21)
    g = np.random.default_rng(4)
    n, (hk, d) = 700, (c.hk, c.d)
    for x in (c.k[0], c.v[0]):
        x[:] = (g.integers(-126, 126, (n, hk, d)) + 0.5) * (1 + g.integers(-3, 4, (n, hk, d)) * 2.0 ** -23)
        x[..., 0] = 127.0  # the scale is 1: the quotients are x
        x[100:] *= g.uniform(0.5, 2.0, (n - 100, hk, 1)).astype(np.float32)
        x[300:330] *= np.float32(1e-38)
        x[330:360] *= np.float32(1e-43)
        x[360:390] = np.where(np.abs(x[360:390]) > 1, x[360:390] * np.float32(1e36), x[360:390])
        x[390:400] = 0.0
    c.fill()
    for which in ("k", "v"):
        code, scale = serving.quantize_i8(getattr(c, which)[0])
        t = np.arange(n)
        page = torch.as_tensor(c.table[0, t // 16].astype(np.int64)).to(DEV)
        at = torch.as_tensor(t % 16).to(DEV)
        assert np.array_equal(getattr(c.cache, which)[page, :, at].cpu().numpy(), code)
        assert np.array_equal(getattr(c.cache, which + "_scale")[page, :, at].cpu().numpy(), scale)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("count", [13, 64, 300])
@pytest.mark.parametrize("rows", [1, 3, 40])
def test_batches_of_many_lengths(spl, rows, count, fmt):
    """Shares of blocks that begin and end anywhere: many short tiles beside long ones, sequences without rows or tokens."""
    g = np.random.default_rng(100 * rows + count)
    seqs = []
    for i in range(count):
        n = int(g.integers(0, (40, 200, 3000)[i % 3]))
        r = 0 if i % 7 == 3 else int(g.integers(1, rows + 1))
        seqs.append((min(r, n) if i % 5 else r, n))
    c = Case(spl, seqs, (8, 2, 64) if rows == 3 else (4, 2, 128), fmt, 32, seed=count)
    c.fill()
    check_sample(c, 3)
    many(c)
    check_sample(c, 2, window=int(g.integers(1, 300)))


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (4, 2, 128)], ids=str)
def test_many_rows_of_as_many_sequences_as_there_may_be(spl, heads, fmt):
    """The prefix sums of 4096 sequences lie where the first copies of keys and values go."""
    g = np.random.default_rng(heads[2])
    seqs = [(int(r), int(r + n)) for r, n in zip(g.integers(1, 3, 4096), g.integers(0, 40, 4096))]
    seqs[0] = seqs[-1] = (40, 500)
    c = many(Case(spl, seqs, heads, fmt, 16, seed=heads[2]))
    c.fill()
    got = check_sample(c, 1)
    for _ in range(3):
        assert np.array_equal(c.attend(), got)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 2, 128)], ids=str)
@pytest.mark.parametrize("rows,keys", [(150, 1200), (33, 2500)])
def test_many_rows_scores_and_values_that_grow_together(spl, rows, keys, heads, fmt):
    """In every tile of 128 keys the scores pass the maximum before it and the values (their scales) those before them, so
    that a tile's sums are rescaled for both."""
    c = many(Case(spl, [(rows, keys)], heads, fmt, 64, seed=rows))
    tile = (np.arange(keys) // 128)[:, None, None]
    c.q = (c.q * 0.25 + 1.0).astype(np.float32)
    c.k[0] = (c.k[0] * 0.25 + 0.6 * (64 / c.d) ** 0.5 * tile).astype(np.float32)  # steps of some 7 powers of two
    c.v[0] *= np.exp2(3.0 * (tile % 8)).astype(np.float32)
    c.fill()
    check_sample(c, 24)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("dim", [64, 128])
def test_long_runs_of_sequences_without_keys(spl, dim, fmt):
    """Units of which no key is copied, by the hundred, before, between and behind those that have some."""
    seqs = [(1, 300 if b in (700, 701, 1900) else 0) for b in range(3000)]
    c = Case(spl, seqs, (4, 2, dim), fmt, 16, seed=dim)
    c.fill()
    for _ in range(3):
        got = check_sample(c, 1)
        assert np.all(got[[b for b, (_, n) in enumerate(seqs) if n == 0]] == 0)


@pytest.mark.parametrize("vocab", [2 ** 31 - 1, 2 ** 31 - 4])
def test_verify_draws_again_from_the_longest_row(spl, vocab):
    """A draft that is rejected where p is nowhere above q, over as many entries as there may be: the second draw's indexes
    reach 2^31."""
    P, e = torch.zeros((2, vocab), device=DEV), torch.ones((1, vocab), device=DEV)
    P[0, 7] = 0.25
    P[0, vocab - 2:] = 0.5
    accepted, token = i32([-9]), i32([-9])
    spl.spl_verify_drafts(accepted, token, P, P[:1], i32([7]), torch.ones(1, device=DEV), e, i32([0, 2]), i32([0, 1]))
    assert accepted.tolist() == [0] and token.tolist() == [vocab - 2]
    assert spl.spl_get_device_status() == spl.SPL_OK
    del P, e
    torch.cuda.empty_cache()


def bits(t):
    """For comparisons in which a NaN equals itself."""
    return t.view(torch.int16) if t.dtype is torch.float16 else t


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("window", [0, 2, 30])
def test_a_length_past_the_table(spl, window, fmt):
    """Rows stand where the length says, not where the table ends: those past it are not written (nor any earlier token
    overwritten), and see the keys that there are."""
    for kernel in (lambda c: c, many):
        c = kernel(Case(spl, [(6, 80), (2, 20)], (4, 2, 64), fmt, 16, seed=6))
        c.table = np.ascontiguousarray(c.table[:, :5])  # room for 80 tokens
        c.fill()
        batch = c.batch()
        batch.kv_len.copy_(i32([83, 20]))
        c.batch = lambda all_rows=False, batch=batch: batch
        got = c.attend(window)
        assert spl.spl_get_device_status() == spl.SPL_EINVAL
        k, v = c.stored("k", 0), c.stored("v", 0)
        for i in range(6):
            lo, hi = serving.visible(77 + i, 80, window)
            q = c.q[i:i + 1]
            ref, mass = serving.attention(q, k[lo:hi], v[lo:hi], hi - lo, 2, 0.125)
            assert np.all(np.abs(got[i] - ref[0]) <= tolerance(q, k[lo:hi], 0.125, hi - lo, 2, mass)[0]), i
        assert window != 2 or np.all(got[5] == 0)  # position 82 sees 81 and 82
        before = bits(c.cache.k).clone()
        x = torch.randn((8, 128), device=DEV)
        spl.spl_kv_append(c.cache, batch, x, x)
        assert spl.spl_get_device_status() == spl.SPL_EINVAL
        changed = (bits(c.cache.k) != before).any(-1).any(1).nonzero().tolist()
        want = [[int(c.table[b, p // 16]), p % 16] for b, p in ((0, 77), (0, 78), (0, 79), (1, 18), (1, 19))]
        assert sorted(changed) == sorted(want)


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("length", [-1, -3, -2 ** 31])
def test_a_negative_length_is_reported(spl, length, fmt):
    c = Case(spl, [(3, 40), (2, 20)], (4, 2, 64), fmt, 16, seed=6)
    c.fill()
    want = c.check()
    before = bits(c.cache.k).clone()
    batch = c.batch()
    batch.kv_len.copy_(i32([length, 20]))
    c.batch = lambda all_rows=False: batch
    x = torch.zeros((5, 128), device=DEV)
    K, V = torch.full((60, 128), 3.0, device=DEV), torch.full((60, 128), 3.0, device=DEV)
    spl.spl_kv_read(K, V, c.cache, batch, i32([0, 40, 60]))
    assert spl.spl_get_device_status() == spl.SPL_EINVAL
    assert bool((K[:40] == 3.0).all()) and not bool((K[40:] == 3.0).any())
    for kernel in (lambda c: c, many):
        got = kernel(c).attend()
        assert spl.spl_get_device_status() == spl.SPL_EINVAL
        assert np.all(got[:3] == 0) and np.allclose(got[3:], want[3:], rtol=0, atol=1e-5)
    spl.spl_kv_append(c.cache, batch, x, x)
    assert spl.spl_get_device_status() == spl.SPL_EINVAL
    slots = {tuple(t) for t in (bits(c.cache.k) != before).any(-1).any(1).nonzero().tolist()}
    assert slots == {(int(c.table[1, 1]), 2), (int(c.table[1, 1]), 3)}


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("page", [16, 64, 128, 256])
@pytest.mark.parametrize("window", [0, 200])
def test_keys_on_pages_outside_the_pool_are_hidden(spl, window, page, fmt):
    """Both kernels leave out the keys of a page whose id is outside the pool, as if they were not visible."""
    for kernel in (lambda c: c, many):
        c = kernel(Case(spl, [(40, 1000), (3, 150), (130, 130)], (4, 2, 64), fmt, page, seed=page))
        c.fill()
        gone = [np.zeros(n, dtype=bool) for _, n in c.seqs]
        for b, at, bad in ((0, 3, -5), (0, 1000 // page, 1 << 30), (0, 900 // page, -1), (1, 0, c.cache.pages), (2, 0, -2 ** 31)):
            c.table[b, at] = bad
            gone[b][at * page:(at + 1) * page] = True
        got = c.attend(window)
        assert spl.spl_get_device_status() == spl.SPL_EINVAL
        for b, (r, n) in enumerate(c.seqs):
            k, v = c.stored("k", b), c.stored("v", b)
            for i in range(0, r, 1 if r < 40 else 7):
                lo, hi = serving.visible(n - r + i, n, window)
                q, mine = c.q[c.start[b] + i:c.start[b] + i + 1], got[c.start[b] + i]
                at = np.flatnonzero(~gone[b][lo:hi]) + lo
                if len(at) == 0:
                    assert np.all(mine == 0)
                    continue
                ref, mass = serving.attention(q, k[at], v[at], len(at), 2, 0.125)
                tol = tolerance(q, k[at], 0.125, n, 2, mass)[0] + 2.0 ** -32 * n * np.max(np.abs(v))
                assert np.all(np.abs(mine - ref[0]) <= tol), (b, i)
        assert spl.spl_get_device_status() == spl.SPL_OK


@pytest.mark.parametrize("fmt", ["f16", "i8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scale", [0.0, None])
def test_errors_do_not_grow_with_the_length(spl, scale, dim, fmt):
    """131072 keys in one block's piece (as many sequences as SMs, all of them on the same pages), with values whose sums
    grow.  Relative to the output a chain of 16 keys truncates at most 2^-22 of its size (1.2 times the output's share);
    of the 1024 sums of each of 8 warps, rounded to nearest, the errors add up as sqrt(1024 / 3 / 8) 2^-24 / sqrt(3), three of
    them 7e-7; exp is within 2^-21 and a probability's halves within 2^-22, of either sign: 1.5e-6 in all."""
    keys, page = 131072, 256
    seqs = torch.cuda.get_device_properties(0).multi_processor_count
    c = Case(spl, [(1, keys)], (4, 1, dim), fmt, page, seed=dim)
    c.fill()
    g = np.random.default_rng(1)
    q = g.standard_normal((seqs, 4 * dim)).astype(np.float32)
    batch = spl.KVBatch(i32(list(range(seqs + 1))), i32([keys] * seqs),
                        torch.as_tensor(np.repeat(c.table[:, :keys // page], seqs, axis=0)).to(DEV), seqs, 1)
    out = torch.empty((seqs, 4 * dim), device=DEV)
    spl.spl_paged_attention(out, torch.as_tensor(q).to(DEV), c.cache, batch, 4, scale=scale)
    got = out.cpu().numpy().reshape(seqs, 4, dim)
    k, v = c.stored("k", 0), c.stored("v", 0)
    for b in (0, seqs // 2, seqs - 1):
        ref, _ = serving.attention(q[b].reshape(1, 4, dim), k, v, keys, 4, 1 / np.sqrt(dim) if scale is None else scale)
        err = np.linalg.norm(got[b] - ref[0]) / np.linalg.norm(ref)
        assert err < 1.5e-6, f"sequence {b}: {err:.3g}"
    assert spl.spl_get_device_status() == spl.SPL_OK


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("small,large", [(0.0, 1e12), (1e-20, 1e12), (1e-30, 1e9), (0.0, 1e25), (1e25, 0.0)])
def test_int8_values_of_very_different_sizes(spl, small, large, dim):
    """The first half of the keys have values far smaller than the second (or none): their weight counts all the same, also
    where other blocks have them."""
    for kernel in (lambda c: c, many):
        c = kernel(Case(spl, [(200, 6000)], (4, 1, dim), "i8", 64, seed=dim))
        c.v[0][:3000] *= np.float32(small)
        c.v[0][3000:] *= np.float32(large)
        c.fill()
        for scale in (0.0, None):
            check_sample(c, 12, scale=scale)


@pytest.mark.parametrize("rows", [1, 3, 200])
@pytest.mark.parametrize("dim", [64, 128])
def test_int8_values_next_to_the_largest(spl, rows, dim):
    """Values of some 1e34, whose sums in units of 2^-13 would pass fp32's range: outputs are as large as the values."""
    for kernel in (lambda c: c, many):
        c = kernel(Case(spl, [(rows, 3000), (rows, 700)], (4, 2, dim), "i8", 64, seed=rows))
        for v in c.v:
            v *= np.float32(1e34)
        c.fill()
        got = check_sample(c, 12)
        assert np.isfinite(got).all()


def test_a_piece_that_takes_longer_than_a_wait_may(spl):
    """2^27 keys (on the same few pages) for every block: some warps have nothing to do for more than a second, and wait.
    All scores are 0 and the values small integers, the same for every key: every sum but a row's last ones is exact."""
    keys, page, dim = 1 << 27, 256, 64
    rows = 128 * torch.cuda.get_device_properties(0).multi_processor_count
    cache = spl.KVCache.empty(4, 1, dim, page, "f16")
    v = torch.arange(dim, device=DEV) - 20.0
    cache.k.fill_(1.0)
    cache.v.copy_(v.expand_as(cache.v))
    table = i32([[3, 1, 0, 2] * (keys // (4 * page))])
    q, out = torch.ones((rows, dim), device=DEV), torch.empty((rows, dim), device=DEV)
    spl.spl_paged_attention(out, q, cache, spl.KVBatch(i32([0, rows]), i32([keys]), table, rows), 1, scale=0.0)
    assert spl.spl_get_device_status() == spl.SPL_OK
    assert bool(((out - v).abs() <= 2.0 ** -21 * v.abs()).all())  # the last sum, the total's, the quotient, the product
