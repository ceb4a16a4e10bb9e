"""The serving operators' refusals and empty calls, which need no GPU, and the oracle against closed forms."""

import collections
import ctypes
import os

import numpy as np
import pytest

from oracle import serving


@pytest.fixture(scope="module")
def spl():
    from paper_2609_15039_gb300 import build, spl as binding
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    binding.lib()
    return binding


@pytest.fixture(scope="module")
def base():
    buf = (ctypes.c_float * 64)()
    p = ctypes.cast(buf, ctypes.c_void_p).value
    yield p + (16 - p % 16) % 16
    del buf


def cache_of(spl, base, **kw):
    f = dict(k=base, v=base, k_scale=base, v_scale=base, pages=4, kv_heads=2, page_size=16, head_dim=64, format=1)
    f.update(kw)
    return spl.spl_kv_cache(*f.values())


def batch_of(spl, base, **kw):
    f = dict(row_start=base, kv_len=base, page_table=base, seqs=2, max_pages=2, max_rows=1)
    f.update(kw)
    return spl.spl_kv_batch(*f.values())


CACHES = [({"format": 2}, "EINVAL"), ({"pages": -1}, "EINVAL"), ({"kv_heads": 0}, "EINVAL"), ({"k": None}, "EINVAL"),
          ({"v_scale": None}, "EINVAL"), ({"head_dim": 96}, "ESHAPE"), ({"page_size": 48}, "ESHAPE"),
          ({"page_size": 8}, "ESHAPE"), ({"page_size": 512}, "ESHAPE"), ({"kv_heads": 1025}, "ESHAPE"),
          ({"pages": 1 << 26}, "ESHAPE"), ({"pages": 1 << 40}, "ESHAPE"), ({"k": 8}, "EALIGN"), ({"k_scale": 4}, "EALIGN")]
BATCHES = [({"seqs": -1}, "EINVAL"), ({"max_rows": -1}, "EINVAL"), ({"row_start": None}, "EINVAL"),
           ({"page_table": None}, "EINVAL"), ({"seqs": 4097}, "ESHAPE"), ({"max_pages": 1 << 27}, "ESHAPE"),
           ({"max_pages": 1 << 60}, "ESHAPE"), ({"kv_len": 2}, "EALIGN")]


def shifted(fields, base):
    """Small numbers in place of pointers are offsets."""
    pointers = ("k", "v", "k_scale", "v_scale", "row_start", "kv_len", "page_table")
    return {n: base + v if n in pointers and v else v for n, v in fields.items()}


def every(spl, cache, batch, p):
    """The three operators' answers to one cache and batch."""
    L = spl.lib()
    c, b = (ctypes.byref(x) if x is not None else None for x in (cache, batch))
    return (L.spl_kv_append(c, b, p, 128, p, 128, 2, None), L.spl_kv_read(p, p, c, b, p, 2, None),
            L.spl_paged_attention(p, 256, p, 256, c, b, 2, 4, 1.0, 0, p, 1 << 40, None))


@pytest.mark.parametrize("fields,error", CACHES, ids=str)
def test_caches_that_are_refused(spl, base, fields, error):
    want = getattr(spl, "SPL_" + error)
    assert every(spl, cache_of(spl, base, **shifted(fields, base)), batch_of(spl, base), base) == (want,) * 3


@pytest.mark.parametrize("fields,error", BATCHES, ids=str)
def test_batches_that_are_refused(spl, base, fields, error):
    want = getattr(spl, "SPL_" + error)
    assert every(spl, cache_of(spl, base), batch_of(spl, base, **shifted(fields, base)), base) == (want,) * 3


def test_null_structs_and_empty_calls(spl, base):
    L, c, b = spl.lib(), cache_of(spl, base), batch_of(spl, base)
    assert every(spl, None, b, base) == (spl.SPL_EINVAL,) * 3
    assert every(spl, c, None, base) == (spl.SPL_EINVAL,) * 3
    c, b, none = ctypes.byref(c), ctypes.byref(b), ctypes.byref(batch_of(spl, None, seqs=0, max_pages=0))
    assert L.spl_kv_append(c, b, None, 0, None, 0, 0, None) == spl.SPL_OK
    assert L.spl_kv_append(c, none, None, 0, None, 0, 0, None) == spl.SPL_OK
    assert L.spl_kv_read(None, None, c, b, None, 0, None) == spl.SPL_OK
    assert L.spl_paged_attention(None, 0, None, 0, c, b, 0, 4, 1.0, 0, None, 0, None) == spl.SPL_OK
    assert L.spl_paged_attention(None, 0, None, 0, c, none, 0, 4, 1.0, 0, None, 0, None) == spl.SPL_OK
    assert L.spl_verify_drafts(None, None, None, 0, None, 0, None, None, None, 0, None, None, 0, 0, 0, 9, None, 0,
                               None) == spl.SPL_OK


def test_rows_that_are_refused(spl, base):
    L, c, b = spl.lib(), ctypes.byref(cache_of(spl, base)), ctypes.byref(batch_of(spl, base))
    append = lambda k, ldk, v, ldv, rows: L.spl_kv_append(c, b, k, ldk, v, ldv, rows, None)  # noqa: E731
    assert append(None, 128, base, 128, 2) == spl.SPL_EINVAL
    assert append(base, 124, base, 128, 2) == spl.SPL_EINVAL
    assert append(base, 128, base, 128, -1) == spl.SPL_EINVAL
    assert append(base, 130, base, 128, 2) == spl.SPL_EALIGN
    assert append(base, 128, base + 4, 128, 2) == spl.SPL_EALIGN
    assert append(base, 128, base, 128, 1 << 33) == spl.SPL_ESHAPE
    read = lambda k, start, rows: L.spl_kv_read(k, base, c, b, start, rows, None)  # noqa: E731
    assert read(None, base, 2) == spl.SPL_EINVAL and read(base, None, 2) == spl.SPL_EINVAL
    assert read(base, base, -2) == spl.SPL_EINVAL and read(base, base, 1 << 33) == spl.SPL_ESHAPE
    assert read(base + 8, base, 2) == spl.SPL_EALIGN and read(base, base + 2, 2) == spl.SPL_EALIGN


def test_attention_that_is_refused(spl, base):
    L, c, b = spl.lib(), ctypes.byref(cache_of(spl, base)), ctypes.byref(batch_of(spl, base))
    good = dict(out=base, ldo=256, Q=base, ldq=256, rows=2, heads=4, scale=1.0, window=0, ws=base, size=1 << 40)

    def call(**kw):
        a = {**good, **kw}
        return L.spl_paged_attention(a["out"], a["ldo"], a["Q"], a["ldq"], c, b, a["rows"], a["heads"], a["scale"],
                                     a["window"], a["ws"], a["size"], None)
    for kw in ({"out": None}, {"Q": None}, {"ldo": 252}, {"ldq": -256}, {"rows": -1}, {"heads": 3}, {"heads": 0},
               {"scale": float("nan")}, {"scale": float("inf")}, {"window": -1}):
        assert call(**kw) == spl.SPL_EINVAL, kw
    for kw in ({"rows": 1 << 60}, {"rows": 1 << 31}, {"heads": 2 * 1025}):
        assert call(**kw) == spl.SPL_ESHAPE, kw
    for kw in ({"out": base + 4}, {"Q": base + 8}, {"ldo": 258}, {"ldq": 257}, {"ws": base + 8}):
        assert call(**kw) == spl.SPL_EALIGN, kw
    need = L.spl_paged_attention_workspace_bytes(c, b, 2, 4)
    assert need >= 65536
    assert call(size=need - 1) == spl.SPL_EWORKSPACE and call(ws=None) == spl.SPL_EWORKSPACE
    assert L.spl_paged_attention_workspace_bytes(c, b, 0, 4) == 0
    assert L.spl_paged_attention_workspace_bytes(c, b, 2, 3) == 0


def test_verification_that_is_refused(spl, base):
    L = spl.lib()
    names = "accepted token P ldp Q ldq draft u e lde row_start draft_start rows drafts seqs vocab ws size".split()
    good = dict(zip(names, (base, base, base, 8, base, 8, base, base, base, 8, base, base, 3, 2, 2, 8, base, 64)))
    call = lambda **kw: L.spl_verify_drafts(*{**good, **kw}.values(), None)  # noqa: E731
    pointers = [n for n in names if good[n] == base and n != "ws"]
    for n in pointers:
        assert call(**{n: None}) == spl.SPL_EINVAL, n
        assert call(**{n: base + 2}) == spl.SPL_EALIGN, n
    for kw in ({"vocab": 0}, {"vocab": -1}, {"ldp": 7}, {"ldq": 7}, {"lde": 7}, {"rows": -1}, {"drafts": -1}, {"seqs": -1}):
        assert call(**kw) == spl.SPL_EINVAL, kw
    big = {"ldp": 1 << 32, "ldq": 1 << 32, "lde": 1 << 32}
    for kw in ({"seqs": 4097}, {"rows": 1 << 31}, {"drafts": 1 << 31}, {"vocab": 1 << 31, **big}):
        assert call(**kw) == spl.SPL_ESHAPE, kw
    need = L.spl_verify_drafts_workspace_bytes(2)
    assert call(size=need - 1) == spl.SPL_EWORKSPACE and call(ws=None) == spl.SPL_EWORKSPACE
    assert call(ws=base + 8) == spl.SPL_EALIGN


# ---------------------------------------------------------------------------------- the oracle
def test_oracle_attention_closed_forms():
    """Equal scores average the visible values; one key gives its value; a window and missing keys."""
    v = np.arange(5.0)[:, None, None] * np.ones((1, 1, 4))
    q, k = np.zeros((3, 1, 4)), np.ones((5, 1, 4))
    out, mass = serving.attention(q, k, v, 5, 1, 1.0)
    assert np.allclose(out[:, 0, 0], [1.0, 1.5, 2.0]) and np.allclose(mass, out)
    out, _ = serving.attention(q, k, v, 5, 1, 1.0, window=2)
    assert np.allclose(out[:, 0, 0], [1.5, 2.5, 3.5])
    out, _ = serving.attention(q, k[:1], v[:1] + 7, 1, 1, 1.0)
    assert np.allclose(out[:, 0, 0], [0, 0, 7])


def test_oracle_quantisation():
    x = np.array([[1.0, -2.0, 0.5], [0.0, 0.0, 0.0], [np.inf, 1.0, 2.0]], dtype=np.float32)
    code, scale = serving.quantize_i8(x)
    assert code[0].tolist() == [64, -127, 32] and scale[0] == np.float32(2.0) / np.float32(127.0)
    assert scale[1] == 0 and not code[1].any() and np.isnan(scale[2])
    assert serving.quantize_f16(np.float32([1e6, -1e6, 0.1])).tolist() == [65504.0, -65504.0, np.float16(0.1)]


def test_oracle_verification_keeps_the_target_distribution():
    """Exact: the token that follows a draft is distributed as p, whatever q (the race's choice by inversion)."""
    g = np.random.default_rng(0)
    p, q = g.dirichlet(np.ones(6)), g.dirichlet(np.ones(6))
    accept = np.minimum(1.0, p / q)
    rest = np.maximum(p - q, 0)
    assert np.allclose(q * accept + (1 - q @ accept) * rest / rest.sum(), p)
    n, token = serving.verify(np.stack([p, p]), q[None], [2], [0.0], 1 / np.arange(1.0, 7.0))
    assert n == 1 and token == int(np.argmax(p * np.arange(1.0, 7.0)))


def test_pages_are_taken_and_given_back(monkeypatch):
    import torch
    from paper_2609_15039_gb300 import serving
    made = []
    monkeypatch.setattr(serving.spl, "KVBatch", lambda *a: made.append(a) or made[-1])
    monkeypatch.setattr(torch.Tensor, "cuda", lambda self: self)
    p = serving.Pages(pages=5, page_size=16, seqs=2, max_len=48)
    start, lens, table, rows, most = p.grow([17, 16])
    assert start.tolist() == [0, 17, 33] and lens.tolist() == [17, 16] and (rows, most) == (33, 17)
    assert len(p.free) == 2 and len(set(p.own[0] + p.own[1])) == 3
    assert table[0, :2].tolist() == p.own[0] and table[1, 0] == p.own[1][0]
    p.grow([0, 1])
    p.cut([16, 16])
    assert p.lens == [16, 16] and len(p.free) == 3
    with pytest.raises(ValueError):
        p.grow([0, 33])  # past the table
    p.grow([32, 0])
    with pytest.raises(ValueError):
        p.grow([0, 17])  # no page left


Batch = collections.namedtuple("Batch", "row_start kv_len table rows max_rows")


class Slots:
    """A decoder that only keeps which token lies in which slot, and looks that its sequences find their own."""

    def __init__(self, pages, vocab):
        import torch
        self.pages, self.vocab, self.held = pages, vocab, {}
        self.embedding = torch.zeros((vocab, 1))
        self.seen = [[] for _ in pages.lens]

    def at(self, b, pos):
        size = self.pages.page_size
        return int(self.pages.table[b, pos // size]), pos % size

    def forward(self, tokens, batch):
        import torch
        start, lens = batch.row_start.tolist(), batch.kv_len.tolist()
        for b, n in enumerate(lens):
            new = tokens[start[b]:start[b + 1]].tolist()
            self.seen[b] = self.seen[b][:n - len(new)] + new
            for i, t in enumerate(new):
                self.held[self.at(b, n - len(new) + i)] = (b, t)
        for b, n in enumerate(lens):
            assert [self.held.get(self.at(b, i)) for i in range(n)] == [(b, t) for t in self.seen[b][:n]]
        return torch.zeros((len(tokens), self.vocab))


@pytest.mark.parametrize("prompts,page", [([14] * 4, 16), ([62] * 8, 64), ([16, 15, 14, 13, 12], 16)], ids=str)
def test_drafts_and_target_find_their_own_tokens(monkeypatch, prompts, page):
    """Sequences that pass the end of a page in one round: whatever is accepted, each finds its own tokens in its slots,
    in the draft's cache as in the target's."""
    import torch
    from paper_2609_15039_gb300 import serving
    g = torch.Generator()
    g.manual_seed(5)
    monkeypatch.setattr(serving.spl, "KVBatch", Batch)
    monkeypatch.setattr(torch.Tensor, "cuda", lambda self: self)

    def verify(accepted, token, P, Q, x, u, e, row_start, draft_start):
        accepted.copy_(torch.randint(0, 5, accepted.shape, generator=g))
        token.copy_(torch.randint(0, P.shape[1], token.shape, generator=g))

    monkeypatch.setattr(serving.spl, "spl_verify_drafts", verify)
    n, count = len(prompts), len(prompts) * -(-200 // page)
    pages = serving.Pages(count, page, n, 200)
    target, draft = Slots(pages, 1000), Slots(pages, 1000)
    out, history = serving.generate(target, draft, pages, [[100 * b + i for i in range(m)] for b, m in enumerate(prompts)],
                                    drafts=4, rounds=12)
    lens = [m + len(o) - 1 for m, o in zip(prompts, out)]
    assert pages.lens == lens and len(history) == 12
    assert len(pages.free) == count - sum(-(-m // page) for m in lens)


def test_a_batch_without_room_takes_nothing(monkeypatch):
    """A batch that does not fit is refused as a whole: no sequence has grown, no page is gone."""
    import torch
    from paper_2609_15039_gb300 import serving
    monkeypatch.setattr(serving.spl, "KVBatch", Batch)
    monkeypatch.setattr(torch.Tensor, "cuda", lambda self: self)
    p = serving.Pages(pages=3, page_size=16, seqs=2, max_len=48)
    p.grow([5, 5])
    for new in ([17, 33], [28, 28], [1, 44]):  # pages of both, of the second alone, past the table
        with pytest.raises(ValueError):
            p.grow(new)
        assert p.lens == [5, 5] and len(p.free) == 1 and [len(o) for o in p.own] == [1, 1]
    assert p.grow([27, 11]).kv_len.tolist() == [32, 16]


def test_generation_without_drafts(monkeypatch):
    """No drafts: a token a round, by the target alone."""
    import torch
    from paper_2609_15039_gb300 import serving
    monkeypatch.setattr(serving.spl, "KVBatch", Batch)
    monkeypatch.setattr(torch.Tensor, "cuda", lambda self: self)

    def verify(accepted, token, P, Q, x, u, e, row_start, draft_start):
        assert Q.shape == (0, 50) and x.numel() == u.numel() == 0 and draft_start.tolist() == [0, 0, 0]
        accepted.zero_()
        token.copy_(P.argmax(-1))

    monkeypatch.setattr(serving.spl, "spl_verify_drafts", verify)
    pages = serving.Pages(8, 16, 2, 64)
    out, history = serving.generate(Slots(pages, 50), Slots(pages, 50), pages, [[1, 2, 3], [4]], drafts=0, rounds=5)
    assert [len(o) for o in out] == [6, 6] and history == [[0, 0]] * 5 and pages.lens == [8, 6]


def test_an_empty_prompt_is_refused(monkeypatch):
    """It has no row whose logits its first token could follow."""
    import torch
    from paper_2609_15039_gb300 import serving
    monkeypatch.setattr(serving.spl, "KVBatch", Batch)
    monkeypatch.setattr(torch.Tensor, "cuda", lambda self: self)
    for prompts in ([[1, 2, 3], []], [[], [4]]):
        pages = serving.Pages(8, 16, 2, 64)
        with pytest.raises(ValueError):
            serving.generate(Slots(pages, 50), Slots(pages, 50), pages, prompts, drafts=0, rounds=0)
        assert pages.lens == [0, 0] and len(pages.free) == 8


def test_an_unknown_format_is_refused(spl):
    for name in ("int8", "fp16", None):
        with pytest.raises(ValueError):
            spl.KVCache.empty(1, 1, 64, 16, name)
