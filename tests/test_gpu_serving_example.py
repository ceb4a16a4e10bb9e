"""Generation with the paged cache and drafted tokens, end to end on the GPU."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def serving():
    from paper_2609_15039_gb300 import serving, spl
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    spl.lib()
    return serving


def plain(decoder, tokens):
    """The logits of one sequence's tokens in 64 bits, without cache or masks."""
    d = decoder.head_dim
    x = decoder.embedding[torch.tensor(tokens)].double().cpu().numpy()
    norm = lambda t: t / np.sqrt((t * t).mean(-1, keepdims=True) + 1e-6)  # noqa: E731
    for layer in decoder.layers:
        w = {g.name: g.W.double().cpu().numpy() for g in layer.groups}
        y = norm(x) @ w["qkv"].T
        q1 = layer.group("qkv").columns("q")[1]
        q = y[:, :q1].reshape(len(tokens), -1, d)
        k, v = (y[:, slice(*layer.group("qkv").columns(n))].reshape(len(tokens), -1, d) for n in "kv")
        group = q.shape[1] // k.shape[1]
        mixed = np.zeros_like(q)
        for h in range(q.shape[1]):
            s = q[:, h] @ k[:, h // group].T / np.sqrt(d)
            s = np.where(np.tril(np.ones_like(s)) > 0, s, -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            mixed[:, h] = p / p.sum(1, keepdims=True) @ v[:, h // group]
        x = x + mixed.reshape(len(tokens), -1) @ w["o"].T
        gate, up = np.split(norm(x) @ w["gateup"].T, 2, axis=1)
        x = x + (gate / (1 + np.exp(-gate)) * up) @ w["down"].T
    return norm(x) @ decoder.head.double().cpu().numpy().T


@pytest.mark.parametrize("eps", [float("inf"), 8.0])
def test_chunks_give_the_logits_of_the_whole(serving, eps):
    """A prompt in ragged chunks, one token at a time at the end, against all of it at once in 64 bits.  The cache's
    binary16 rounds keys and values by 2^-12 each; through two layers of a few sums of unit size that leaves the logits
    (of size 4) within 1e-2, with masks or without."""
    target, _, pages = serving.synthetic(2, seqs=3, max_len=320, eps=eps)
    g = np.random.default_rng(3)
    tokens = [g.integers(0, 1024, n).tolist() for n in (300, 151, 64)]
    got = [[], [], []]
    at = [0, 0, 0]
    for new in ((130, 151, 1), (1, 0, 0), (167, 0, 60), (1, 0, 1), (1, 0, 1), (0, 0, 1)):
        batch = pages.grow(list(new))
        flat = [t for b, n in enumerate(new) for t in tokens[b][at[b]:at[b] + n]]
        logits = target.forward(torch.tensor(flat, device="cuda"), batch).cpu().numpy()
        start = 0
        for b, n in enumerate(new):
            got[b].append(logits[start:start + n])
            start, at[b] = start + n, at[b] + n
    for b, t in enumerate(tokens):
        assert at[b] == len(t)
        assert np.max(np.abs(np.concatenate(got[b]) - plain(target, t))) < 1e-2
    from paper_2609_15039_gb300 import spl
    assert spl.spl_get_device_status() == spl.SPL_OK


def test_a_decoder_accepts_its_own_drafts(serving):
    """With the decoder itself as draft the two distributions differ by rounding alone: all drafts are accepted, and
    the pages end up as the kept tokens need them."""
    target, _, pages = serving.synthetic(1, seqs=4, max_len=200, formats=("f16", "f16"))
    total = len(pages.free)
    prompts = [list(range(b, b + n)) for b, n in enumerate((64, 1, 37, 100))]
    out, history = serving.generate(target, _, pages, prompts, drafts=3, rounds=6)
    assert sum(map(sum, history)) >= 4 * 3 * 6 - 1  # (a draw within rounding of the edge is a chance of 1e-4)
    assert [len(o) for o in out] == [1 + sum(h[b] + 1 for h in history) for b in range(4)]
    lens = [len(p) + len(o) - 1 for p, o in zip(prompts, out)]  # the last token is pending
    assert pages.lens == lens and len(pages.free) == total - sum(-(-n // 64) for n in lens)


def test_sequences_that_pass_the_end_of_a_page_together(serving):
    """Equal prompts of 62 tokens on pages of 64, and the decoder itself as draft: all drafts are accepted, so each sequence
    finds its own keys and values in both caches."""
    target, draft, pages = serving.synthetic(1, seqs=4, max_len=200, formats=("f16", "f16"))
    prompts = [list(range(100 * b, 100 * b + 62)) for b in range(4)]
    out, history = serving.generate(target, draft, pages, prompts, drafts=3, rounds=20)
    assert sum(map(sum, history)) >= 4 * 3 * 20 - 2  # (a draw within rounding of the edge is a chance of 1e-4)
    assert pages.lens == [62 + len(o) - 1 for o in out]


@pytest.mark.parametrize("layers", [1, 2])
def test_no_noise_is_drawn_twice(serving, monkeypatch, layers):
    """Blocks of the generator that hide an input, of target and draft together: none hides two."""
    target, draft, pages = serving.synthetic(layers, seqs=2, max_len=64, page_size=16, eps=8.0)
    drawn = []
    for name, at in (("spl_noise_mask", 2), ("spl_noise_mask_f64", 1)):
        def call(*args, call=getattr(serving.spl, name), at=at, offset=0):
            drawn.append((args[-1], offset, offset + -(-args[at].numel() // 4)))
            return call(*args, offset=offset)
        monkeypatch.setattr(serving.spl, name, call)
    serving.generate(target, draft, pages, [[1, 2, 3], [4]], drafts=2, rounds=2)
    assert len(drawn) == 4 * (layers * 3 + 1 * 7)
    drawn.sort()
    for (seed, _, end), (other, begin, _) in zip(drawn, drawn[1:]):
        assert seed != other or end <= begin


def test_a_smaller_draft_and_int8(serving, capsys):
    assert serving.main(["--sequences", "3", "--layers", "2", "--rounds", "5", "--prompt", "33", "--eps", "4"]) == 0
    line = capsys.readouterr().out
    assert "status SPL_OK" in line
    taken = int(line.split(" s, ")[1].split(" of ")[0])
    assert 0 < taken < 3 * 4 * 5
