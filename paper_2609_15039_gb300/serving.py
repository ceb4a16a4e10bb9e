"""Generation with a paged KV cache and drafted tokens around the masked linears.

A decoder's outsourced products run masked (noise, correction, masked product with the unmask in its
epilogue); what lies between them stays in the library's serving operators: the new tokens' keys and
values are columns of the fused Q|K|V output and go into the paged cache (spl_kv_append), the rows
attend over it (spl_paged_attention), and the masked O product follows.  ``generate`` lets a smaller
decoder propose tokens that the larger one checks in one pass of a few rows a sequence
(spl_verify_drafts): the tokens are distributed as if the larger one had sampled each by itself.

    python -m paper_2609_15039_gb300.serving --sequences 8 --drafts 4 --rounds 16

runs it on random weights and prints how many drafts were accepted.  Where the pages lie and how
long the sequences are is the host's (``Pages``); a rejected draft costs nothing but its length, its
slots are written again.
"""

import argparse
import time

import torch

from . import spl, workloads as wl
from .layer import MaskedLayer


class Pages:
    """Which pages hold which sequence.  Caches of equal page_size and pages share it (one a layer)."""

    def __init__(self, pages, page_size, seqs, max_len):
        self.page_size, self.free = page_size, list(range(pages))[::-1]
        self.lens = [0] * seqs
        self.own = [[] for _ in range(seqs)]
        self.table = torch.zeros((seqs, -(-max_len // page_size)), dtype=torch.int32)

    def grow(self, new):
        """Adds new[b] tokens to each sequence; returns the batch of those rows."""
        needs, left = [], len(self.free)
        for b, n in enumerate(new):  # all of them or none
            needs.append(-(-(self.lens[b] + n) // self.page_size))
            left -= max(0, needs[b] - len(self.own[b]))
            if needs[b] > self.table.shape[1] or left < 0:
                raise ValueError(f"Pages: no room for {n} more tokens of sequence {b}")
        for b, (n, need) in enumerate(zip(new, needs)):
            while len(self.own[b]) < need:
                page = self.free.pop()
                self.table[b, len(self.own[b])] = page
                self.own[b].append(page)
            self.lens[b] += n
        start = torch.tensor([0] + list(new)).cumsum(0).to(torch.int32)
        lens = torch.tensor(self.lens, dtype=torch.int32)
        return spl.KVBatch(start.cuda(), lens.cuda(), self.table.cuda(), int(start[-1]), max(new))

    def rewind(self, lens):
        """Drops the tokens past the given lengths; their pages stay with the sequences, for the same tokens again."""
        for b, n in enumerate(lens):
            assert n <= self.lens[b]
            self.lens[b] = n

    def cut(self, lens):
        """Drops the tokens past the given lengths, and the pages that then hold none."""
        self.rewind(lens)
        for b, n in enumerate(lens):
            while len(self.own[b]) > -(-n // self.page_size):
                self.free.append(self.own[b].pop())


class CachedDecoder:
    """Decoder layers (attention and MLP, residual, RMS-normalised inputs) with one paged cache each."""

    def __init__(self, layers, embedding, head, kv_heads, head_dim, pages, page_size, format="f16", eps=float("inf"),
                 mech="gaussian", seed=0):
        self.layers, self.embedding, self.head = layers, embedding, head
        self.kv_heads, self.head_dim = kv_heads, head_dim
        self.eps, self.mech, self.seed, self.drawn = eps, mech, seed, 0
        self.caches = [spl.KVCache.empty(pages, kv_heads, head_dim, page_size, format) for _ in layers]
        self.workspace = spl.workspace(0)

    def _room(self, nbytes):
        if self.workspace.numel() < nbytes:
            self.workspace = spl.workspace(nbytes)
        return self.workspace

    def masked(self, layer, name, x):
        """x W^T of a group, x hidden by noise that is drawn once and used once."""
        g, wide = layer.group(name), torch.float64 if name in layer.fp64 else torch.float32
        rows, offset = x.shape[0], self.drawn
        self.drawn += -(-x.numel() // 4)  # blocks of four draws
        eta, noisy = torch.empty_like(x), torch.empty_like(x, dtype=wide)
        c, y = (torch.empty((rows, g.N), device=x.device, dtype=t) for t in (wide, torch.float32))
        drawn = (layer.deltas[name], self.eps, self.mech, self.seed)
        if name in layer.fp64:  # noise far larger than the input: mask and correction in binary64
            ws = self._room(spl.spl_f64_workspace_bytes(rows, g.K, g.N))
            spl.spl_noise(eta, *drawn, offset=offset)
            spl.spl_noise_mask_f64(noisy, x, *drawn, offset=offset)
            spl.spl_precompute_noise_product_f64(c, eta, g.W, workspace=ws)
            spl.spl_masked_linear_unmask_f64(y, noisy, g.W, c, workspace=ws)
        else:
            ws = self._room(spl.spl_linear_workspace_bytes(rows, g.K, g.N))
            spl.spl_noise_mask(noisy, eta, x, *drawn, offset=offset)
            spl.spl_precompute_noise_product(c, eta, g.wt, workspace=ws)
            spl.spl_masked_linear_unmask(y, noisy, g.wt, c, workspace=ws)
        return y

    def forward(self, tokens, batch):
        """Logits [rows, vocab] of the batch's new tokens (int64 [rows]), which join the caches."""
        norm = lambda t: t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6)  # noqa: E731
        x = self.embedding[tokens]
        for layer, cache in zip(self.layers, self.caches):
            qkv, (_, q1) = layer.group("qkv"), layer.group("qkv").columns("q")
            y = self.masked(layer, "qkv", norm(x))
            k, v = (y[:, slice(*qkv.columns(n))] for n in "kv")
            spl.spl_kv_append(cache, batch, k, v)
            heads = q1 // self.head_dim
            mixed = torch.empty((x.shape[0], q1), device=x.device)
            ws = self._room(spl.spl_paged_attention_workspace_bytes(cache, batch, heads))
            spl.spl_paged_attention(mixed, y[:, :q1], cache, batch, heads, workspace=ws)
            x = x + self.masked(layer, "o", mixed)
            gate, up = self.masked(layer, "gateup", norm(x)).chunk(2, dim=1)
            x = x + self.masked(layer, "down", (torch.nn.functional.silu(gate) * up).contiguous())
        return norm(x) @ self.head.T


def sample(p, generator):
    """A token of each row of probabilities p: the race of exponentials that spl_verify_drafts decides by."""
    return (p / torch.empty_like(p).exponential_(generator=generator)).argmax(-1)


def generate(target, draft, pages, prompts, drafts, rounds, seed=0):
    """Prompts (lists of token ids) continued for ``rounds`` rounds of up to drafts + 1 tokens each, by the target's
    distribution; both decoders' caches lie on ``pages``.  Returns (tokens per sequence, accepted drafts per round)."""
    if not all(map(len, prompts)):
        raise ValueError("generate: a prompt has at least one token")
    dev, n = target.embedding.device, len(prompts)
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    probs = lambda logits: torch.softmax(logits, -1)  # noqa: E731
    batch = pages.grow([len(p) for p in prompts])
    flat = torch.tensor([t for p in prompts for t in p], device=dev)
    draft.forward(flat, batch)
    last = batch.row_start[1:].long() - 1
    pending = sample(probs(target.forward(flat, batch)[last]), gen)  # chosen, not yet in the caches
    out = [[int(t)] for t in pending]
    starts = lambda per: torch.arange(n + 1, dtype=torch.int32, device=dev) * per  # noqa: E731
    history = []
    for _ in range(rounds):
        base = list(pages.lens)
        chosen, proposals = [pending], []
        for i in range(drafts + 1):  # the last pass only adds the last draft to the cache
            logits = draft.forward(chosen[-1], pages.grow([1] * n))
            if i < drafts:
                proposals.append(probs(logits))
                chosen.append(sample(proposals[-1], gen))
        pages.rewind(base)  # the target sees the same tokens, all at once, where the draft has them
        rows = torch.stack(chosen, dim=1)  # [n, drafts + 1]
        P = probs(target.forward(rows.reshape(-1), pages.grow([drafts + 1] * n)))
        Q = torch.stack(proposals, dim=1).flatten(0, 1) if drafts else P[:0]
        x = rows[:, 1:].reshape(-1).to(torch.int32)
        u = torch.rand(n * drafts, generator=gen, device=dev)
        e = torch.empty((n, P.shape[1]), device=dev).exponential_(generator=gen)
        accepted, token = (torch.empty(n, dtype=torch.int32, device=dev) for _ in range(2))
        spl.spl_verify_drafts(accepted, token, P, Q, x, u, e, starts(drafts + 1), starts(drafts))
        kept = accepted.tolist()
        pages.cut([b + 1 + a for b, a in zip(base, kept)])  # the pending token and the accepted drafts stay
        for b, a in enumerate(kept):
            out[b] += rows[b, 1:1 + a].tolist() + [int(token[b])]
        pending = token.long()
        history.append(kept)
    return out, history


def synthetic(layers, vocab=1024, heads=(8, 2, 64), d_ff=1024, seqs=8, max_len=512, page_size=64, seed=0, eps=float("inf"),
              formats=("f16", "i8")):
    """A decoder on random weights, a draft that is its first layer alone, and pages for both."""
    hq, hk, dim = heads
    shape = wl.ModelShape("synthetic", layers, hq * dim, d_ff, hq * dim, hk * dim, vocab)
    built = []
    for i in range(layers):
        w = {name: wl.weight(N, K, wl.layer_seed(seed, i, j), std=0.5 / K ** 0.5)
             for j, (name, K, N, _) in enumerate(shape.projections())}
        built.append(MaskedLayer.from_weights(shape, w))
        built[-1].sensitivities(power_iters=50)
        built[-1].fp64 = {"down"}
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    embedding, head = (torch.randn((vocab, shape.d_model), generator=g, device="cuda") for _ in range(2))
    head *= 4.0 / shape.d_model ** 0.5  # (not the embedding's: such a decoder would repeat its input)
    count = seqs * -(-max_len // page_size)
    make = lambda n, f, s: CachedDecoder(built[:n], embedding, head, hk, dim, count, page_size, f, eps, seed=s)  # noqa: E731
    draws = 2 * seed, 2 * seed + 1  # each decoder's own: noise hides one input only
    return make(layers, formats[0], draws[0]), make(1, formats[1], draws[1]), Pages(count, page_size, seqs, max_len)


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--sequences", type=int, default=8)
    p.add_argument("--layers", type=int, default=4)
    p.add_argument("--drafts", type=int, default=4)
    p.add_argument("--rounds", type=int, default=16)
    p.add_argument("--prompt", type=int, default=100)
    p.add_argument("--eps", type=float, default=float("inf"))
    a = p.parse_args(argv)
    room = a.prompt + (a.drafts + 1) * (a.rounds + 1)
    target, draft, pages = synthetic(a.layers, seqs=a.sequences, max_len=room, eps=a.eps)
    g = torch.Generator()
    g.manual_seed(1)
    prompts = [torch.randint(1024, (a.prompt,), generator=g).tolist() for _ in range(a.sequences)]
    began = time.perf_counter()
    out, history = generate(target, draft, pages, prompts, a.drafts, a.rounds)
    spent = time.perf_counter() - began
    status = spl.spl_get_device_status()
    taken = sum(map(sum, history))
    print(f"{sum(map(len, out))} tokens of {a.sequences} sequences in {spent:.2f} s, "
          f"{taken} of {a.sequences * a.drafts * a.rounds} drafts accepted, status {spl.status_string(status)}")
    return 0 if status == spl.SPL_OK else 1


if __name__ == "__main__":
    raise SystemExit(main())
