"""The serving operators over a paged cache, as cases to be timed and compared.

Four operators sit around the library's masked products in a serving step: the keys and values that the Q|K|V
product made are written to a paged cache (16 bits, or 8 bits with a scale for each token and head), read back from
it, attended to by a chunk of new tokens of each sequence, and the tokens that a draft proposed are verified against
the target's probabilities.  Head layouts are those of the library's two model shapes (24 or 32 query heads on 8
key heads of 128) and small generic ones of 64.

``run`` computes them in elementary 32-bit torch operations, or, where ``own`` is true, through the library.
"""

import math

import torch

own = False
DEV = "cuda"
LLAMA, QWEN = "24/8x128", "32/8x128"
HEADS = {LLAMA: (24, 8, 128), QWEN: (32, 8, 128), "8/8x64": (8, 8, 64), "14/2x64": (14, 2, 64)}


# ---------------------------------------------------------------------------------- the cases
def listed():
    return [
        # decode: one new token's keys and values into a 16-bit cache, the call's latency
        {"name": "append_llama_1", "kind": "append", "heads": LLAMA, "format": "f16", "page": 64, "seqs": 1,
         "rows": 1, "past": 299, "ragged": False},
        # prefill of a batch of prompts: chunks of ragged length into an 8-bit cache, and what it then holds
        {"name": "roundtrip_qwen_8x1000", "kind": "roundtrip", "heads": QWEN, "format": "i8", "page": 64, "seqs": 8,
         "rows": 1000, "past": 0, "ragged": True},
        # a server batch of 15 short sequences read back from an 8-bit cache
        {"name": "read_llama_15x700", "kind": "read", "heads": LLAMA, "format": "i8", "page": 16, "seqs": 15,
         "rows": 1, "past": 700, "ragged": True},
        # one long context read back (to move it to the host, or to another format)
        {"name": "read_qwen_1x60001", "kind": "read", "heads": QWEN, "format": "f16", "page": 128, "seqs": 1,
         "rows": 1, "past": 60000, "ragged": False},
        # decode of one sequence with a prompt of 300 tokens, the attention call's latency
        {"name": "attend_llama_1x300", "kind": "attention", "heads": LLAMA, "format": "f16", "page": 64, "seqs": 1,
         "rows": 1, "past": 299, "ragged": False, "window": 0},
        # decode of a server batch of 15 prompts that have grown to different lengths, 8-bit cache
        {"name": "attend_qwen_15x900", "kind": "attention", "heads": QWEN, "format": "i8", "page": 64, "seqs": 15,
         "rows": 1, "past": 900, "ragged": True, "window": 0},
        # decode of a large batch with long contexts, bound by the reading of the cache
        {"name": "attend_llama_64x16000", "kind": "attention", "heads": LLAMA, "format": "f16", "page": 64,
         "seqs": 64, "rows": 1, "past": 16000, "ragged": True, "window": 0},
        # five drafted tokens of each of 16 sequences, verified in one pass over an 8-bit cache
        {"name": "attend_qwen_16x5", "kind": "attention", "heads": QWEN, "format": "i8", "page": 32, "seqs": 16,
         "rows": 5, "past": 8000, "ragged": True, "window": 0},
        # prefill of a prompt of 512 tokens
        {"name": "attend_llama_512", "kind": "attention", "heads": LLAMA, "format": "f16", "page": 64, "seqs": 1,
         "rows": 512, "past": 0, "ragged": False, "window": 0},
        # a chunk of a long prompt: 2048 tokens behind 10001 that are in the cache
        {"name": "attend_qwen_2048", "kind": "attention", "heads": QWEN, "format": "f16", "page": 128, "seqs": 1,
         "rows": 2048, "past": 10001, "ragged": False, "window": 0},
        # a server batch of 15 sequences with up to four drafts each, over Llama's vocabulary
        {"name": "verify_llama_15x4", "kind": "verify", "vocab": 128256, "seqs": 15, "drafts": 4},
        # a large batch with up to eight drafts, over Qwen's vocabulary
        {"name": "verify_qwen_64x8", "kind": "verify", "vocab": 151936, "seqs": 64, "drafts": 8},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "roundtrip", "read", "attention", "attention", "attention", "attention", "verify"])
    if kind == "verify":
        return {"kind": kind, "vocab": _log_int(rng, 1000, 151936), "seqs": _log_int(rng, 1, 64),
                "drafts": rng.randint(1, 8)}
    c = {"kind": kind, "heads": rng.choice(list(HEADS)), "format": rng.choice(["f16", "i8"]),
         "page": rng.choice([16, 32, 64, 128]), "ragged": rng.random() < 0.6}
    if kind == "attention":
        rows = rng.choice([1, 1, _log_int(rng, 2, 12), _log_int(rng, 13, 2048)])
        seqs = _log_int(rng, 1, 64 if rows == 1 else max(1, min(32, 2048 // rows)))
        past = rng.choice([0, _log_int(rng, 1, 16000)]) if rows > 1 else _log_int(rng, 1, 16000)
        while rows * seqs * (past + rows) > 1.6e7:
            past //= 2
        window = rng.choice([0, 0, 0, _log_int(rng, 1, past + rows)])
        return {**c, "seqs": seqs, "rows": rows, "past": past, "window": window}
    total = _log_int(rng, 1, 60000)
    seqs = rng.randint(1, min(64, total))
    if kind == "read":
        return {**c, "seqs": seqs, "rows": 1, "past": total // seqs}
    rows = max(1, total // 4 // seqs)
    if kind == "append":  # the pool itself is returned; an 8-bit one is read back (a round trip)
        c["format"] = "f16"
    return {**c, "seqs": seqs, "rows": rows, "past": rng.choice([0, rng.randint(1, 2000)])}


def _ragged(case):
    """New rows and length of each sequence of a case: (rows, len), by the case alone.  Ragged batches spread them,
    the first sequence keeping the full sizes; of three or more the last has nothing at all."""
    n, rows, past = case["seqs"], case["rows"], case["past"]
    if not case["ragged"]:
        return [rows] * n, [past + rows] * n
    part = [1.0 - 0.9 * ((i * 0.6180339887498949) % 1.0) for i in range(n)]
    new = [max(1, round(rows * (p if rows > 16 else 1))) for p in part]
    lens = [r + int(past * p) for r, p in zip(new, part)]
    if n >= 3:
        new[-1] = lens[-1] = 0
    return new, lens


def _starts(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


# ---------------------------------------------------------------------------------- inputs
def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    if case["kind"] == "verify":
        return _prepare_verify(case, g)
    hq, hk, d = HEADS[case["heads"]]
    new, lens = _ragged(case)
    page, fmt = case["page"], case["format"]
    need = [-(-n // page) for n in lens]
    per_seq = max(max(need), 1)
    pages = sum(need) + 3  # some pages of the pool are others'
    order = torch.randperm(pages, generator=g, device=DEV)[:sum(need)].to(torch.int32)
    table = torch.zeros((len(lens), per_seq), dtype=torch.int32, device=DEV)
    used = torch.arange(per_seq, device=DEV)[None, :] < _int32(need)[:, None]
    table[used] = order
    shape = (pages, hk, page, d)
    s = {"case": case, "heads": (hq, hk, d), "rows": sum(new), "max_rows": max(max(new), 1),
         "row_start": _int32(_starts(new)), "kv_len": _int32(lens), "table": table, "fmt": fmt, "page": page,
         "max_len": max(max(lens), 1), "out_start": _int32(_starts(lens)), "tokens": sum(lens)}
    channel = 1.0 + torch.rand((hk, 1, d), generator=g, device=DEV)  # channels differ in size

    def stored():
        """A pool as it is in use: values of tokens written earlier, in every slot."""
        x = torch.empty(shape, dtype=torch.float16 if fmt == "f16" else torch.int8, device=DEV)
        sc = None if fmt == "f16" else torch.empty(shape[:3], device=DEV)
        step = max(1, (1 << 26) // (hk * page * d))
        for a in range(0, pages, step):
            v = torch.randn((min(step, pages - a),) + shape[1:], generator=g, device=DEV) * channel
            if fmt == "f16":
                x[a:a + step] = v.half()
            else:
                amax = v.abs().amax(-1)
                sc[a:a + step] = amax / 127.0
                x[a:a + step] = torch.round(v / sc[a:a + step, :, :, None]).clamp(-127, 127).to(torch.int8)
        return x, sc

    s["k"], s["k_scale"] = stored()
    s["v"], s["v_scale"] = stored()
    # the rows of the fused Q|K|V product, of which each operator takes its columns
    qkv = torch.randn((s["rows"], (hq + 2 * hk) * d), generator=g, device=DEV)
    s["q"], s["k_new"], s["v_new"] = qkv.split([hq * d, hk * d, hk * d], dim=1)
    s["scale"] = 1.0 / math.sqrt(d)
    if own:
        from paper_2609_15039_gb300 import spl
        s["cache"] = spl.KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        s["batch"] = spl.KVBatch(s["row_start"], s["kv_len"], table, rows=s["rows"], max_rows=s["max_rows"])
        if case["kind"] == "attention":
            s["workspace"] = spl.workspace(spl.spl_paged_attention_workspace_bytes(s["cache"], s["batch"], hq), DEV)
    return s


def _prepare_verify(case, g):
    n, k, vocab = case["seqs"], case["drafts"], case["vocab"]
    new = [1 + (k - (i * 2) % (k + 1)) for i in range(n)]  # a target row for each draft and one more
    rows, drafts = sum(new), sum(new) - n

    def probabilities(m, near=None):
        logits = 2.5 * torch.randn((m, vocab), generator=g, device=DEV)
        if near is not None:
            logits = near + 0.5 * logits
        return torch.softmax(logits, dim=1), logits

    p, lp = probabilities(rows)
    row_start = _starts(new)
    of_draft = _int32([row_start[b] + i for b in range(n) for i in range(new[b] - 1)]).long()
    q, _ = probabilities(drafts, lp[of_draft])  # a draft is like its target
    x = (torch.multinomial(q, 1, generator=g) if drafts else torch.zeros((0, 1), device=DEV)).view(-1)
    u = torch.rand(drafts, generator=g, device=DEV)
    e = (-torch.log1p(-torch.rand((n, vocab), generator=g, device=DEV))).clamp(min=1e-30)  # exponential, above 0
    s = {"case": case, "p": p, "q": q, "draft": x.to(torch.int32), "u": u, "e": e, "row_start": _int32(row_start),
         "draft_start": _int32([a - b for b, a in enumerate(row_start)]), "seqs": n, "drafts": k}
    if own:
        from paper_2609_15039_gb300 import spl
        s["workspace"] = spl.workspace(spl.spl_verify_drafts_workspace_bytes(n), DEV)
    return s


# ---------------------------------------------------------------------------------- one pass
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2609_15039_gb300 import spl
    kind = s["case"]["kind"]
    if kind == "verify":
        n = s["seqs"]
        accepted = torch.empty(n, dtype=torch.int32, device=DEV)
        token = torch.empty(n, dtype=torch.int32, device=DEV)
        spl.spl_verify_drafts(accepted, token, s["p"], s["q"], s["draft"], s["u"], s["e"], s["row_start"],
                              s["draft_start"], workspace=s["workspace"])
        return {"accepted": accepted, "token": token}
    hq, hk, d = s["heads"]
    if kind == "attention":
        out = torch.empty((s["rows"], hq * d), device=DEV)
        spl.spl_paged_attention(out, s["q"], s["cache"], s["batch"], hq, scale=s["scale"],
                                window=s["case"]["window"], workspace=s["workspace"])
        return out
    if kind in ("append", "roundtrip"):
        spl.spl_kv_append(s["cache"], s["batch"], s["k_new"], s["v_new"])
    if kind == "append":
        return {"k": s["k"], "v": s["v"]}
    k = torch.empty((s["tokens"], hk * d), device=DEV)
    v = torch.empty((s["tokens"], hk * d), device=DEV)
    spl.spl_kv_read(k, v, s["cache"], s["batch"], s["out_start"])
    return {"k": k, "v": v}


def _slots(s, seq, pos):
    """Page and place in it of position pos of sequence seq."""
    return s["table"][seq, pos // s["page"]].long(), pos % s["page"]


def _seq_of(starts, n):
    """Sequence and place in it of each of n packed rows."""
    r = torch.arange(n, device=DEV)
    seq = torch.searchsorted(starts[1:].contiguous().long(), r, right=True)
    return seq, r - starts[seq]


def _values(s, name, page, at):
    """fp32 values of stored vectors [..., heads, d]."""
    x = s[name][page, :, at].float()
    return x if s["fmt"] == "f16" else x * s[name + "_scale"][page, :, at][..., None]


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "verify":
        return _verify_plain(s)
    if kind == "attention":
        return _attention_plain(s)
    if kind in ("append", "roundtrip"):
        _append_plain(s, "k")
        _append_plain(s, "v")
    if kind == "append":
        return {"k": s["k"], "v": s["v"]}
    seq, at = _seq_of(s["out_start"], s["tokens"])
    page, off = _slots(s, seq, at)
    return {"k": _values(s, "k", page, off).flatten(1), "v": _values(s, "v", page, off).flatten(1)}


def _append_plain(s, name):
    _, hk, d = s["heads"]
    seq, i = _seq_of(s["row_start"], s["rows"])
    new = s["row_start"][1:] - s["row_start"][:-1]
    page, off = _slots(s, seq, s["kv_len"][seq] - new[seq] + i)
    x = s[name + "_new"].unflatten(1, (hk, d))
    if s["fmt"] == "f16":
        s[name][page, :, off] = x.clamp(-65504.0, 65504.0).half()
        return
    scale = x.abs().amax(-1) / torch.full((1,), 127.0, device=DEV)
    code = torch.round(x / scale[..., None]).clamp(-127, 127)
    code = torch.where(scale[..., None] > 0, code, torch.zeros_like(code))
    s[name][page, :, off] = code.to(torch.int8)
    s[name + "_scale"][page, :, off] = scale


def _attention_plain(s):
    hq, hk, d = s["heads"]
    n, rows, longest, chunk = s["kv_len"].numel(), s["rows"], s["max_len"], s["max_rows"]
    window = s["case"]["window"]
    pos = torch.arange(longest, device=DEV)
    page, off = _slots(s, torch.arange(n, device=DEV)[:, None], pos[None, :])
    k = _values(s, "k", page, off).permute(0, 2, 1, 3)  # [n, hk, longest, d]
    v = _values(s, "v", page, off).permute(0, 2, 1, 3)
    seq, i = _seq_of(s["row_start"], rows)
    q = torch.zeros((n, chunk, hq, d), device=DEV)  # every chunk padded to the longest
    q[seq, i] = s["q"].unflatten(1, (hq, d))
    q = q.unflatten(2, (hk, hq // hk)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [n, hk, chunk g, d]
    new = s["row_start"][1:] - s["row_start"][:-1]
    at = (s["kv_len"] - new)[:, None] + torch.arange(chunk, device=DEV)[None, :]  # [n, chunk]
    seen = (pos <= at[:, :, None]) & (pos < s["kv_len"][:, None, None])
    if window:
        seen &= pos > at[:, :, None] - window
    seen = seen.repeat_interleave(hq // hk, dim=1)[:, None]
    score = (q @ k.transpose(2, 3)) * s["scale"]
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.unflatten(2, (chunk, hq // hk)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [n, chunk, hq, d]
    return o[seq, i].flatten(1)


def _verify_plain(s):
    n, k = s["seqs"], s["drafts"]
    start = s["row_start"].long()
    count = start[1:] - start[:-1] - 1  # drafts of each sequence
    i = torch.arange(k, device=DEV)
    there = i[None, :] < count[:, None]
    first = s["draft_start"][:-1].long()  # first draft of each sequence
    at = torch.where(there, first[:, None] + i, torch.zeros_like(there, dtype=torch.long))
    x = s["draft"][at].long()
    target = s["p"][torch.where(there, start[:-1, None] + i, start[:-1, None]), x]
    taken = there & (s["u"][at] * s["q"][at, x] < target)
    accepted = taken.to(torch.int32).cumprod(1).sum(1)
    whole = accepted == count
    p = s["p"][start[:-1] + accepted]
    q = s["q"][torch.where(whole, torch.zeros_like(first), first + accepted)]
    left = torch.where(whole[:, None], p, (p - q).clamp(min=0.0))
    left = torch.where((left > 0).any(1, keepdim=True), left, p)
    ratio = left / s["e"]
    best = ratio.amax(1, keepdim=True)
    ids = torch.arange(ratio.shape[1], device=DEV)
    token = torch.where(ratio == best, ids, torch.full_like(ids, ratio.shape[1])).amin(1)
    return {"accepted": accepted.to(torch.int32), "token": token.to(torch.int32)}


# ---------------------------------------------------------------------------------- the least work
def work(case):
    if case["kind"] == "verify":
        n, k = case["seqs"], case["drafts"]
        drafts = sum(k - (i * 2) % (k + 1) for i in range(n))
        # a row of p and of e for each sequence; where a draft was rejected (more than half) one of q
        return {"bytes": n * case["vocab"] * 4 * 2.5 + drafts * 16 + 8 * n, "flops": n * case["vocab"] * 3}
    hq, hk, d = HEADS[case["heads"]]
    new, lens = _ragged(case)
    slot = hk * (2 * d if case["format"] == "f16" else d + 4)  # a stored token's keys or values
    rows, tokens = sum(new), sum(lens)
    if case["kind"] == "attention":
        w = case["window"]
        pairs = keys = 0
        for r, n in zip(new, lens):
            if not r:
                continue
            lo = n - r + 1  # keys of the first row
            if not w:
                pairs += r * (lo + n) // 2
                keys += n
            else:
                short = max(0, min(w, n + 1) - lo)  # rows that see fewer than a window
                pairs += sum(range(lo, lo + min(short, r))) + (r - min(short, r)) * min(w, n)
                keys += min(n, r - 1 + w)
        return {"bytes": 2 * slot * keys + 8 * rows * hq * d, "flops": 4 * d * hq * pairs}
    read = 2 * tokens * (slot + 4 * hk * d)
    write = 2 * rows * (slot + 4 * hk * d)
    back, wrote = case["kind"] != "append", case["kind"] != "read"
    return {"bytes": read * back + write * wrote, "flops": 2 * hk * d * (tokens * back + rows * wrote)}


# ---------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "verify":
        return _verify_exact(s)
    hq, hk, d = s["heads"]
    starts, lens = s["row_start"].tolist(), s["kv_len"].tolist()
    if case["kind"] in ("append", "roundtrip"):
        for name in ("k", "v"):
            s[name] = s[name].double()
            for b, n in enumerate(lens):
                for r in range(starts[b + 1] - starts[b]):
                    at = n - (starts[b + 1] - starts[b]) + r
                    row = s[name + "_new"][starts[b] + r].double().view(hk, d)
                    where = (int(s["table"][b, at // s["page"]]), slice(None), at % s["page"])
                    if s["fmt"] == "f16":
                        s[name][where] = row.clamp(-65504, 65504).half().double()
                    else:
                        unit = (row.abs().amax(1, keepdim=True) / 127).float().double()
                        s[name][where] = torch.round(row / unit)
                        s[name + "_scale"][where] = unit[:, 0].float()
    if case["kind"] == "append":
        return {"k": s["k"], "v": s["v"]}

    def sequence(name, b):
        """[len, heads, d] of sequence b in 64 bits."""
        x = s[name][s["table"][b].long()].double()
        if s["fmt"] == "i8":
            x = x * s[name + "_scale"][s["table"][b].long()].double()[..., None]
        return x.transpose(1, 2).flatten(0, 1)[:lens[b]]

    if case["kind"] != "attention":
        whole = {name: [sequence(name, b).flatten(1) for b in range(len(lens))] for name in ("k", "v")}
        return {name: torch.cat(v) for name, v in whole.items()}
    out = torch.zeros((s["rows"], hq, d), dtype=torch.float64, device=DEV)
    q = s["q"].double().view(-1, hq, d)
    for b, n in enumerate(lens):
        if starts[b + 1] == starts[b]:
            continue
        k, v = sequence("k", b), sequence("v", b)
        for a in range(starts[b], starts[b + 1], 256):
            z = min(a + 256, starts[b + 1])
            pos = torch.arange(a, z, device=DEV) - starts[b + 1] + n
            j = torch.arange(n, device=DEV)
            hidden = j[None, :] > pos[:, None]
            if case["window"]:
                hidden |= j[None, :] <= pos[:, None] - case["window"]
            for h in range(hq):
                t = s["scale"] * (q[a:z, h] @ k[:, h * hk // hq].T)
                out[a:z, h] = torch.softmax(t.masked_fill(hidden, -math.inf), dim=1) @ v[:, h * hk // hq]
    return out.flatten(1)


def _verify_exact(s):
    """The same decisions with every product, difference and quotient in 64 bits."""
    accepted, token = [], []
    starts = s["row_start"].tolist()
    for b in range(s["seqs"]):
        first, k = starts[b] - b, starts[b + 1] - starts[b] - 1
        n = 0
        while n < k:
            x = int(s["draft"][first + n])
            if not float(s["u"][first + n]) * float(s["q"][first + n, x]) < float(s["p"][starts[b] + n, x]):
                break
            n += 1
        left = s["p"][starts[b] + n].double()
        if n < k:
            rest = torch.relu(left - s["q"][first + n].double())
            left = rest if bool((rest > 0).any()) else left
        accepted.append(n)
        token.append(int(torch.argmax(left / s["e"][b].double())))
    return {"accepted": torch.tensor(accepted, dtype=torch.int32), "token": torch.tensor(token, dtype=torch.int32)}
