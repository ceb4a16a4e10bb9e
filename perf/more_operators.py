"""Serving over a bounded cache with trees of drafts, as cases to be timed and compared.

Beside the cache, the attention over it and the verification of a chain of drafts stand the operators of this file:
attention of drafted tokens that form a tree, the walk down that tree by the target's probabilities with the move of the
accepted path's keys and values to their places, the attention weight that each stored token has gathered, and the
eviction of all but the heaviest and the latest tokens.  Head layouts are those of the library's two model shapes (24 or
32 query heads on 8 key heads of 128) and small generic ones of 64.

``run`` computes them in elementary 32-bit torch operations, or, where ``own`` is true, through the library.
"""

import math

import torch

own = False
DEV = "cuda"
LLAMA, QWEN = "24/8x128", "32/8x128"
HEADS = {LLAMA: (24, 8, 128), QWEN: (32, 8, 128), "8/8x64": (8, 8, 64), "14/2x64": (14, 2, 64)}
ACCEPT = 0.75  # the target's probability that one of a node's children follows


# ---------------------------------------------------------------------------------- the cases
def listed():
    return [
        # a tree of 16 drafts behind a prompt of 300 tokens, one sequence: the call's latency
        {"name": "tree_llama_1x16", "kind": "tree", "heads": LLAMA, "format": "f16", "page": 64, "seqs": 1, "rows": 16,
         "past": 300, "ragged": False, "branch": 2, "window": 0},
        # trees of up to 40 drafts of 15 sequences over an 8-bit cache, some far shorter
        {"name": "tree_qwen_15x40", "kind": "tree", "heads": QWEN, "format": "i8", "page": 32, "seqs": 15, "rows": 40,
         "past": 5000, "ragged": True, "branch": 3, "window": 0},
        # large trees over long contexts, bound by the products
        {"name": "tree_llama_16x64", "kind": "tree", "heads": LLAMA, "format": "f16", "page": 64, "seqs": 16,
         "rows": 64, "past": 12000, "ragged": True, "branch": 4, "window": 0},
        # one sequence's tree verified over Llama's vocabulary: latency
        {"name": "accept_llama_1x16", "kind": "accept", "heads": LLAMA, "format": "f16", "page": 64, "seqs": 1,
         "rows": 16, "past": 300, "ragged": False, "branch": 2, "vocab": 128256},
        # a server batch's trees verified over Qwen's vocabulary
        {"name": "accept_qwen_40x40", "kind": "accept", "heads": QWEN, "format": "f16", "page": 32, "seqs": 40,
         "rows": 40, "past": 100, "ragged": True, "branch": 3, "vocab": 151936},
        # one decode step's weights of one sequence: latency
        {"name": "weigh_llama_1x300", "kind": "weigh", "heads": LLAMA, "format": "f16", "page": 64, "seqs": 1,
         "rows": 1, "past": 299, "ragged": False, "window": 0, "decay": 1.0},
        # a decode step of a large batch with long contexts, bound by the reading of the keys
        {"name": "weigh_llama_64x16000", "kind": "weigh", "heads": LLAMA, "format": "f16", "page": 64, "seqs": 64,
         "rows": 1, "past": 16000, "ragged": True, "window": 0, "decay": 1.0},
        # the last 32 tokens of 15 prompts choose what is kept of them, 8-bit cache
        {"name": "weigh_qwen_15x32", "kind": "weigh", "heads": QWEN, "format": "i8", "page": 32, "seqs": 15,
         "rows": 32, "past": 6000, "ragged": True, "window": 0, "decay": 0.98},
        # a chunk of a long prompt, every row counts
        {"name": "weigh_qwen_2048", "kind": "weigh", "heads": QWEN, "format": "f16", "page": 128, "seqs": 1,
         "rows": 2048, "past": 10001, "ragged": False, "window": 0, "decay": 1.0},
        # a sequence that has passed its budget by a quarter, moved together where it lies
        {"name": "evict_llama_1x1250", "kind": "evict", "heads": LLAMA, "format": "f16", "page": 64, "seqs": 1,
         "past": 1250, "ragged": False, "keep": 1000, "recent": 250, "fresh": False},
        # 15 prompts cut to 800 tokens each after their prefill, 8-bit cache, and what it then holds
        {"name": "evict_qwen_15x5000", "kind": "evict", "heads": QWEN, "format": "i8", "page": 16, "seqs": 15,
         "past": 5000, "ragged": True, "keep": 800, "recent": 64, "fresh": False},
        # a large batch of long contexts halved, into other pages (the old ones are shared)
        {"name": "evict_llama_32x16000", "kind": "evict", "heads": LLAMA, "format": "f16", "page": 64, "seqs": 32,
         "past": 16000, "ragged": True, "keep": 6000, "recent": 1000, "fresh": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "accept", "weigh", "weigh", "weigh", "evict", "evict"])
    c = {"kind": kind, "heads": rng.choice(list(HEADS)), "format": rng.choice(["f16", "i8"]),
         "page": rng.choice([16, 32, 64, 128]), "ragged": rng.random() < 0.6}
    if kind == "accept":
        rows = _log_int(rng, 1, 64)
        return {**c, "vocab": _log_int(rng, 1000, 151936), "seqs": _log_int(rng, 1, max(1, min(64, 1600 // rows))),
                "rows": rows, "past": rng.choice([0, _log_int(rng, 1, 500)]), "branch": rng.randint(1, 4)}
    if kind == "evict":
        past = _log_int(rng, 2, 16000)
        keep = _log_int(rng, 1, past)
        return {**c, "seqs": _log_int(rng, 1, max(1, min(32, 250000 // past))), "past": past, "keep": keep,
                "recent": rng.choice([0, keep, rng.randint(0, keep), min(keep, 32)]), "fresh": rng.random() < 0.5}
    if kind == "tree":
        rows = _log_int(rng, 1, 150)
        seqs = _log_int(rng, 1, max(1, min(32, 1024 // rows)))
        past = rng.choice([0, _log_int(rng, 1, 12000), _log_int(rng, 1, 12000)])
        more = {"branch": rng.randint(1, 4)}
    else:
        rows = rng.choice([1, 1, _log_int(rng, 2, 12), _log_int(rng, 13, 2048)])
        seqs = _log_int(rng, 1, 64 if rows == 1 else max(1, min(32, 2048 // rows)))
        past = rng.choice([0, _log_int(rng, 1, 16000)]) if rows > 1 else _log_int(rng, 1, 16000)
        more = {"decay": rng.choice([1.0, 1.0, 0.9, 0.0])}
    while rows * seqs * (past + rows) > 1.2e7:
        past //= 2
    return {**c, "seqs": seqs, "rows": rows, "past": past, "window": rng.choice([0, 0, 0, _log_int(rng, 1, past + rows)]),
            **more}


def _ragged(case):
    """New rows and length of each sequence of a case: (rows, len), by the case alone.  Ragged batches spread them,
    the first sequence keeping the full sizes; of three or more the last has nothing at all."""
    n, rows, past = case["seqs"], case.get("rows", 0), case["past"]
    if not case["ragged"]:
        return [rows] * n, [past + rows] * n
    part = [1.0 - 0.9 * ((i * 0.6180339887498949) % 1.0) for i in range(n)]
    new = [min(rows, max(1, round(rows * (p if rows > 12 else 1)))) for p in part]
    lens = [r + int(past * p) for r, p in zip(new, part)]
    if n >= 3:
        new[-1] = lens[-1] = 0
    return new, lens


def _starts(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def _parents(rows, branch):
    """Node i > 0 hangs on node (i - 1) // branch; node 0 is the token that the target has chosen already."""
    return [max(0, i - 1) // branch if i else -1 for i in range(rows)]


def _depths(parents):
    out = []
    for p in parents:
        out.append(out[p] + 1 if p >= 0 else 0)
    return out


# ---------------------------------------------------------------------------------- inputs
def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    hq, hk, d = HEADS[case["heads"]]
    new, lens = _ragged(case)
    page, fmt, kind = case["page"], case["format"], case["kind"]
    kept = [min(n, case["keep"]) for n in lens] if kind == "evict" else lens
    need = [-(-n // page) for n in lens]
    other = [-(-n // page) for n in kept] if case.get("fresh") else [0] * len(lens)
    per_seq = max(max(need), 1)
    pages = sum(need) + sum(other) + 3  # some pages of the pool are others'
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)

    def table_of(counts, ids):
        t = torch.zeros((len(lens), per_seq), dtype=torch.int32, device=DEV)
        t[torch.arange(per_seq, device=DEV)[None, :] < _int32(counts)[:, None]] = ids
        return t

    shape = (pages, hk, page, d)
    s = {"case": case, "heads": (hq, hk, d), "rows": sum(new), "max_rows": max(max(new), 1), "row_start": _int32(_starts(new)),
         "kv_len": _int32(lens), "table": table_of(need, order[:sum(need)]), "fmt": fmt, "page": page,
         "max_len": max(max(lens), 1), "out_start": _int32(_starts(kept)), "tokens": sum(kept), "scale": 1.0 / math.sqrt(d)}
    s["fresh"] = table_of(other, order[sum(need):sum(need) + sum(other)]) if case.get("fresh") else None
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
    if kind in ("weigh", "evict"):  # weights gathered so far: most tokens little, a few much
        s["score"] = torch.exp(2.0 * torch.randn(shape[:3], generator=g, device=DEV)) * (4.0 / s["max_len"])
    if kind in ("tree", "weigh"):  # the rows of the fused Q|K|V product, of which the operators take the first columns
        qkv = torch.randn((s["rows"], (hq + 2 * hk) * d), generator=g, device=DEV)
        s["q"] = qkv[:, :hq * d]
    if kind in ("tree", "accept"):
        parents = _parents(s["max_rows"], case["branch"])
        s["levels"] = max(_depths(parents)) + 1
        s["parent"] = _int32([p for n in new for p in parents[:n]])
        words = -(-s["max_rows"] // 32)
        masks = []
        for i, p in enumerate(parents):
            masks.append((masks[p] if p >= 0 else 0) | 1 << i)
        split = [[m >> 32 * w & 0xffffffff for w in range(words)] for m in masks]
        signed = [[v - (1 << 32) if v >> 31 else v for v in m] for m in split]
        s["seen"] = _int32([m for n in new for m in signed[:n]]).view(-1, words)
    if kind == "accept":
        _prepare_accept(s, new, parents, g)
    return s


def _prepare_accept(s, new, parents, g):
    n, rows, vocab, most = len(new), s["rows"], s["case"]["vocab"], s["max_rows"]
    # a node's token, unlike those of its siblings
    base = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    seq = torch.repeat_interleave(torch.arange(n, device=DEV), _int32(new).long(), output_size=rows)
    node = torch.arange(rows, device=DEV) - s["row_start"][seq]
    s["x"] = ((base[seq] + node * 7919) % vocab).to(torch.int32)
    p = torch.softmax(2.5 * torch.randn((rows, vocab), generator=g, device=DEV), dim=1)
    # the drafts are good: a node's children have ACCEPT of its probability together, the first of them most
    branch = s["case"]["branch"]
    share = torch.tensor([2.0 ** -i for i in range(branch)], device=DEV)
    child = node >= 1
    up = (torch.div(node - 1, branch, rounding_mode="floor") + s["row_start"][seq])[child].long()
    weight = share[((node - 1) % branch)[child]]
    total = torch.zeros(rows, device=DEV).index_add_(0, up, weight)
    p *= torch.where(total > 0, 1.0 - ACCEPT, 1.0)[:, None]
    p.index_put_((up, s["x"][child].long()), ACCEPT * weight / total[up], accumulate=True)
    s["p"] = p
    e = torch.rand((n * s["levels"], vocab), generator=g, device=DEV)
    s["e"] = (-torch.log1p(-e)).clamp(min=1e-30)  # exponential, above 0


# ---------------------------------------------------------------------------------- one pass
def run(s):
    return (_run_own if own else _run_plain)(s)


def _handles(s):
    """The library's handles on the state's tensors, which a program keeps."""
    from paper_2609_15039_gb300 import spl
    if "cache" not in s:
        kind, hq = s["case"]["kind"], s["heads"][0]
        s["cache"] = spl.KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        s["batch"] = spl.KVBatch(s["row_start"], s["kv_len"], s["table"], rows=s["rows"], max_rows=s["max_rows"])
        need = 0
        if kind == "tree":
            need = spl.spl_paged_attention_workspace_bytes(s["cache"], s["batch"], hq)
        elif kind == "weigh":
            need = spl.spl_kv_weigh_workspace_bytes(s["cache"], s["batch"], hq)
        elif kind == "evict":
            need = spl.spl_kv_evict_workspace_bytes(s["cache"], s["batch"], s["case"]["keep"])
            s["len"] = torch.empty_like(s["kv_len"])
            there = s["table"] if s["fresh"] is None else s["fresh"]
            s["after"] = spl.KVBatch(s["row_start"], s["len"], there, rows=s["rows"], max_rows=s["max_rows"])
        s["workspace"] = spl.workspace(need, DEV)
    return spl


def _run_own(s):
    spl = _handles(s)
    case, kind, (hq, _, d) = s["case"], s["case"]["kind"], s["heads"]
    if kind == "tree":
        out = torch.empty((s["rows"], hq * d), device=DEV)
        spl.spl_tree_attention(out, s["q"], s["cache"], s["batch"], s["seen"], hq, scale=s["scale"],
                               window=case["window"], workspace=s["workspace"])
        return out
    if kind == "weigh":
        spl.spl_kv_weigh(s["score"], s["q"], s["cache"], s["batch"], hq, scale=s["scale"], window=case["window"],
                         decay=case["decay"], workspace=s["workspace"])
        return s["score"]
    if kind == "evict":
        spl.spl_kv_evict(s["cache"], s["score"], s["batch"], case["keep"], case["recent"], s["len"], out_table=s["fresh"],
                         workspace=s["workspace"])
        return {**_own_held(spl, s, s["after"]), "score": s["score"], "len": s["len"]}
    n = case["seqs"]
    accepted, token = (torch.empty(n, dtype=torch.int32, device=DEV) for _ in range(2))
    path = torch.empty((n, s["levels"]), dtype=torch.int32, device=DEV)
    spl.spl_verify_tree(accepted, path, token, s["p"], s["x"], s["parent"], s["e"], s["row_start"])
    spl.spl_kv_keep_path(s["cache"], s["batch"], path, accepted)
    return {**_own_held(spl, s, s["batch"]), "accepted": accepted, "path": path, "token": token}


def _own_held(spl, s, batch):
    """What the cache holds: its pools, or (8 bits) the sequences read back."""
    if s["fmt"] == "f16":
        return {"k": s["k"], "v": s["v"]}
    k, v = (torch.empty((s["tokens"], s["heads"][1] * s["heads"][2]), device=DEV) for _ in range(2))
    spl.spl_kv_read(k, v, s["cache"], batch, s["out_start"])
    return {"k": k, "v": v}


def _seq_of(starts, n):
    """Sequence and place in it of each of n packed rows."""
    r = torch.arange(n, device=DEV)
    seq = torch.searchsorted(starts[1:].contiguous().long(), r, right=True)
    return seq, r - starts[seq]


def _values(s, name, page, at):
    """fp32 values of stored vectors [..., heads, d]."""
    x = s[name][page, :, at].float()
    return x if s["fmt"] == "f16" else x * s[name + "_scale"][page, :, at][..., None]


def _held(s, table):
    if s["fmt"] == "f16":
        return {"k": s["k"], "v": s["v"]}
    seq, at = _seq_of(s["out_start"], s["tokens"])
    page = table[seq, at // s["page"]].long()
    return {name: _values(s, name, page, at % s["page"]).flatten(1) for name in ("k", "v")}


def _run_plain(s):
    return {"tree": _tree_plain, "accept": _accept_plain, "weigh": _weigh_plain, "evict": _evict_plain}[s["case"]["kind"]](s)


def _probabilities(s, tree):
    """Softmax of the rows' scores over their sequences' keys [n, hk, chunk group, longest], and where the rows lie."""
    hq, hk, d = s["heads"]
    n, longest, chunk, window = s["kv_len"].numel(), s["max_len"], s["max_rows"], s["case"]["window"]
    pos = torch.arange(longest, device=DEV)
    page = s["table"][:, pos // s["page"]].long()
    k = _values(s, "k", page, pos % s["page"]).permute(0, 2, 1, 3)  # [n, hk, longest, d]
    seq, i = _seq_of(s["row_start"], s["rows"])
    q = torch.zeros((n, chunk, hq, d), device=DEV)  # every chunk padded to the longest
    q[seq, i] = s["q"].unflatten(1, (hq, d))
    q = q.unflatten(2, (hk, hq // hk)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [n, hk, chunk g, d]
    new = s["row_start"][1:] - s["row_start"][:-1]
    context = (s["kv_len"] - new)[:, None]
    at = context + torch.arange(chunk, device=DEV)[None, :]  # [n, chunk]
    if tree:
        bit = (pos[None, :] - context)[:, None, :].expand(n, chunk, longest)  # of the row's mask
        inside = (bit >= 0) & (bit < new[:, None, None])
        words = torch.zeros((n, chunk, s["seen"].shape[1]), dtype=torch.int32, device=DEV)
        words[seq, i] = s["seen"]
        word = words.gather(2, torch.where(inside, bit // 32, torch.zeros_like(bit)).long())
        seen = torch.where(inside, (word >> (bit % 32)) & 1 == 1, bit < 0)
        if window:  # the last of those that it sees
            seen &= seen.to(torch.int32).flip(2).cumsum(2).flip(2) <= window
    else:
        seen = (pos <= at[:, :, None]) & (pos < s["kv_len"][:, None, None])
        if window:
            seen &= pos > at[:, :, None] - window
    real = torch.arange(chunk, device=DEV)[None, :] < new[:, None]
    seen = (seen & real[:, :, None]).repeat_interleave(hq // hk, dim=1)[:, None]
    score = (q @ k.transpose(2, 3)) * s["scale"]
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total > 0, total, torch.ones_like(total)), page, seq, i


def _tree_plain(s):
    hq, hk, _ = s["heads"]
    p, page, seq, i = _probabilities(s, True)
    pos = torch.arange(s["max_len"], device=DEV)
    v = _values(s, "v", page, pos % s["page"]).permute(0, 2, 1, 3)
    o = (p @ v).unflatten(2, (s["max_rows"], hq // hk)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [n, chunk, hq, d]
    return o[seq, i].flatten(1)


def _weigh_plain(s):
    p, page, _, _ = _probabilities(s, False)
    weight = p.sum(2).permute(0, 2, 1)  # [n, longest, hk]
    pos = torch.arange(s["max_len"], device=DEV)
    new = s["row_start"][1:] - s["row_start"][:-1]
    there = pos[None, :] < s["kv_len"][:, None]
    old = (pos[None, :] < (s["kv_len"] - new)[:, None])[there]
    where = (page[there], slice(None), (pos % s["page"])[None, :].expand_as(there)[there])
    before = s["score"][where]
    s["score"][where] = torch.where(old[:, None], before * s["case"]["decay"], torch.zeros_like(before)) + weight[there]
    return s["score"]


def _move_plain(s, seq, head, source, target, table):
    """Stored tokens of (sequence, head) from the positions `source` to `target` of `table`, all at once."""
    page = s["table"][seq, source // s["page"]].long()
    to = table[seq, target // s["page"]].long()
    for name in ("k", "v", "k_scale", "v_scale", "score"):
        if s.get(name) is not None:
            s[name][to, head, target % s["page"]] = s[name][page, head, source % s["page"]]


def _evict_plain(s):
    case, hk, longest = s["case"], s["heads"][1], s["max_len"]
    n, keep, recent = case["seqs"], case["keep"], case["recent"]
    pos = torch.arange(longest, device=DEV)
    page = s["table"][:, pos // s["page"]].long()
    lens = s["kv_len"][:, None]
    score = s["score"][page, :, pos % s["page"]].permute(0, 2, 1)  # [n, hk, longest]
    late, there = pos[None, :] >= lens - recent, pos[None, :] < lens
    score = torch.where(late[:, None], torch.full_like(score, math.inf), score)
    score = torch.where(there[:, None], score, torch.full_like(score, -math.inf))
    order = torch.sort(score, dim=2, descending=True, stable=True).indices  # equal ones: the earliest first
    rank = torch.empty_like(order).scatter_(2, order, pos.expand_as(order))
    stays = (rank < keep) & there[:, None]
    place = stays.to(torch.int64).cumsum(2) - 1
    seq, head, source = stays.nonzero(as_tuple=True)
    table = s["table"] if s["fresh"] is None else s["fresh"]
    _move_plain(s, seq, head, source, place[stays], table)
    return {**_held(s, table), "score": s["score"], "len": s["kv_len"].clamp(max=keep)}


def _accept_plain(s):
    n, levels = s["case"]["seqs"], s["levels"]
    start, rows = s["row_start"].long(), s["rows"]
    new = start[1:] - start[:-1]
    seq, i = _seq_of(s["row_start"], rows)
    e = s["e"].view(n, levels, -1)
    ids = torch.arange(e.shape[2], device=DEV)
    at, going = torch.zeros(n, dtype=torch.long, device=DEV), new > 0
    accepted = torch.zeros(n, dtype=torch.int32, device=DEV)
    token = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    path = torch.full((n, levels), -1, dtype=torch.int32, device=DEV)
    nobody = torch.full((n,), rows, dtype=torch.long, device=DEV)
    for d in range(levels):  # a level follows from the one before
        ratio = s["p"][torch.where(going, start[:-1] + at, torch.zeros_like(at))] / e[:, d]
        best = ratio.amax(1, keepdim=True)
        t = torch.where(ratio == best, ids, torch.full_like(ids, ids.numel())).amin(1)
        token = torch.where(going, t.to(torch.int32), token)
        follows = (i > 0) & (s["parent"] == at[seq]) & (s["x"] == t[seq]) & going[seq]
        child = nobody.scatter_reduce(0, seq, torch.where(follows, i.long(), torch.full_like(seq, rows)), "amin")
        going = going & (child < rows) & (d + 1 < levels)
        path[:, d] = torch.where(going, child, torch.full_like(child, -1)).to(torch.int32)
        accepted += going.to(torch.int32)
        at = torch.where(going, child, at)
    seq, d = (path >= 0).nonzero(as_tuple=True)
    context = (s["kv_len"].long() - new)[seq]
    head = torch.arange(s["heads"][1], device=DEV)
    _move_plain(s, seq[:, None], head[None, :], (context + path[seq, d])[:, None], (context + 1 + d)[:, None], s["table"])
    return {**_held(s, s["table"]), "accepted": accepted, "path": path, "token": token}


# ---------------------------------------------------------------------------------- the least work
def _pairs(case, new, lens):
    """(row, key) pairs that see each other, and keys that some row sees."""
    w, pairs, keys = case["window"], 0, 0
    tree = _depths(_parents(max(new + [1]), case["branch"])) if case["kind"] == "tree" else None
    for r, n in zip(new, lens):
        if not r:
            continue
        if tree:
            counts = [n - r + depth + 1 for depth in tree[:r]]
        else:
            counts = range(n - r + 1, n + 1)
        pairs += sum(min(c, w) for c in counts) if w else sum(counts)
        keys += min(n, r - 1 + w) if w else n
    return pairs, keys


def work(case):
    hq, hk, d = HEADS[case["heads"]]
    new, lens = _ragged(case)
    vector = 2 * d if case["format"] == "f16" else d + 4  # a stored token's keys or values of a head
    rows = sum(new)
    if case["kind"] == "tree":
        pairs, keys = _pairs(case, new, lens)
        return {"bytes": 2 * hk * vector * keys + 8 * rows * hq * d, "flops": 4 * d * hq * pairs}
    if case["kind"] == "weigh":
        pairs, keys = _pairs(case, new, lens)
        return {"bytes": hk * (vector * keys + 8 * sum(lens)) + 4 * rows * hq * d, "flops": 2 * d * hq * pairs}
    back = 0 if case["format"] == "f16" else 2 * hk * (vector + 4 * d)  # a token that is read back
    if case["kind"] == "evict":
        kept = sum(min(n, case["keep"]) for n in lens)
        long = sum(n for n in lens if n > case["keep"])  # tokens of which some go
        moved = kept if case["fresh"] else sum(case["keep"] for n in lens if n > case["keep"])
        return {"bytes": 4 * hk * long + 2 * hk * (2 * vector + 4) * moved + back * kept, "flops": hk * sum(lens)}
    levels = max(_depths(_parents(max(new), case["branch"]))) + 1
    looked = sum(ACCEPT ** i for i in range(levels)) * sum(1 for r in new if r)  # nodes on the way down, on average
    return {"bytes": 8 * case["vocab"] * looked + 8 * rows + back * sum(lens), "flops": case["vocab"] * looked}


# ---------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"tree": _tree_exact, "accept": _accept_exact, "weigh": _weigh_exact, "evict": _evict_exact}[case["kind"]](s)


def _sequence(s, name, b, length, table):
    """[heads, length, d] of sequence b in 64 bits."""
    ids = table[b].long()
    x = s[name][ids].double()
    if s["fmt"] == "i8":
        x = x * s[name + "_scale"][ids].double()[..., None]
    return x.transpose(0, 1).flatten(1, 2)[:, :length]


def _exact_held(s, lens, table):
    if s["fmt"] == "f16":
        return {"k": s["k"], "v": s["v"]}
    return {name: torch.cat([_sequence(s, name, b, n, table).transpose(0, 1).flatten(1) for b, n in enumerate(lens)])
            for name in ("k", "v")}


def _softmax_rows(s, b, visible):
    """For 128 rows of sequence b at a time: (first, last row, softmax [hk, group, rows, len]) in 64 bits, visible(row) the
    row's keys as a list of truth values."""
    hq, hk, d = s["heads"]
    first, last = s["row_start"][b:b + 2].tolist()
    length = int(s["kv_len"][b])
    k = _sequence(s, "k", b, length, s["table"])
    q = s["q"].double().view(-1, hk, hq // hk, d)
    for a in range(first, last, 128):
        z = min(a + 128, last)
        hidden = torch.stack([~visible(r - first) for r in range(a, z)])
        t = s["scale"] * torch.einsum("rhgd,hjd->hgrj", q[a:z], k)
        p = torch.softmax(t.masked_fill(hidden, -math.inf), dim=3)
        yield a, z, torch.nan_to_num(p)  # a row that sees nothing


def _last(seen, window):
    """The last `window` true places."""
    if window:
        seen = seen.clone()
        seen[seen.nonzero()[:-window, 0]] = False
    return seen


def _tree_exact(s):
    hq, hk, d = s["heads"]
    out = torch.zeros((s["rows"], hk, hq // hk, d), dtype=torch.float64, device=DEV)
    lens, starts = s["kv_len"].tolist(), s["row_start"].tolist()
    bits = torch.arange(32, device=DEV)
    for b, n in enumerate(lens):
        context = n - (starts[b + 1] - starts[b])

        def visible(i, b=b, n=n, context=context):
            mask = (s["seen"][starts[b] + i].long()[:, None] >> bits & 1).bool().flatten()[:n - context]
            mask = torch.cat([mask, torch.zeros(n - context - mask.numel(), dtype=torch.bool, device=DEV)])
            return _last(torch.cat([torch.ones(context, dtype=torch.bool, device=DEV), mask]), s["case"]["window"])
        if n > context:
            v = _sequence(s, "v", b, n, s["table"])
            for a, z, p in _softmax_rows(s, b, visible):
                out[a:z] = torch.einsum("hgrj,hjd->rhgd", p, v)
    return out.flatten(1)


def _weigh_exact(s):
    score = s["score"].double()
    lens, starts = s["kv_len"].tolist(), s["row_start"].tolist()
    for b, n in enumerate(lens):
        new = starts[b + 1] - starts[b]
        total = torch.zeros((s["heads"][1], n), dtype=torch.float64, device=DEV)
        j = torch.arange(n, device=DEV)
        for _, _, p in _softmax_rows(s, b, lambda i: _last(j <= n - new + i, s["case"]["window"])):
            total += p.sum((1, 2))
        where = (s["table"][b][j // s["page"]].long(), slice(None), j % s["page"])
        score[where] = (score[where] * (s["case"]["decay"] * (j < n - new))[:, None]) + total.T
    return score


def _evict_exact(s):
    case, table = s["case"], s["table"] if s["fresh"] is None else s["fresh"]
    kept = []
    for b, n in enumerate(s["kv_len"].tolist()):
        keep = min(n, case["keep"])
        kept.append(keep)
        j = torch.arange(n, device=DEV)
        score = s["score"][s["table"][b][j // s["page"]].long(), :, j % s["page"]].double().T.cpu()
        to = torch.arange(keep, device=DEV)
        stay = []
        for h in range(s["heads"][1]):
            early = n - min(n, case["recent"])
            best = sorted(range(early), key=score[h].tolist().__getitem__, reverse=True)  # stable: the earliest of equals
            stay.append(torch.tensor(sorted(best[:keep - (n - early)]) + list(range(early, n)), dtype=torch.long))
        if not keep:
            continue
        head, stay = torch.arange(len(stay), device=DEV)[:, None], torch.stack(stay).to(DEV)
        for name in ("k", "v", "k_scale", "v_scale", "score"):
            if s[name] is not None:
                moved = s[name][s["table"][b][stay // s["page"]].long(), head, stay % s["page"]]
                s[name][table[b][to // s["page"]].long()[None, :], head, (to % s["page"])[None, :]] = moved
    return {**_exact_held(s, kept, table), "score": s["score"].double(), "len": torch.tensor(kept, dtype=torch.int32)}


def _accept_exact(s):
    """The same walk with every quotient in 64 bits."""
    starts, levels = s["row_start"].tolist(), s["levels"]
    parent, x, lens = s["parent"].tolist(), s["x"].tolist(), s["kv_len"].tolist()
    accepted, token, path = [], [], []
    for b, n in enumerate(lens):
        first, nodes = starts[b], starts[b + 1] - starts[b]
        way, t = [], -1
        while nodes:
            row = s["p"][first + (way[-1] if way else 0)].double() / s["e"][b * levels + len(way)].double()
            t = int(torch.argmax(row))
            at = way[-1] if way else 0
            after = [c for c in range(1, nodes) if parent[first + c] == at and x[first + c] == t]
            if not after or len(way) + 1 == levels:
                break
            way.append(after[0])
        for i, c in enumerate(way):
            for name in ("k", "v", "k_scale", "v_scale"):
                if s[name] is not None:
                    source, target = n - nodes + c, n - nodes + 1 + i
                    place = [(int(s["table"][b, at // s["page"]]), slice(None), at % s["page"]) for at in (source, target)]
                    s[name][place[1]] = s[name][place[0]].clone()
        accepted.append(len(way))
        token.append(t)
        path.append(way + [-1] * (levels - len(way)))
    return {**_exact_held(s, lens, s["table"]), "accepted": torch.tensor(accepted, dtype=torch.int32),
            "path": torch.tensor(path, dtype=torch.int32), "token": torch.tensor(token, dtype=torch.int32)}
