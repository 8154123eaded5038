"""Measured cases of the operators on a cache kept in pages: a chunk of new tokens is appended and attends to the cache,
with or without a sliding window and first tokens that stay visible; the weight that every cached row has been given is
accumulated; the rows with the least of it are evicted.

A case is a dict of plain values.  The kinds:
  append      rows of the new tokens of one layer go to their places in the cache
  attend      attention of the new tokens of every sequence over its own cached rows, grouped heads or not; `window` > 0: over
              the last `window` positions and the first `sinks`
  weigh       the attention weights of that step, summed per cached row and key head onto the weights of earlier steps
  evict       every sequence of more than `budget` cached rows keeps its first, its most recent and its heaviest ones
The cache is [page][key head][page_size][head_dim], as one layer of a serving program has it.  A plan (lengths and page lists,
checked and laid out on the device) is made once per iteration and serves all layers of the model, so it belongs to what a
program has in hand before one layer's call.

run() computes the operators in elementary torch operations, or, where `own` is true, by the library's calls.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # the new rows of a full server's iteration: one token of each of 96 requests
        {"name": "append_decode_bf16", "kind": "append", "dtype": "bf16", "seqs": 96, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 16, "new_lo": 1, "new_hi": 1, "len_lo": 20, "len_hi": 1500, "window": 0, "sinks": 0},
        # prompts of a few hundred tokens arriving at a GPT-1.3B-shaped server
        {"name": "append_chunks_f16", "kind": "append", "dtype": "f16", "seqs": 5, "heads": 16, "kv_heads": 16, "head_dim": 128,
         "page": 64, "new_lo": 130, "new_hi": 1024, "len_lo": 130, "len_hi": 2048, "window": 0, "sinks": 0},
        # the smallest server: a tiny fp32 GPT whose requests bring one to a few tokens; latency
        {"name": "attend_tiny_f32", "kind": "attend", "dtype": "f32", "seqs": 7, "heads": 4, "kv_heads": 4, "head_dim": 64,
         "page": 16, "new_lo": 1, "new_hi": 5, "len_lo": 5, "len_hi": 128, "window": 0, "sinks": 0},
        # a full server's decode step with grouped heads: one token each, caches of every length
        {"name": "attend_decode_bf16", "kind": "attend", "dtype": "bf16", "seqs": 64, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 64, "new_lo": 1, "new_hi": 1, "len_lo": 1, "len_hi": 8192, "window": 0, "sinks": 0},
        # two long prompts, the last 2048 tokens of each: the products bound it
        {"name": "attend_chunk_bf16", "kind": "attend", "dtype": "bf16", "seqs": 2, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 64, "new_lo": 2048, "new_hi": 2048, "len_lo": 7000, "len_hi": 8192, "window": 0, "sinks": 0},
        # chunks of prompts beside decoding requests, a head for every key head (the 7B shape), odd lengths
        {"name": "attend_mixed_f16", "kind": "attend", "dtype": "f16", "seqs": 13, "heads": 32, "kv_heads": 32, "head_dim": 128,
         "page": 16, "new_lo": 1, "new_hi": 333, "len_lo": 40, "len_hi": 2048, "window": 0, "sinks": 0},
        # decode of streams far longer than their window
        {"name": "window_decode_bf16", "kind": "attend", "dtype": "bf16", "seqs": 24, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 32, "new_lo": 1, "new_hi": 1, "len_lo": 700, "len_hi": 20000, "window": 1024, "sinks": 4},
        # a chunk of a long document
        {"name": "window_chunk_bf16", "kind": "attend", "dtype": "bf16", "seqs": 1, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 64, "new_lo": 4001, "new_hi": 4001, "len_lo": 12345, "len_hi": 12345, "window": 2048, "sinks": 4},
        # which cached rows a decode step looked at
        {"name": "weigh_decode_bf16", "kind": "weigh", "dtype": "bf16", "seqs": 32, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 64, "new_lo": 1, "new_hi": 1, "len_lo": 100, "len_hi": 8192, "window": 0, "sinks": 0},
        # the same for a chunk of a prompt, GPT-1.3B shape
        {"name": "weigh_chunk_f16", "kind": "weigh", "dtype": "f16", "seqs": 2, "heads": 16, "kv_heads": 16, "head_dim": 128,
         "page": 16, "new_lo": 700, "new_hi": 1024, "len_lo": 1500, "len_hi": 4096, "window": 0, "sinks": 0},
        # a small fp32 model's few requests outgrow their budget
        {"name": "evict_small_f32", "kind": "evict", "dtype": "f32", "seqs": 3, "heads": 12, "kv_heads": 12, "head_dim": 64,
         "page": 16, "new_lo": 1, "new_hi": 1, "len_lo": 100, "len_hi": 400, "window": 0, "sinks": 4, "budget": 128, "recent": 32},
        # a full server halves its caches
        {"name": "evict_many_bf16", "kind": "evict", "dtype": "bf16", "seqs": 32, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 64, "new_lo": 1, "new_hi": 1, "len_lo": 500, "len_hi": 4096, "window": 0, "sinks": 4, "budget": 1024, "recent": 256},
    ]


def _log(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "window", "weigh", "evict"])
    kv = rng.choice([1, 2, 4, 5, 8, 16, 32])
    c = {"kind": "attend" if kind == "window" else kind, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "kv_heads": kv,
         "head_dim": rng.choice([64, 128, 128]), "page": rng.choice([16, 32, 48, 64, 256])}
    c["heads"] = kv * rng.choice([g for g in (1, 2, 3, 4, 8) if kv * g <= 32])
    c["window"], c["sinks"] = (_log(rng, 30, 3000), rng.choice([0, 1, 4, 70])) if kind == "window" else (0, 0)
    if rng.random() < 0.5 or kind == "evict":           # decode: a token or a few of each of many requests
        c["seqs"], c["new_lo"] = _log(rng, 1, 48), 1
        c["new_hi"] = rng.choice([1, 1, 3, 8])
        rows = 10**9 // (c["seqs"] * kv * c["head_dim"] * (4 if c["dtype"] == "f32" else 2))     # a pass costs no more than the largest listed
        c["len_hi"] = _log(rng, 40, max(100, min(6000, rows)))
        c["len_lo"] = max(c["new_hi"], _log(rng, 1, c["len_hi"]))
    else:                                               # chunks of a few prompts, decoding requests beside them or not
        c["seqs"] = rng.randint(1, 4)
        c["new_hi"] = _log(rng, 20, 1500)
        c["new_lo"] = rng.choice([1, c["new_hi"] // 2, c["new_hi"]])
        c["len_hi"] = max(c["new_hi"], _log(rng, 100, 5000))
        c["len_lo"] = max(c["new_hi"], c["len_hi"] // 2)
    if kind == "evict":
        c["len_lo"], c["len_hi"] = c["len_lo"] + 20, c["len_hi"] + 40
        c["budget"] = rng.randint(10, c["len_hi"] - 1)
        c["sinks"] = rng.randint(0, min(8, c["budget"] // 2))
        c["recent"] = rng.randint(0, c["budget"] // 2)
    return c


def _lengths(c):
    """(new tokens, cached rows with them) of every sequence: spread evenly over the case's ranges, in a shuffled order."""
    n = c["seqs"]
    at = lambda lo, hi, i: hi if n == 1 else lo + (hi - lo) * i // (n - 1)  # noqa: E731
    rng = random.Random(n * 1000003 + c["len_hi"])
    new, lens = [at(c["new_lo"], c["new_hi"], i) for i in range(n)], [at(c["len_lo"], c["len_hi"], i) for i in range(n)]
    rng.shuffle(new)
    rng.shuffle(lens)
    return new, [max(a, b) for a, b in zip(new, lens)]


def _visible(c, new, length):
    """(visible pairs of a query and a key, cached rows that some query sees) of one sequence."""
    w, s, before = c["window"], c["sinks"] if c["kind"] != "evict" else 0, length - new
    if not w:
        return new * before + new * (new + 1) // 2, length
    pairs = sum(min(p + 1, w) + min(s, max(0, p + 1 - w)) for p in range(before, length))
    first = max(0, before + 1 - w)
    return pairs, length - first + min(s, first)


def work(c):
    new, lens = _lengths(c)
    e, d, kv, h, t = 4 if c["dtype"] == "f32" else 2, c["head_dim"], c["kv_heads"], c["heads"], sum(new)
    if c["kind"] == "append":
        return {"bytes": 4 * t * kv * d * e, "flops": 0}
    if c["kind"] == "evict":
        cut = [n for n in lens if n > c["budget"]]
        moved = len(cut) * (c["budget"] - c["sinks"])     # the first rows stay where they are
        return {"bytes": kv * (4 * sum(cut) + 4 * moved * d * e + 8 * c["budget"] * len(cut)), "flops": 0}
    seen = [_visible(c, a, b) for a, b in zip(new, lens)]
    pairs, rows = h * sum(p for p, _ in seen), kv * sum(r for _, r in seen)
    if c["kind"] == "weigh":
        return {"bytes": t * h * (d * e + 4) + rows * (d * e + 8), "flops": 2 * d * pairs}
    return {"bytes": t * h * (2 * d * e + 4) + 2 * rows * d * e, "flops": 4 * d * pairs}


def prepare(case, seed):
    c = dict(case)
    new, lens = _lengths(c)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, d, kv, h, page = DTYPES[c["dtype"]], c["head_dim"], c["kv_heads"], c["heads"], c["page"]
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)  # noqa: E731
    counts = [-(-n // page) for n in lens]
    pages = sum(counts) + 3                              # some pages belong to nobody
    order, host, taken = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu(), torch.zeros((len(lens), max(counts)), dtype=torch.int32), 0
    for b, n in enumerate(counts):
        host[b, :n] = order[taken:taken + n]
        taken += n
    s = {"case": c, "new": new, "lens": lens, "table": host.cuda(), "new_dev": torch.tensor(new, device="cuda"), "lens_dev": torch.tensor(lens, device="cuda")}
    s["k_cache"], s["v_cache"] = randn(pages, kv, page, d).to(dt), randn(pages, kv, page, d).to(dt)
    t = sum(new)
    if c["kind"] == "append":
        s["k"], s["v"] = randn(t, kv, d).to(dt), randn(t, kv, d).to(dt)
    elif c["kind"] == "evict":
        w = torch.exp(1.5 * randn(len(lens), kv, max(lens)))           # a few rows hold most of the weight
        s["weights"] = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.03, torch.zeros_like(w), w)   # or none was given
        s["kept"] = torch.full((len(lens), kv, c["budget"]), -1, dtype=torch.int32, device="cuda")
        s["weights_out"] = torch.zeros((len(lens), kv, c["budget"]), dtype=torch.float32, device="cuda")
    else:
        s["q"] = (1.5 * randn(t, h, d)).to(dt)
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((t, h), dtype=torch.float32, device="cuda")
        if c["kind"] == "weigh":                          # what the step's attention left
            s["lse"] = torch.cat([_exact_scores(s, b)[1] for b in range(len(lens))]).float()
            s["weights"] = torch.exp(randn(len(lens), kv, max(lens)))
    if own:
        import paper_2305_13484_amd as fl
        window, sinks = (c["window"], c["sinks"]) if c["kind"] != "evict" else (0, 0)
        s["plan"] = fl.PagedPlan(dt, h, kv, d, page, pages, new, lens, host.numpy(), window=window, sinks=sinks)
    return s


# ------------------------------------------------------------------ the plain forms

def _cached(s, cache):
    """The sequences' cached rows in 32 bits, [sequence][key head][position][head_dim], zeros behind the last."""
    kv, page, pos = s["case"]["kv_heads"], s["case"]["page"], torch.arange(max(s["lens"]), device="cuda")
    rows = cache[s["table"].long()[:, pos // page][:, None], torch.arange(kv, device="cuda")[None, :, None], (pos % page)[None, None]].float()
    return rows.masked_fill((pos >= s["lens_dev"][:, None])[:, None, :, None], 0.0)


def _new_places(s):
    """Of every new token: its sequence, its number in it, its position."""
    b = torch.repeat_interleave(torch.arange(len(s["new"]), device="cuda"), s["new_dev"])
    i = torch.arange(len(b), device="cuda") - (s["new_dev"].cumsum(0) - s["new_dev"])[b]
    return b, i, s["lens_dev"][b] - s["new_dev"][b] + i


def _plain_append(s):
    b, _, pos = _new_places(s)
    page = s["case"]["page"]
    at = s["table"].long()[b, pos // page]
    s["k_cache"][at, :, pos % page] = s["k"]
    s["v_cache"][at, :, pos % page] = s["v"]
    return s["k_cache"], s["v_cache"]


def _scores(s):
    """Scaled scores [sequence][key head][head of its group x new token][position], minus infinity where a key is not visible."""
    c = s["case"]
    b, i, pos = _new_places(s)
    n, kv, d = max(s["new"]), c["kv_heads"], c["head_dim"]
    q = torch.zeros((len(s["new"]), n, c["heads"], d), dtype=torch.float32, device="cuda")
    q[b, i] = s["q"].float()
    group = c["heads"] // kv
    q = q.view(len(s["new"]), n, kv, group, d).permute(0, 2, 3, 1, 4).reshape(len(s["new"]), kv, group * n, d)
    score = torch.matmul(q, _cached(s, s["k_cache"]).transpose(2, 3)).mul_(1 / math.sqrt(d))
    at = (s["lens_dev"] - s["new_dev"])[:, None, None] + torch.arange(n, device="cuda")[None, :, None]
    key = torch.arange(max(s["lens"]), device="cuda")
    hidden = (key > at) | (torch.arange(n, device="cuda")[None, :, None] >= s["new_dev"][:, None, None])
    if c["window"]:
        hidden |= (key <= at - c["window"]) & (key >= c["sinks"])
    score.view(len(s["new"]), kv, group, n, -1).masked_fill_(hidden[:, None, None], float("-inf"))
    return score, b, i


def _by_token(s, x, b, i):
    """[sequence][key head][head of its group x new token][...] to [new token][head][...]."""
    kv, n = s["case"]["kv_heads"], max(s["new"])
    x = x.view(x.shape[0], kv, -1, n, *x.shape[3:])[b, :, :, i]
    return x.reshape(x.shape[0], kv * x.shape[2], *x.shape[3:])


def _plain_attend(s):
    score, b, i = _scores(s)
    top = score.amax(3, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = score.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    out = torch.matmul(p, _cached(s, s["v_cache"])) / total
    return _by_token(s, out, b, i).to(s["q"].dtype), _by_token(s, (top + total.log())[..., 0], b, i)


DECAY = 0.95


def _plain_weigh(s):
    c = s["case"]
    score, b, i = _scores(s)
    lse = torch.zeros((len(s["new"]), max(s["new"]), c["heads"]), dtype=torch.float32, device="cuda")
    lse[b, i] = s["lse"]
    lse = lse.view(*lse.shape[:2], c["kv_heads"], -1).permute(0, 2, 3, 1).reshape(len(s["new"]), c["kv_heads"], -1, 1)
    given = score.sub_(lse).exp_().sum(2)
    pos, n = torch.arange(max(s["lens"]), device="cuda"), s["lens_dev"][:, None]
    old = torch.where((pos < n - s["new_dev"][:, None])[:, None], DECAY * s["weights"], torch.zeros_like(given))     # new rows begin with none
    s["weights"].copy_(torch.where((pos < n)[:, None], old + given, s["weights"]))
    return s["weights"]


def _plain_evict(s):
    c, n = s["case"], s["lens_dev"][:, None, None]
    budget, pos = c["budget"], torch.arange(max(s["lens"]), device="cuda")
    key = torch.where((pos < c["sinks"]) | (pos >= n - c["recent"]), torch.full_like(s["weights"], float("inf")), s["weights"])
    key = torch.where(pos < n, key, torch.full_like(key, -1.0))
    order = torch.sort(key, dim=2, descending=True, stable=True).indices[:, :, :budget]      # ties: the lowest position
    rank = torch.arange(order.shape[2], device="cuda")
    kept = torch.sort(torch.where(rank < n, order, torch.full_like(order, pos.numel())), dim=2).values
    kept = torch.where(n > budget, kept, torch.where(rank < n, rank, torch.full_like(kept, pos.numel())))
    live = kept < n
    at = torch.where(live, kept, torch.zeros_like(kept))
    s["kept"][:, :, :rank.numel()] = torch.where(live, kept, torch.full_like(kept, -1)).to(torch.int32)
    w = s["weights_out"][:, :, :rank.numel()]
    w.copy_(torch.where(live, s["weights"].gather(2, at), w))
    b, h, j = torch.nonzero(live, as_tuple=True)
    src, table, page = at[b, h, j], s["table"].long(), c["page"]
    for cache in (s["k_cache"], s["v_cache"]):
        cache[table[b, j // page], h, j % page] = cache[table[b, src // page], h, src % page]
    return s["k_cache"], s["v_cache"], s["weights_out"], s["kept"]


def run(s):
    c = s["case"]
    if own:
        import paper_2305_13484_amd as fl
        if c["kind"] == "append":
            return fl.k_paged_append(s["plan"], s["k"], s["v"], s["k_cache"], s["v_cache"])
        if c["kind"] == "attend":
            return fl.k_paged_attention(s["plan"], s["q"], s["k_cache"], s["v_cache"], out=s["out"], lse=s["lse"])
        if c["kind"] == "weigh":
            return fl.k_paged_weights(s["plan"], s["q"], s["k_cache"], s["lse"], s["weights"], decay=DECAY)
        fl.k_paged_evict(s["plan"], s["k_cache"], s["v_cache"], s["weights"], c["budget"], first=c["sinks"], recent=c["recent"],
                         weights_out=s["weights_out"], kept=s["kept"])
        return s["k_cache"], s["v_cache"], s["weights_out"], s["kept"]
    return {"append": _plain_append, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}[c["kind"]](s)


# ------------------------------------------------------------------ from the definition, in 64 bits, one sequence after the other

def _exact_rows(s, cache, b):
    """Cached rows of sequence b, [position][key head][head_dim]."""
    page = s["case"]["page"]
    mine = cache[s["table"][b].long()[: -(-s["lens"][b] // page)]]
    return mine.permute(0, 2, 1, 3).reshape(-1, mine.shape[1], mine.shape[3])[: s["lens"][b]]


def _exact_scores(s, b):
    """(scores of every head [head][new token][position] with hidden keys at minus infinity, lse [new token][head])."""
    c, new, n = s["case"], s["new"][b], s["lens"][b]
    first, group, d = sum(s["new"][:b]), c["heads"] // c["kv_heads"], c["head_dim"]
    q = s["q"][first:first + new].double()
    k = _exact_rows(s, s["k_cache"], b).double()
    p, j = torch.arange(n - new, n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    seen = j <= p
    if c["window"]:
        seen &= (p - j < c["window"]) | (j < c["sinks"])
    x = torch.stack([(q[:, h] @ k[:, h // group].T.contiguous()) / math.sqrt(d) for h in range(c["heads"])])
    x[:, ~seen] = float("-inf")
    return x, torch.logsumexp(x, 2).T.contiguous()


def exact(case, seed):
    s = prepare(case, seed)
    c, new, lens, kv, page = s["case"], s["new"], s["lens"], s["case"]["kv_heads"], s["case"]["page"]
    group = c["heads"] // kv
    if c["kind"] == "append":
        k, v = s["k_cache"].double(), s["v_cache"].double()
        rows = [(int(s["table"][b, p // page]), p % page) for b in range(len(new)) for p in range(lens[b] - new[b], lens[b])]
        at, off = (torch.tensor(x, device="cuda") for x in zip(*rows))
        for h in range(kv):
            k[at, h, off], v[at, h, off] = s["k"][:, h].double(), s["v"][:, h].double()
        return k, v
    if c["kind"] == "attend":
        out, lse = [], []
        for b in range(len(new)):
            x, z = _exact_scores(s, b)
            v = _exact_rows(s, s["v_cache"], b).double()
            out.append(torch.stack([torch.exp(x[h] - z[:, h, None]) @ v[:, h // group].contiguous() for h in range(c["heads"])], 1))
            lse.append(z)
        return torch.cat(out), torch.cat(lse)
    if c["kind"] == "weigh":
        w = s["weights"].double()
        for b in range(len(new)):
            x, _ = _exact_scores(s, b)
            first = sum(new[:b])
            p = torch.exp(x - s["lse"][first:first + new[b]].double().T[:, :, None])
            w[b, :, :lens[b] - new[b]] *= DECAY
            w[b, :, lens[b] - new[b]:lens[b]] = 0
            w[b, :, :lens[b]] += p.view(kv, group, new[b], -1).sum((1, 2))
        return w
    k, v, w_out, kept = s["k_cache"].clone(), s["v_cache"].clone(), s["weights_out"].double(), s["kept"]
    table, budget = s["table"].cpu(), c["budget"]
    for b, n in enumerate(lens):
        w = s["weights"][b, :, :n].double().cpu()
        for h in range(kv):
            if n <= budget:
                rows = list(range(n))
            else:
                sure = set(range(c["sinks"])) | set(range(n - c["recent"], n))
                rest = sorted((p for p in range(n) if p not in sure), key=lambda p, v=w[h].tolist(): (-v[p], p))
                rows = sorted(sure | set(rest[: budget - len(sure)]))
            kept[b, h, :len(rows)] = torch.tensor(rows, dtype=torch.int32)
            w_out[b, h, :len(rows)] = w[h, rows].cuda()
            src, dst = torch.tensor(rows), torch.arange(len(rows))
            for new_cache, cache in ((k, s["k_cache"]), (v, s["v_cache"])):
                new_cache[table[b, dst // page].long().cuda(), h, (dst % page).cuda()] = cache[table[b, src // page].long().cuda(), h, (src % page).cuda()]
    return k.double(), v.double(), w_out, kept
