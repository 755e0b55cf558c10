"""The operators of a long generation's decode step: what its keys have been worth, which of them stay in the cache, and what
its tokens do to the next logits.  Cases, plain forms, references.

A case is a dict of plain values.  Its "kind" names the call:
  weights  tkv_key_weights: the attention weight that a step's queries give each key, added to what the key had
  evict    tkv_evict_keys: the first, the last and the heaviest keys of each path and head, moved to a shorter table
  adjust   tkv_adjust_logits: penalties for the tokens of each row's path, biases, and a grammar's mask
Every call takes a batch of rows with block tables, as the attention of drafted trees does: q_lo = q_hi = 1 is single-token
decode, more are drafted trees or (chain) a step that is verified.
The shape of a batch (tables, trees, settings) follows from the case alone; the values from the seed.
With `own` the calls go to the library; without, they are computed in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16


def listed():
    return [
        # one short prompt, a small draft: launches and latency count
        {"name": "weights_tiny", "kind": "weights", "hq": 8, "hkv": 2, "d": 64, "rows": 1, "q_lo": 8, "q_hi": 8, "ctx_lo": 1000,
         "ctx_hi": 1000, "chain": False, "coef": True, "tree": 0},
        # single tokens of a serving batch, ragged contexts: every step, so the keys' bytes count
        {"name": "weights_decode", "kind": "weights", "hq": 12, "hkv": 2, "d": 128, "rows": 64, "q_lo": 1, "q_hi": 1,
         "ctx_lo": 300, "ctx_hi": 6144, "chain": False, "coef": False, "tree": 0},
        # one long context and its draft, of which a part was accepted
        {"name": "weights_long", "kind": "weights", "hq": 28, "hkv": 4, "d": 128, "rows": 1, "q_lo": 32, "q_hi": 32,
         "ctx_lo": 30000, "ctx_hi": 30000, "chain": False, "coef": True, "tree": 0},
        # the last tokens of prompts, whose weights say which of the prompts' keys stay: the arithmetic counts
        {"name": "weights_prompt", "kind": "weights", "hq": 32, "hkv": 8, "d": 128, "rows": 8, "q_lo": 64, "q_hi": 256,
         "ctx_lo": 2000, "ctx_hi": 12000, "chain": True, "coef": False, "tree": 0},
        # a few short paths, small heads, odd numbers
        {"name": "evict_small", "kind": "evict", "hq": 14, "hkv": 2, "d": 64, "rows": 5, "ctx_lo": 301, "ctx_hi": 1501,
         "budget": 255, "sink": 4, "recent": 33, "tree": 0},
        # one long context, cut to a fifteenth
        {"name": "evict_long", "kind": "evict", "hq": 28, "hkv": 4, "d": 128, "rows": 1, "ctx_lo": 30000, "ctx_hi": 30000,
         "budget": 2048, "sink": 4, "recent": 256, "tree": 0},
        # a serving batch; some paths are shorter than the budget and move whole
        {"name": "evict_batch", "kind": "evict", "hq": 12, "hkv": 2, "d": 128, "rows": 64, "ctx_lo": 300, "ctx_hi": 6144,
         "budget": 1024, "sink": 16, "recent": 128, "tree": 0},
        # prompts of a larger model, right after they were read: the copied bytes count
        {"name": "evict_prompts", "kind": "evict", "hq": 32, "hkv": 8, "d": 128, "rows": 32, "ctx_lo": 2000, "ctx_hi": 12000,
         "budget": 2000, "sink": 4, "recent": 500, "tree": 0},
        # a small batch's next tokens, straight from the head's bf16 logits
        {"name": "adjust_few", "kind": "adjust", "rows": 5, "q_lo": 1, "q_hi": 1, "ctx_lo": 200, "ctx_hi": 1000, "vocab": 151936,
         "in16": True, "out16": True, "grammar": 0.2, "bias": 0.2, "tree": 0},
        # the nodes of drafted trees, all of them under a grammar, an odd vocabulary
        {"name": "adjust_trees", "kind": "adjust", "rows": 16, "q_lo": 4, "q_hi": 32, "ctx_lo": 500, "ctx_hi": 6144,
         "vocab": 32003, "in16": True, "out16": False, "grammar": 1.0, "bias": 0.3, "tree": 0},
        # a few requests with very long paths
        {"name": "adjust_long", "kind": "adjust", "rows": 16, "q_lo": 1, "q_hi": 1, "ctx_lo": 8000, "ctx_hi": 30000,
         "vocab": 152064, "in16": False, "out16": False, "grammar": 0.0, "bias": 0.1, "tree": 0},
        # the branching step of a speculative tree
        {"name": "adjust_many", "kind": "adjust", "rows": 1000, "q_lo": 1, "q_hi": 1, "ctx_lo": 100, "ctx_hi": 4000,
         "vocab": 151936, "in16": False, "out16": False, "grammar": 0.1, "bias": 0.1, "tree": 0},
    ]


# query heads, KV heads and head dimension of the repository's configurations and tests
HEADS = [(8, 2, 64), (12, 2, 128), (28, 4, 128), (32, 8, 128), (14, 2, 64), (16, 1, 64), (4, 4, 64), (15, 5, 128),
         (40, 8, 128)]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    hq, hkv, d = rng.choice(HEADS)
    heads = {"hq": hq, "hkv": hkv, "d": d}
    tree = rng.randrange(1 << 20)
    kind = rng.choice(["weights", "evict", "adjust"])
    ctx = log(1, 30000)
    span = {"ctx_lo": max(1, ctx // rng.randint(1, 8)), "ctx_hi": ctx}
    if kind == "weights":
        q = log(1, 256)
        rows = max(1, min(log(1, 64), 400000 // (ctx + q), 250000000 // ((ctx + q) * q * hq)))
        return {"kind": kind, **heads, "rows": rows, "q_lo": rng.randint(1, q), "q_hi": q, **span, "chain": rng.random() < 0.3,
                "coef": rng.random() < 0.5, "tree": tree}
    if kind == "evict":
        budget = log(1, 4000)
        return {"kind": kind, **heads, "rows": max(1, min(log(1, 64), 200000 // ctx)), **span, "budget": budget,
                "sink": rng.choice([0, 1, 4, 64]), "recent": rng.choice([0, 1, budget // 8, budget // 2]), "tree": tree}
    vocab = rng.choice([151936, 152064, 128256, 32000, 32003, 50257, log(500, 150000)])
    q = rng.choice([1, 1, log(1, 32)])
    rows = max(1, min(log(1, 1000), 2_000_000 // ctx, 100_000_000 // (vocab * q)))
    return {"kind": kind, "rows": rows, "q_lo": rng.randint(1, q), "q_hi": q, **span, "vocab": vocab, "in16": rng.random() < 0.5,
            "out16": rng.random() < 0.3, "grammar": rng.choice([0.0, 0.1, 1.0]), "bias": rng.choice([0.0, 0.2]), "tree": tree}


# ----------------------------------------------------------------------------- the batch's shape

def _steps(rng, n):
    """Lengths of the blocks of n tokens: steps of 16 to 256 tokens, each in blocks of its own, the last of them partial."""
    lens = []
    while n > 0:
        m = min(n, int(rng.integers(16, 257)))
        lens += [BLOCK] * ((m - 1) // BLOCK) + [(m - 1) % BLOCK + 1]
        n -= m
    return lens


def _masks(rng, L, words, chain):
    """Bit j of a token's words: it sees drafted token j (itself and its ancestors)."""
    m = np.zeros((L, words), dtype=np.uint64)
    for i in range(L):
        p = i - 1 if chain else int(rng.integers(max(-1, i - 6), i)) if i else -1
        if p >= 0:
            m[i] = m[p]
        m[i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return m


def _batch(case):
    """The batch as the calls take it, on the host."""
    rng = np.random.default_rng([case["tree"], 1])
    n_rows = case["rows"]
    ctx = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=n_rows)
    L = rng.integers(case["q_lo"], case["q_hi"] + 1, size=n_rows) if "q_lo" in case else np.zeros(n_rows, dtype=np.int64)
    lens = [_steps(rng, int(c)) + _steps(rng, int(n)) for c, n in zip(ctx, L)]
    kv_len = ctx + L
    kept = np.minimum(kv_len, case.get("budget", 0))
    n_new = -(-kept // BLOCK)
    n = sum(len(x) for x in lens)
    ids = rng.permutation(n + int(n_new.sum())).astype(np.int32)
    block_len = np.zeros(len(ids), dtype=np.int32)
    block_len[ids[:n]] = np.concatenate(lens)
    words = max(1, -(-int(L.max()) // 64))
    masks = [_masks(rng, int(m), words, case.get("chain", False)) for m in L]
    return {"q_ptr": np.cumsum([0] + [int(x) for x in L]).astype(np.int32),
            "kv_ptr": np.cumsum([0] + [len(x) for x in lens]).astype(np.int32), "kv_len": kv_len, "L": L, "kept": kept,
            "kv_blocks": ids[:n], "block_len": block_len, "max_q": max(1, int(L.max())), "max_blocks": max(len(x) for x in lens),
            "mask": np.concatenate(masks), "new_ptr": np.cumsum([0] + [int(x) for x in n_new]).astype(np.int32),
            "new_blocks": ids[n:]}


def _settings(case, n_tok, kv_len):
    """Each row's penalties and prompt length, its biased tokens, each token's grammar (-1: none)."""
    rng = np.random.default_rng([case["tree"], 2])
    n, vocab = case["rows"], case["vocab"]
    rep = rng.choice([1.0, 1.05, 1.1, 1.3], size=n).astype(np.float32)
    pres = rng.choice([0.0, 0.5, 1.5], size=n).astype(np.float32)
    freq = rng.choice([0.0, 0.1, 0.5], size=n).astype(np.float32)
    prompt = (kv_len * rng.uniform(0.0, 0.9, size=n)).astype(np.int32)
    count = np.where(rng.random(n) < case["bias"], rng.integers(1, min(300, vocab) + 1, size=n), 0)
    ptr = np.cumsum([0] + [int(c) for c in count]).astype(np.int32)
    token = rng.integers(0, vocab, size=int(ptr[-1])).astype(np.int32)
    value = rng.choice([-100.0, -5.0, -1.0, 1.0, 5.0], size=int(ptr[-1])).astype(np.float32)
    grammar = np.where(rng.random(n_tok) < case["grammar"], rng.integers(0, 8, size=n_tok), -1).astype(np.int32)
    return rep, pres, freq, prompt, ptr, token, value, grammar


# ----------------------------------------------------------------------------- inputs and the call

def _normal(g, *shape, scale=1.0, dtype=torch.bfloat16):
    """N(0, scale^2) values drawn in pieces, so that no whole fp32 copy of a large tensor is made."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 26):
        piece = flat[a:a + (1 << 26)]
        piece.copy_(torch.empty(piece.numel(), device="cuda").normal_(0.0, scale, generator=g))
    return out


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    b = _batch(case)
    nb = len(b["block_len"])
    s = {"kind": case["kind"], "max_q": b["max_q"], "max_blocks": b["max_blocks"], "q_indptr": _dev(b["q_ptr"]),
         "kv_indptr": _dev(b["kv_ptr"]), "kv_blocks": _dev(b["kv_blocks"]), "block_len": _dev(b["block_len"]),
         "mask": _dev(b["mask"].view(np.int64))}
    n, rows, keys = int(b["q_ptr"][-1]), case["rows"], BLOCK * b["max_blocks"]
    if case["kind"] == "adjust":
        vocab = case["vocab"]
        rep, pres, freq, prompt, ptr, token, value, grammar = _settings(case, n, b["kv_len"])
        words = -(-vocab // 32)
        # frequent tokens have low numbers
        u = torch.rand(nb, BLOCK, generator=g, device="cuda", dtype=torch.float64)
        # grammars: one of every 32 words has all bits, others a few or none
        bits = torch.randint(0, 1 << 32, (8, words), generator=g, device="cuda")
        bits &= torch.randint(0, 1 << 32, (8, words), generator=g, device="cuda")
        pick = torch.randint(0, 32, (8, words), generator=g, device="cuda")
        bits = torch.where(pick == 0, (1 << 32) - 1, torch.where(pick < 16, bits, 0))
        bits[:, 0] = (1 << 32) - 1
        bits = torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int()
        s.update(tokens=(vocab * u ** 3).int(), prompt_len=_dev(prompt), repetition=_dev(rep), presence=_dev(pres),
                 frequency=_dev(freq), bias_indptr=_dev(ptr), bias_token=_dev(token), bias_value=_dev(value),
                 grammar=_dev(grammar), allowed=bits,
                 logits=_normal(g, n, vocab, scale=3.0, dtype=torch.bfloat16 if case["in16"] else torch.float32),
                 out=torch.empty(n, vocab, dtype=torch.bfloat16 if case["out16"] else torch.float32, device="cuda"))
        return s
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    # what keys were worth: over several orders of magnitude, and nothing at all for some
    w = torch.exp(2.0 * torch.randn(rows, hkv, keys, generator=g, device="cuda") - 6.0)
    w = torch.where(torch.rand(rows, hkv, keys, generator=g, device="cuda") < 0.05, 0.0, w)
    s.update(k=_normal(g, nb, hkv, BLOCK, d), before=w)
    if case["kind"] == "evict":
        most = case["budget"]
        s.update(v=_normal(g, nb, hkv, BLOCK, d), sink=case["sink"], recent=case["recent"], new_indptr=_dev(b["new_ptr"]),
                 new_blocks=_dev(b["new_blocks"]), budget=torch.full((rows,), most, dtype=torch.int32, device="cuda"),
                 kept=torch.empty(rows, hkv, most, dtype=torch.int32, device="cuda"),
                 n_kept=torch.empty(rows, dtype=torch.int32, device="cuda"), weights=torch.zeros_like(w))
        return s
    s.update(q=_normal(g, n, hq, d), weights=torch.zeros_like(w), decay=0.95, coef=None)
    if case["coef"]:
        s["coef"] = (torch.rand(n, generator=g, device="cuda") < 0.7).float()
    x, _, _ = _scores(s)
    lse = torch.logsumexp(x, -1)                                  # [rows, hkv, most tokens, G]
    row, i = _token_rows(s)
    s["lse"] = lse.transpose(1, 2)[row, i].reshape(n, hq).contiguous()
    return s


def run(state):
    s = state
    if own:
        import paper_2609_39334_amd as tkv
        if s["kind"] == "weights":
            tkv.tkv_key_weights(s["q_indptr"], s["kv_indptr"], s["kv_blocks"], s["block_len"], s["mask"], s["max_q"],
                                s["max_blocks"], s["q"], s["k"], s["lse"], s["weights"], before=s["before"], decay=s["decay"],
                                coef=s["coef"])
            return [s["weights"]]
        if s["kind"] == "evict":
            tkv.tkv_evict_keys(s["kv_indptr"], s["kv_blocks"], s["block_len"], s["max_blocks"], s["new_indptr"], s["new_blocks"],
                               s["budget"], s["sink"], s["recent"], s["before"], s["k"], s["v"], s["weights"], s["kept"],
                               s["n_kept"])
            return [s["kept"], s["n_kept"], s["weights"], s["k"], s["v"]]
        tkv.tkv_adjust_logits(s["q_indptr"], s["kv_indptr"], s["kv_blocks"], s["block_len"], s["mask"], s["max_q"],
                              s["max_blocks"], s["tokens"], s["logits"], prompt_len=s["prompt_len"], repetition=s["repetition"],
                              presence=s["presence"], frequency=s["frequency"], bias_indptr=s["bias_indptr"],
                              bias_token=s["bias_token"], bias_value=s["bias_value"], grammar=s["grammar"],
                              allowed=s["allowed"], out=s["out"])
        return [s["out"]]
    return {"weights": _plain_weights, "evict": _plain_evict, "adjust": _plain_adjust}[s["kind"]](s)


# ----------------------------------------------------------------------------- plain forms

def _table(s):
    """Each row's blocks, padded with block 0 [rows, max_blocks]; whether a slot of them holds a key [rows, keys], and the
    key's number in the path; the rows' lengths."""
    at = s["kv_indptr"][:-1, None].long() + torch.arange(s["max_blocks"], device="cuda")
    inside = at < s["kv_indptr"][1:, None]
    ids = torch.where(inside, s["kv_blocks"][at.clamp(max=len(s["kv_blocks"]) - 1)], 0).long()
    lens = torch.where(inside, s["block_len"][ids], 0).long()
    slot = torch.arange(BLOCK, device="cuda")
    live = (slot < lens[..., None]).flatten(1)
    number = ((torch.cumsum(lens, 1) - lens)[..., None] + slot).flatten(1)
    return ids, live, number, lens.sum(1)


def _token_rows(s):
    """Each query token's row, and its place in it."""
    n = torch.arange(len(s["mask"]), device="cuda")
    row = torch.searchsorted(s["q_indptr"][1:].contiguous(), n, right=True)
    return row, n - s["q_indptr"][row]


def _scores(s):
    """log2-free scores of the rows' tokens against their slots [rows, hkv, tokens, G, keys] in fp32, -inf where a token does
    not see a slot's key; the slots that hold keys, and whether these were there before the step."""
    ids, live, number, N = _table(s)
    hq, d = s["q"].shape[1:]
    hkv, most = s["k"].shape[1], s["max_q"]
    rows, keys = live.shape
    L = (s["q_indptr"][1:] - s["q_indptr"][:-1]).long()
    t = torch.arange(most, device="cuda")
    at = (s["q_indptr"][:-1, None] + t).clamp(max=len(s["mask"]) - 1).long()
    q = s["q"][at].float().view(rows, most, hkv, -1, d).permute(0, 2, 1, 3, 4).reshape(rows * hkv, -1, d)
    k = s["k"][ids].float().permute(0, 2, 4, 1, 3).reshape(rows * hkv, d, keys)
    x = torch.matmul(q, k).view(rows, hkv, most, hq // hkv, keys) / math.sqrt(d)
    j = number - (N - L)[:, None]                                 # a key's number among the step's (negative: context)
    jc = j.clamp(min=0).clamp(max=64 * s["mask"].shape[1] - 1)
    word = s["mask"][at].gather(2, (jc // 64)[:, None, :].expand(rows, most, keys))
    seen = (j < 0)[:, None] | ((word >> (jc % 64)[:, None]) & 1 == 1)
    seen = seen & live[:, None] & (t < L[:, None])[..., None]
    return torch.where(seen[:, None, :, None], x, -math.inf), live, live & (j < 0)


def _plain_weights(s):
    x, live, context = _scores(s)
    rows, hkv, most, G, keys = x.shape
    t = torch.arange(most, device="cuda")
    at = (s["q_indptr"][:-1, None] + t).clamp(max=len(s["mask"]) - 1).long()
    lse = s["lse"][at].view(rows, most, hkv, G).transpose(1, 2)
    p = torch.exp(x - lse[..., None])
    if s["coef"] is not None:
        p = p * s["coef"][at][:, None, :, None, None]
    w = p.sum((2, 3)) + torch.where(context[:, None], s["decay"] * s["before"], 0.0)
    s["weights"].copy_(torch.where(live[:, None], w, s["weights"]))
    return [s["weights"]]


def _plain_evict(s):
    ids, live, number, N = _table(s)
    rows, hkv, keys = s["before"].shape
    n_kept = torch.minimum(N, s["budget"].long())
    sink = n_kept.clamp(max=s["sink"])
    recent = (n_kept - sink).clamp(max=s["recent"])
    always = (number < sink[:, None]) | (number >= (N - recent)[:, None])
    worth = torch.where(always[:, None], math.inf, s["before"])
    worth = torch.where(live[:, None], worth, -math.inf)
    order = torch.sort(worth, dim=2, descending=True, stable=True)[1]
    rank = torch.empty_like(order).scatter_(2, order, torch.arange(keys, device="cuda").expand(rows, hkv, keys))
    keep = live[:, None] & (rank < n_kept[:, None, None])
    most = s["kept"].shape[2]
    place = torch.where(keep, torch.cumsum(keep, 2) - 1, most)    # of a kept key in the new path
    index = torch.arange(keys, device="cuda").expand(rows, hkv, keys)
    kept = torch.full((rows, hkv, most + 1), -1, dtype=torch.long, device="cuda").scatter_(2, place, index)[..., :most]
    s["kept"].copy_(kept)
    s["n_kept"].copy_(n_kept)
    new = torch.arange(most, device="cuda")
    there = (new < n_kept[:, None])[:, None].expand(rows, hkv, most)
    src = kept.clamp(min=0)
    m = min(most, keys)
    moved = s["before"].gather(2, src[..., :m])
    s["weights"][..., :m].copy_(torch.where(there[..., :m], moved, s["weights"][..., :m]))
    r, h, i = torch.nonzero(there, as_tuple=True)
    src = src[r, h, i]
    to = s["new_blocks"][(s["new_indptr"][r] + i // BLOCK).long()].long()
    for pool in (s["k"], s["v"]):
        pool[to, h, i % BLOCK] = pool[ids[r, src // BLOCK], h, src % BLOCK]
    return [s["kept"], s["n_kept"], s["weights"], s["k"], s["v"]]


def _plain_adjust(s):
    ids, live, number, N = _table(s)
    n, vocab = s["logits"].shape
    rows, keys = live.shape
    L = (s["q_indptr"][1:] - s["q_indptr"][:-1]).long()
    token = s["tokens"][ids].flatten(1).long()
    j = number - (N - L)[:, None]
    # what every token of a row sees: how often each token of the vocabulary occurs in the context, in all and past the prompt
    later = number >= s["prompt_len"][:, None]
    one = torch.ones(rows, keys, dtype=torch.int32, device="cuda")
    seen = torch.zeros(rows, vocab + 1, dtype=torch.int32, device="cuda")
    count = seen.clone()
    seen.scatter_add_(1, torch.where(live & (j < 0), token, vocab), one)
    count.scatter_add_(1, torch.where(live & (j < 0) & later, token, vocab), one)
    # and what each sees of the drafted ones
    most = s["max_q"]
    drafted = torch.full((rows, most + 1), vocab, dtype=torch.long, device="cuda")
    past = torch.zeros(rows, most + 1, dtype=torch.bool, device="cuda")
    place = torch.where(live & (j >= 0), j, most)
    drafted.scatter_(1, place, token)
    past.scatter_(1, place, later)
    row, _ = _token_rows(s)
    t = torch.arange(most, device="cuda")
    bit = ((s["mask"][:, t // 64] >> (t % 64)) & 1 == 1) & (t < L[row][:, None])
    at = torch.where(bit, drafted[row, :most], vocab)
    seen, count = seen[row], count[row]
    one = torch.ones_like(at, dtype=torch.int32)
    seen.scatter_add_(1, at, one)
    count.scatter_add_(1, torch.where(past[row, :most], at, vocab), one)
    seen, count = seen[:, :vocab], count[:, :vocab]

    x = s["logits"].float()
    rep = s["repetition"][row][:, None]
    x = torch.where(seen > 0, torch.where(x > 0, x / rep, x * rep), x)
    x = x - s["frequency"][row][:, None] * count - torch.where(count > 0, s["presence"][row][:, None], 0.0)
    # the last of a token's biases
    m = len(s["bias_token"])
    if m:
        owner = torch.searchsorted(s["bias_indptr"][1:].contiguous(), torch.arange(m, device="cuda"), right=True)
        entry = torch.zeros(rows * vocab, dtype=torch.int32, device="cuda")
        entry.scatter_reduce_(0, owner * vocab + s["bias_token"], torch.arange(1, m + 1, dtype=torch.int32, device="cuda"), "amax")
        entry = entry.view(rows, vocab)[row]
        x = x + torch.where(entry > 0, s["bias_value"][(entry - 1).clamp(min=0)], 0.0)
    v = torch.arange(vocab, device="cuda")
    word = s["allowed"][s["grammar"].clamp(min=0)][:, v // 32]
    free = (s["grammar"] < 0)[:, None] | ((word >> (v % 32).int()) & 1 == 1)
    s["out"].copy_(torch.where(free, x, -math.inf))
    return [s["out"]]


# ----------------------------------------------------------------------------- what it cannot do without

def work(case):
    b = _batch(case)
    rows, total, table = case["rows"], int(b["kv_len"].sum()), 8 * len(b["kv_blocks"])
    if case["kind"] == "adjust":
        n, vocab = int(b["q_ptr"][-1]), case["vocab"]
        grammar = _settings(case, n, b["kv_len"])[7]
        return {"bytes": n * vocab * ((2 if case["in16"] else 4) + (2 if case["out16"] else 4)) + 4 * total + table
                + int((np.unique(grammar) >= 0).sum()) * vocab // 8, "flops": 4 * n * vocab}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["kind"] == "evict":
        kept = int(b["kept"].sum())
        return {"bytes": 4 * hkv * total + table + kept * hkv * (8 * d + 8) + 4 * rows, "flops": hkv * total}
    n, words = b["mask"].shape
    drafted = int(np.unpackbits(b["mask"].view(np.uint8)).sum())
    seen = drafted + int((b["L"] * (b["kv_len"] - b["L"])).sum())
    return {"bytes": hkv * (2 * d + 8) * total + n * (hq * (2 * d + 4) + 8 * words) + table, "flops": 2 * d * hq * seen}


# ----------------------------------------------------------------------------- the same in 64 bits

def _path(b, r):
    """The slots of row r's path, in order: their index in its table, and their place in the pool."""
    ids = b["kv_blocks"][b["kv_ptr"][r]:b["kv_ptr"][r + 1]]
    lens = b["block_len"][ids]
    index = np.concatenate([BLOCK * e + np.arange(n) for e, n in enumerate(lens)])
    return index, ids[index // BLOCK].astype(np.int64) * BLOCK + index % BLOCK


def _bits(b, r):
    """Which of its drafted tokens each of row r's tokens sees, [L, L]."""
    m = b["mask"][b["q_ptr"][r]:b["q_ptr"][r + 1]]
    return np.unpackbits(m.view(np.uint8).reshape(len(m), -1), axis=1, bitorder="little")[:, :len(m)].astype(bool)


def _exact_weights(case, b, s):
    out = torch.zeros_like(s["before"], dtype=torch.float64)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    G = hq // hkv
    for r in range(case["rows"]):
        index, at = (_dev(x) for x in _path(b, r))
        a, e = int(b["q_ptr"][r]), int(b["q_ptr"][r + 1])
        hidden = np.zeros((e - a, len(at)), dtype=bool)
        hidden[:, len(at) - (e - a):] = ~_bits(b, r)
        hidden = _dev(hidden)
        for h in range(hkv):
            keys = s["k"][at // BLOCK, h, at % BLOCK].double()
            had = 0.95 * s["before"][r, h, index].double()
            had[len(at) - (e - a):] = 0
            for c in range(G * h, G * h + G):
                x = s["q"][a:e, c].double() @ keys.t().contiguous() * d ** -0.5
                p = torch.exp(x - s["lse"][a:e, c, None].double()).masked_fill(hidden, 0.0)
                had += (torch.ones(e - a, device="cuda").double() if s["coef"] is None else s["coef"][a:e].double()) @ p
            out[r, h, index] = had
    return [out]


def _exact_evict(case, b, s):
    k, v, w = s["k"].double(), s["v"].double(), torch.zeros_like(s["before"], dtype=torch.float64)
    before = s["before"].cpu().numpy().astype(np.float64)
    for r in range(case["rows"]):
        index, at = _path(b, r)
        n, N = int(b["kept"][r]), len(at)
        first = min(case["sink"], n)
        last = min(case["recent"], n - first)
        to = b["new_blocks"][b["new_ptr"][r]:b["new_ptr"][r + 1]].astype(np.int64)
        to = _dev((to[:, None] * BLOCK + np.arange(BLOCK)).reshape(-1)[:n])
        for h in range(case["hkv"]):
            x = before[r, h, index]
            middle = np.arange(first, N - last)
            pick = middle[np.lexsort((middle, -x[middle]))[:n - first - last]]
            keep = np.sort(np.concatenate((np.arange(first), pick, np.arange(N - last, N))))
            w[r, h, :n] = _dev(x[keep])
            src = _dev(at[keep])
            for new, pool in ((k, s["k"]), (v, s["v"])):
                new[to // BLOCK, h, to % BLOCK] = pool[src // BLOCK, h, src % BLOCK].double()
    return [None, None, w, k, v]


def _exact_adjust(case, b, s):
    vocab, n = case["vocab"], int(b["q_ptr"][-1])
    rep, pres, freq, prompt, ptr, token, value, grammar = _settings(case, n, b["kv_len"])
    said = s["tokens"].cpu().numpy().reshape(-1)
    allowed = np.unpackbits(s["allowed"].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :vocab].astype(bool)
    allowed = _dev(allowed)
    out = torch.empty(n, vocab, dtype=torch.float64, device="cuda")
    for r in range(case["rows"]):
        path = said[_path(b, r)[1]]
        L = int(b["L"][r])
        see = _bits(b, r)
        for i in range(L):
            x = s["logits"][b["q_ptr"][r] + i].double()
            visible = np.concatenate((np.ones(len(path) - L, dtype=bool), see[i]))
            at = _dev(np.unique(path[visible]).astype(np.int64))
            y = x[at]
            x[at] = torch.where(y > 0, y / float(rep[r]), y * float(rep[r]))
            kind, times = np.unique(path[visible & (np.arange(len(path)) >= prompt[r])], return_counts=True)
            x[_dev(kind.astype(np.int64))] -= _dev(float(freq[r]) * times + float(pres[r]))
            given = dict(zip(token[ptr[r]:ptr[r + 1]].tolist(), value[ptr[r]:ptr[r + 1]].tolist()))
            if given:
                x[_dev(np.array(list(given), dtype=np.int64))] += _dev(np.array(list(given.values())))
            m = grammar[b["q_ptr"][r] + i]
            out[b["q_ptr"][r] + i] = x if m < 0 else x.masked_fill(~allowed[m], -math.inf)
    return [out]


def exact(case, seed):
    s, b = prepare(case, seed), _batch(case)
    return {"weights": _exact_weights, "evict": _exact_evict, "adjust": _exact_adjust}[case["kind"]](case, b, s)
