"""The operators of a decode step that drafts a small tree of tokens and verifies it: cases, plain forms, references.

A case is a dict of plain values.  Its "kind" names the call:
  append  tkv_norm_rope_append: norm of each query and key head, rotation, packed queries, K/V written to the pool
  draft   tkv_draft_verify: attention of each row's drafted tokens over its block table, under a visibility mask
  sample  tkv_filter_sample: draws under temperature, top-k, top-p and min-p, grouped by token
The shape of a batch (tables, trees, slots, sampling parameters) follows from the case alone; the values from the seed.
With `own` the calls go to the library; without, they are computed in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16


def listed():
    return [
        # the four rows of a small search append one token each: launches and latency count
        {"name": "append_one", "kind": "append", "hq": 28, "hkv": 4, "d": 128, "rot": 128, "rows": 4, "len_lo": 1, "len_hi": 1,
         "skip": 0.0, "tree": 0},
        # drafted trees of a serving batch, small heads, half of each head rotated, an odd number of tokens
        {"name": "append_nodes", "kind": "append", "hq": 14, "hkv": 2, "d": 64, "rot": 32, "rows": 61, "len_lo": 5,
         "len_hi": 32, "skip": 0.0, "tree": 0},
        # prompts: completed steps of many candidates, a fifth of them already in the pool
        {"name": "append_prompts", "kind": "append", "hq": 32, "hkv": 8, "d": 128, "rot": 128, "rows": 160, "len_lo": 16,
         "len_hi": 190, "skip": 0.2, "tree": 0},
        # one query, a draft of a few tokens under a short prompt
        {"name": "draft_tiny", "kind": "draft", "hq": 8, "hkv": 2, "d": 64, "rows": 1, "q_lo": 8, "q_hi": 8, "ctx_lo": 1000,
         "ctx_hi": 1000, "tree": 0},
        # rows without a draft: single tokens of a serving batch, ragged contexts
        {"name": "draft_single", "kind": "draft", "hq": 12, "hkv": 2, "d": 128, "rows": 64, "q_lo": 1, "q_hi": 1,
         "ctx_lo": 300, "ctx_hi": 6144, "tree": 0},
        # one long context, one tree: the keys have to be split over the chip
        {"name": "draft_long", "kind": "draft", "hq": 28, "hkv": 4, "d": 128, "rows": 1, "q_lo": 32, "q_hi": 32,
         "ctx_lo": 30000, "ctx_hi": 30000, "tree": 0},
        # a serving batch of drafted trees of different sizes under ragged contexts
        {"name": "draft_batch", "kind": "draft", "hq": 28, "hkv": 4, "d": 128, "rows": 32, "q_lo": 4, "q_hi": 32,
         "ctx_lo": 500, "ctx_hi": 6144, "tree": 0},
        # wide trees: the arithmetic counts
        {"name": "draft_wide", "kind": "draft", "hq": 32, "hkv": 8, "d": 128, "rows": 8, "q_lo": 64, "q_hi": 150,
         "ctx_lo": 2000, "ctx_hi": 12000, "tree": 0},
        # a small batch's next tokens, straight from the head's bf16 logits, with one setting for all rows
        {"name": "sample_few", "kind": "sample", "rows": 5, "vocab": 151936, "bf16": True, "potential_hi": 1, "mixed": False,
         "flat": 0.0, "tree": 0},
        # the nodes of drafted trees, each drawn once, requests with settings of their own
        {"name": "sample_nodes", "kind": "sample", "rows": 250, "vocab": 152064, "bf16": False, "potential_hi": 1,
         "mixed": True, "flat": 0.1, "tree": 0},
        # a smaller vocabulary of odd size, several draws a row
        {"name": "sample_odd", "kind": "sample", "rows": 333, "vocab": 32003, "bf16": True, "potential_hi": 64, "mixed": True,
         "flat": 0.1, "tree": 0},
        # the branching step of a speculative tree
        {"name": "sample_many", "kind": "sample", "rows": 1000, "vocab": 151936, "bf16": False, "potential_hi": 4,
         "mixed": True, "flat": 0.1, "tree": 0},
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
    kind = rng.choice(["append", "draft", "draft", "sample", "sample"])
    if kind == "append":
        hi = log(1, 128)
        return {"kind": kind, **heads, "rot": rng.choice([d, d, d // 2, d // 4]), "rows": log(1, 130), "len_lo": (hi + 1) // 2,
                "len_hi": hi, "skip": rng.choice([0.0, 0.2]), "tree": tree}
    if kind == "draft":
        q = log(1, 150)
        ctx = log(1, 30000)
        rows = max(1, min(log(1, 64), 400000 // (ctx + q), 100000000 // ((ctx + q) * q * hq)))
        return {"kind": kind, **heads, "rows": rows, "q_lo": rng.randint(1, q), "q_hi": q, "ctx_lo": ctx // rng.randint(1, 8),
                "ctx_hi": ctx, "tree": tree}
    vocab = rng.choice([151936, 152064, 128256, 32000, 32003, 50257, log(500, 150000)])
    return {"kind": kind, "rows": min(log(1, 1000), 150_000_000 // vocab), "vocab": vocab, "bf16": rng.random() < 0.5,
            "potential_hi": log(1, 64), "mixed": rng.random() < 0.7, "flat": rng.choice([0.0, 0.1, 0.3]), "tree": tree}


# ----------------------------------------------------------------------------- the batch's shape

def _slots(case):
    """The new tokens' pool slots and the pool's blocks: each row's step in scattered blocks of its own, some steps
    deduplicated (no slot); single tokens go somewhere into their row's last block."""
    rng = np.random.default_rng([case["tree"], 1])
    n = rng.integers(case["len_lo"], case["len_hi"] + 1, size=case["rows"])
    blocks = -(-n // BLOCK)
    ids = rng.permutation(int(blocks.sum()))
    first = np.cumsum(blocks) - blocks
    dst = []
    for m, b in zip(n, first):
        at = np.arange(m) + (int(rng.integers(0, BLOCK)) if m == 1 else 0)
        s = ids[b + at // BLOCK] * BLOCK + at % BLOCK
        dst.append(np.full(m, -1) if rng.random() < case["skip"] else s)
    return np.concatenate(dst).astype(np.int32), int(blocks.sum())


def _trees(case):
    """Per row: context length, the lengths of its path's blocks (steps of 16 to 256 tokens, the last block of a step
    partial; the draft continues the last block or starts its own) and each drafted token's parent (-1: the context)."""
    rng = np.random.default_rng([case["tree"], 2])
    rows = []
    for _ in range(case["rows"]):
        ctx = int(rng.integers(case["ctx_lo"], case["ctx_hi"] + 1))
        L = int(rng.integers(case["q_lo"], case["q_hi"] + 1))
        steps, left = [], ctx
        while left > 0:
            n = min(left, int(rng.integers(16, 257)))
            steps.append(n)
            left -= n
        if steps and rng.random() < 0.5:
            steps[-1] += L
        else:
            steps.append(L)
        lens = []
        for n in steps:
            lens += [BLOCK] * ((n - 1) // BLOCK) + [(n - 1) % BLOCK + 1]
        parent = [-1] + [int(rng.integers(max(-1, i - 6), i)) for i in range(1, L)]
        rows.append((ctx, lens, parent))
    return rows


def _mask(parent, words):
    """Bit j of a token's words: it sees drafted token j (itself and its ancestors)."""
    m = np.zeros((len(parent), words), dtype=np.uint64)
    for i, p in enumerate(parent):
        if p >= 0:
            m[i] = m[p]
        m[i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return m


def _batch(case):
    """The batch as the call takes it, on the host."""
    rows = _trees(case)
    n_blocks = sum(len(lens) for _, lens, _ in rows)
    ids = np.random.default_rng([case["tree"], 3]).permutation(n_blocks).astype(np.int32)
    block_len = np.zeros(n_blocks, dtype=np.int32)
    block_len[ids] = np.concatenate([lens for _, lens, _ in rows])
    max_q = max(len(p) for _, _, p in rows)
    words = -(-max_q // 64)
    return {"q_ptr": np.cumsum([0] + [len(p) for _, _, p in rows]), "kv_ptr": np.cumsum([0] + [len(l) for _, l, _ in rows]),
            "kv_len": [c + len(p) for c, _, p in rows], "kv_blocks": ids, "block_len": block_len, "max_q": max_q,
            "max_blocks": max(len(l) for _, l, _ in rows), "mask": np.concatenate([_mask(p, words) for _, _, p in rows])}


def _settings(case):
    """Each row's temperature, top-k (0: off), top-p and min-p (1 and 0: off), and its number of draws."""
    rng = np.random.default_rng([case["tree"], 4])
    n = case["rows"]
    temp, k = np.full(n, 0.8), np.full(n, 20)
    p, m = np.full(n, 0.95), np.zeros(n)
    if case["mixed"]:
        temp = rng.choice([0.0, 0.6, 0.8, 1.0, 1.3], size=n, p=[0.1, 0.2, 0.4, 0.2, 0.1])
        k = rng.choice([0, 1, 20, 50, 200, 1000], size=n, p=[0.4, 0.04, 0.25, 0.2, 0.1, 0.01])
        p = rng.choice([1.0, 0.8, 0.9, 0.95], size=n, p=[0.25, 0.15, 0.2, 0.4])
        m = rng.choice([0.0, 0.02, 0.1], size=n, p=[0.6, 0.2, 0.2])
    potential = np.minimum(rng.geometric(0.5, size=n), case["potential_hi"])
    if case["potential_hi"] > 8:
        potential[rng.integers(0, n, size=max(1, n // 16))] = case["potential_hi"]
    return temp.astype(np.float32), k.astype(np.int32), p.astype(np.float32), m.astype(np.float32), potential.astype(np.int32)


# ----------------------------------------------------------------------------- inputs and the call

def _normal(g, *shape, scale=1.0, dtype=torch.bfloat16):
    """N(0, scale^2) values drawn in pieces, so that no whole fp32 copy of a large tensor is made."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 26):
        piece = flat[a:a + (1 << 26)]
        piece.copy_(torch.empty(piece.numel(), device="cuda").normal_(0.0, scale, generator=g))
    return out


def _logits(case, g):
    """Next-token logits: a bulk of N(0, 2^2) and 64 tokens above it whose logits fall with the logarithm of their rank,
    by a slope and from a height of each row's own (confident rows and undecided ones); a part of the rows is bulk alone."""
    rows, vocab = case["rows"], case["vocab"]
    x = _normal(g, rows, vocab, scale=2.0, dtype=torch.bfloat16 if case["bf16"] else torch.float32)
    top = 9.0 + 6.0 * torch.rand(rows, 1, generator=g, device="cuda")
    slope = 0.6 + 1.6 * torch.rand(rows, 1, generator=g, device="cuda")
    rank = torch.arange(1, 65, device="cuda").float()[None, :]
    head = top - slope * torch.log(rank) + 0.1 * torch.randn(rows, 64, generator=g, device="cuda")
    at = torch.randint(0, vocab, (rows, 64), generator=g, device="cuda")
    head = torch.where(torch.rand(rows, 1, generator=g, device="cuda") < case["flat"], x.gather(1, at).float(), head)
    # the same token twice: its last value, written in order
    for j in range(64):
        x.scatter_(1, at[:, j:j + 1], head[:, j:j + 1].to(x.dtype))
    return x


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = case["kind"]
    if kind == "append":
        dst, nb = _slots(case)
        n, hq, hkv, d, rot = len(dst), case["hq"], case["hkv"], case["d"], case["rot"]
        pos = torch.randint(0, 32768, (n, 1), generator=g, device="cuda").double()
        angle = pos * 1e6 ** (-torch.arange(rot // 2, device="cuda").double() * 2 / rot)
        return {"kind": kind, "hq": hq, "eps": 1e-6, "dst": _dev(dst), "qkv": _normal(g, n, (hq + 2 * hkv) * d),
                "cos": torch.cos(angle).float(), "sin": torch.sin(angle).float(),
                "wq": torch.empty(d, device="cuda").uniform_(0.5, 1.5, generator=g),
                "wk": torch.empty(d, device="cuda").uniform_(0.5, 1.5, generator=g),
                "k": _normal(g, nb, hkv, BLOCK, d), "v": _normal(g, nb, hkv, BLOCK, d)}
    if kind == "draft":
        b = _batch(case)
        n, hq, hkv, d, nb = int(b["q_ptr"][-1]), case["hq"], case["hkv"], case["d"], len(b["block_len"])
        return {"kind": kind, "q_ptr": [int(x) for x in b["q_ptr"]], "kv_ptr": [int(x) for x in b["kv_ptr"]],
                "kv_len": b["kv_len"], "max_q": b["max_q"], "max_blocks": b["max_blocks"],
                "q_indptr": _dev(b["q_ptr"].astype(np.int32)), "kv_indptr": _dev(b["kv_ptr"].astype(np.int32)),
                "kv_blocks": _dev(b["kv_blocks"]), "block_len": _dev(b["block_len"]), "mask": _dev(b["mask"].view(np.int64)),
                "q": _normal(g, n, hq, d), "k": _normal(g, nb, hkv, BLOCK, d), "v": _normal(g, nb, hkv, BLOCK, d),
                "o": torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda"),
                "lse": torch.empty(n, hq, dtype=torch.float32, device="cuda")}
    temp, k, p, m, potential = _settings(case)
    off = np.concatenate([[0], np.cumsum(potential)]).astype(np.int32)
    return {"kind": kind, "logits": _logits(case, g), "temperature": _dev(temp), "top_k": _dev(k), "top_p": _dev(p),
            "min_p": _dev(m), "off": _dev(off), "uniform": torch.rand(int(off[-1]), generator=g, device="cuda"),
            "max_potential": int(potential.max())}


def run(state):
    s = state
    if own:
        import paper_2609_39334_amd as tkv
        if s["kind"] == "append":
            q = tkv.tkv_norm_rope_append(s["qkv"], s["wq"], s["wk"], s["eps"], s["cos"], s["sin"], s["dst"], s["hq"], s["k"],
                                         s["v"])
            return [q, s["k"], s["v"]]
        if s["kind"] == "draft":
            tkv.tkv_draft_verify(s["q_indptr"], s["kv_indptr"], s["kv_blocks"], s["block_len"], s["mask"], s["max_q"],
                                 s["max_blocks"], s["q"], s["k"], s["v"], s["o"], s["lse"])
            return [s["o"], s["lse"]]
        return list(tkv.tkv_filter_sample(s["logits"], s["temperature"], s["off"], s["uniform"], s["max_potential"],
                                          s["top_k"], s["top_p"], s["min_p"]))
    return {"append": _plain_append, "draft": _plain_draft, "sample": _plain_sample}[s["kind"]](s)


# ----------------------------------------------------------------------------- plain forms

def _plain_append(s):
    nb, hkv, _, d = s["k"].shape
    n, hq = len(s["dst"]), s["hq"]
    half = s["cos"].shape[1]
    heads = s["qkv"].view(n, hq + 2 * hkv, d).float()

    def normed(x, w):
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * w
        a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
        c, t = s["cos"][:, None, :], s["sin"][:, None, :]
        return torch.cat((a * c - b * t, b * c + a * t, rest), -1).bfloat16()

    q, k = normed(heads[:, :hq], s["wq"]), normed(heads[:, hq:hq + hkv], s["wk"])
    v = heads[:, hq + hkv:].bfloat16()
    # which token each slot of the pool takes (-1: none); tokens without a slot go to one past the pool
    slots = nb * BLOCK
    at = torch.where((s["dst"] >= 0) & (s["dst"] < slots), s["dst"].long(), slots)
    src = torch.full((slots + 1,), -1, dtype=torch.long, device=q.device)
    src.scatter_(0, at, torch.arange(n, device=q.device))
    src = src[:slots].view(nb, BLOCK)
    taken = (src >= 0)[:, None, :, None]
    for pool, new in ((s["k"], k), (s["v"], v)):
        pool.copy_(torch.where(taken, new[src.clamp(min=0)].transpose(1, 2), pool))
    return [q, s["k"], s["v"]]


def _plain_draft(s):
    q, k, v = s["q"], s["k"], s["v"]
    hq, d = q.shape[1:]
    hkv = k.shape[1]
    slot = torch.arange(BLOCK, device=q.device)
    for r, N in enumerate(s["kv_len"]):
        a, L = s["q_ptr"][r], s["q_ptr"][r + 1] - s["q_ptr"][r]
        ids = s["kv_blocks"][s["kv_ptr"][r]:s["kv_ptr"][r + 1]].long()
        lens = s["block_len"][ids].long()
        live = (slot[None, :] < lens[:, None]).view(-1)
        keys = k[ids].transpose(0, 1).reshape(hkv, -1, d).float()
        vals = torch.where(live[None, :, None], v[ids].transpose(0, 1).reshape(hkv, -1, d).float(), 0.0)
        # a key's number among the drafted tokens (negative: context)
        j = ((torch.cumsum(lens, 0) - lens)[:, None] + slot[None, :]).view(-1) - (N - L)
        jc = j.clamp(0, L - 1)
        bit = (s["mask"][a:a + L][:, jc // 64] >> (jc % 64)) & 1
        seen = live & ((j < 0) | (bit == 1))
        qs = q[a:a + L].view(L, hkv, -1, d).permute(1, 2, 0, 3).reshape(hkv, -1, d).float()
        x = torch.matmul(qs, keys.transpose(1, 2).contiguous()).view(hkv, hq // hkv, L, -1) / math.sqrt(d)
        x = torch.where(seen, x, -math.inf)
        top = x.amax(-1, keepdim=True).clamp(min=-3e38)
        p = torch.exp(x - top)
        z = p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(hkv, -1, p.shape[-1]), vals).view(hkv, hq // hkv, L, d) / z.clamp(min=1e-30)
        s["o"][a:a + L] = o.permute(2, 0, 1, 3).reshape(L, hq, d).bfloat16()
        s["lse"][a:a + L] = (top + torch.log(z))[..., 0].permute(2, 0, 1).reshape(L, hq)
    return [s["o"], s["lse"]]


def _plain_sample(s):
    rows, vocab = s["logits"].shape
    off, n, most = s["off"].long(), len(s["uniform"]), s["max_potential"]
    dev = off.device
    drawn = []  # [rows, most] tokens; entries past a row's draws are not used
    step = max(1, (1 << 25) // vocab)
    for a in range(0, rows, step):
        b = min(rows, a + step)
        x, order = torch.sort(s["logits"][a:b].float() + 0.0, dim=1, descending=True, stable=True)
        temp = s["temperature"][a:b, None].double()
        k = torch.where(s["top_k"][a:b, None] == 0, vocab, s["top_k"][a:b, None].long())
        k = torch.where(temp == 0, 1, k)
        w = torch.exp((x.double() - x[:, :1].double()) / torch.where(temp == 0, 1.0, temp))
        w = torch.where(torch.arange(vocab, device=dev)[None, :] < k, w, 0.0)
        mass = torch.cumsum(w, 1)
        before = torch.nn.functional.pad(mass[:, :-1], (1, 0))
        kept = (before < s["top_p"][a:b, None].double() * mass[:, -1:]) & (w >= s["min_p"][a:b, None].double())
        kept[:, 0] = True
        w = torch.zeros_like(w).scatter_(1, order, torch.where(kept, w, 0.0))
        cdf = torch.cumsum(w, 1)
        at = (off[a:b, None] + torch.arange(most, device=dev)[None, :]).clamp(max=n - 1)
        token = torch.searchsorted(cdf, s["uniform"][at].double() * cdf[:, -1:], right=True)
        last = vocab - 1 - torch.argmax((w > 0).flip(1).to(torch.uint8), 1, keepdim=True)
        drawn.append(torch.minimum(token, last))
    i = torch.arange(n, device=dev)
    row = torch.searchsorted(off[1:].contiguous(), i, right=True)
    token = torch.cat(drawn)[row, i - off[row]]
    key = torch.sort(row * vocab + token)[0]
    row, token = key // vocab, key % vocab
    new = torch.cat((key[:1] == key[:1], key[1:] != key[:-1]))
    groups = torch.zeros(rows, dtype=torch.long, device=dev).scatter_add_(0, row, new.long())
    at = off[row] + torch.cumsum(new, 0) - 1 - (torch.cumsum(groups, 0) - groups)[row]
    tok = torch.full((n,), -1, dtype=torch.int32, device=dev).scatter_(0, at, token.int())
    cnt = torch.zeros(n, dtype=torch.int32, device=dev).scatter_add_(0, at, torch.ones_like(at, dtype=torch.int32))
    return [tok, cnt, groups.int()]


# ----------------------------------------------------------------------------- what it cannot do without

def work(case):
    if case["kind"] == "append":
        dst, _ = _slots(case)
        n, written, hq, hkv, d = len(dst), int((dst >= 0).sum()), case["hq"], case["hkv"], case["d"]
        read = n * (2 * hq * d + 4 * case["rot"] + 4) + written * 4 * hkv * d + 8 * d
        return {"bytes": read + n * 2 * hq * d + written * 4 * hkv * d, "flops": 7 * d * (n * hq + written * hkv)}
    if case["kind"] == "draft":
        b = _batch(case)
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        n, words = b["mask"].shape
        drafted = int(np.unpackbits(b["mask"].view(np.uint8)).sum())
        seen = drafted + sum(int(L) * (N - int(L)) for L, N in zip(np.diff(b["q_ptr"]), b["kv_len"]))
        return {"bytes": 4 * hkv * d * sum(b["kv_len"]) + n * (hq * (4 * d + 4) + 8 * words) + 8 * len(b["kv_blocks"]),
                "flops": 4 * d * hq * seen}
    n = int(_settings(case)[4].sum())
    return {"bytes": case["rows"] * (case["vocab"] * (2 if case["bf16"] else 4) + 24) + 12 * n, "flops": 3 * case["rows"] * case["vocab"]}


# ----------------------------------------------------------------------------- the same in 64 bits

def _exact_append(s):
    n, hq, hkv, d = len(s["dst"]), s["hq"], s["k"].shape[1], s["k"].shape[3]
    x = s["qkv"].double().reshape(n, hq + 2 * hkv, d)
    half = s["cos"].shape[1]
    turn = torch.complex(s["cos"].double(), s["sin"].double())[:, None]

    def head(t, w):
        t = t / ((t ** 2).sum(-1, keepdim=True) / d + s["eps"]).sqrt() * w.double()
        z = torch.complex(t[..., :half].contiguous(), t[..., half:2 * half].contiguous()) * turn
        t[..., :half], t[..., half:2 * half] = z.real, z.imag
        return t

    q, k = head(x[:, :hq].clone(), s["wq"]), head(x[:, hq:hq + hkv].clone(), s["wk"])
    pools = []
    keep = torch.nonzero(s["dst"] >= 0)[:, 0]
    at = s["dst"][keep].long()
    for pool, new in ((s["k"], k), (s["v"], x[:, hq + hkv:])):
        out = pool.double()
        out[at // BLOCK, :, at % BLOCK] = new[keep]
        pools.append(out)
    return [q] + pools


def _exact_draft(s):
    (n, hq, d), hkv = s["q"].shape, s["k"].shape[1]
    o, lse = torch.zeros(n, hq, d, dtype=torch.float64), torch.full((n, hq), -math.inf, dtype=torch.float64)
    blocks, lens = s["kv_blocks"].cpu().tolist(), s["block_len"].cpu().tolist()
    words = s["mask"].cpu().numpy().view(np.uint64)
    o, lse = o.cuda(), lse.cuda()
    for r in range(len(s["kv_len"])):
        a, b = s["q_ptr"][r], s["q_ptr"][r + 1]
        path = [t * BLOCK + i for t in blocks[s["kv_ptr"][r]:s["kv_ptr"][r + 1]] for i in range(lens[t])]
        at = torch.tensor(path, device="cuda")
        N, L = len(path), b - a
        keys, vals = (pool[at // BLOCK, :, at % BLOCK].double() for pool in (s["k"], s["v"]))
        bits = np.unpackbits(words[a:b].view(np.uint8).reshape(L, -1), axis=1, bitorder="little")[:, :L]
        hidden = np.zeros((L, N), dtype=bool)
        hidden[:, max(0, N - L):] = bits[:, max(0, L - N):] == 0
        hidden = torch.from_numpy(hidden).cuda()
        for h in range(hq):
            g = h * hkv // hq
            x = (s["q"][a:b, h].double() @ keys[:, g].t().contiguous()) * d ** -0.5
            x = x.masked_fill(hidden, -math.inf)
            z = torch.logsumexp(x, 1)
            lse[a:b, h] = z
            p = torch.exp(x - torch.where(z == -math.inf, 0.0, z)[:, None])
            o[a:b, h] = p @ vals[:, g].contiguous()
    return [o, lse]


def exact(case, seed):
    if case["kind"] == "sample":
        return None  # tokens and counts are decisions, not computed numbers
    s = prepare(case, seed)
    return _exact_append(s) if case["kind"] == "append" else _exact_draft(s)
