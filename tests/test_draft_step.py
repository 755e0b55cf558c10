"""A drafting decode step as a search runs it: drafted trees appended to the paged cache (norm, rotation, append), verified
in one pass over the cache, the next tokens drawn from truncated distributions, the drafts walked and the accepted
tokens kept.

The forward pass is compared with the same model in float64 on the host, one drafted path at a time, with bf16 rounding where
the device rounds (GEMM outputs, rotated heads, attention and norm outputs).  What remains is fp32 against float64
accumulation: values near a bf16 rounding boundary land one ulp (2^-7 of the value, at most) away, and such flips propagate.
As for the plain decode step the bars are 2% of the largest logit for the largest difference and 1% of the mean magnitude
for the mean.  Draws are compared with a plain implementation on the device's own logits, and are equal.
"""
import numpy as np
import pytest
import torch

import paper_2609_39334_amd as tkv
from paper_2609_39334_amd.model import DecoderShape, SyntheticDecoder

BS = 16


def _bf(x):
    return torch.from_numpy(np.asarray(x, np.float32)).bfloat16().double().numpy()


def _np(t):
    return t.double().cpu().numpy()


def _path_logits(model, tokens, start, k_pools, v_pools, ctx):
    """Logits after each of `tokens`, which follow the context at pool slots ctx (positions 0 .. len(ctx) - 1)."""
    s = model.shape
    half, T = s.d // 2, len(tokens)
    pos = start + np.arange(T)
    ang = pos[:, None] * s.rope_theta ** (-np.arange(half) * 2.0 / s.d)
    cos, sin = np.cos(ang)[:, None], np.sin(ang)[:, None]

    def rms(x, w):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + s.eps) * _np(w)

    def rope(t):
        a, b = t[..., :half], t[..., half:]
        return _bf(np.concatenate((a * cos - b * sin, b * cos + a * sin), -1))

    x = _np(model.embed)[np.asarray(tokens)]
    for li, w in enumerate(model.layers):
        qkv = _bf(_bf(rms(x, w["ln1"])) @ _np(w["wqkv"])).reshape(T, -1, s.d)
        q, k, v = qkv[:, :s.hq], qkv[:, s.hq:s.hq + s.hkv], qkv[:, s.hq + s.hkv:]
        if s.qk_norm:
            q, k = rms(q, w["qn"]), rms(k, w["kn"])
        q, k = rope(q), rope(k)
        keys = np.concatenate((k_pools[li][ctx // BS, :, ctx % BS], k))
        vals = np.concatenate((v_pools[li][ctx // BS, :, ctx % BS], v))
        o = np.zeros((T, s.hq, s.d))
        for h in range(s.hq):
            g = h * s.hkv // s.hq
            sc = q[:, h] @ keys[:, g].T / np.sqrt(s.d)
            sc[np.arange(len(keys))[None] > len(ctx) + np.arange(T)[:, None]] = -np.inf
            p = np.exp(sc - sc.max(-1, keepdims=True))
            o[:, h] = (p / p.sum(-1, keepdims=True)) @ vals[:, g]
        x = x + _bf(_bf(o).reshape(T, -1) @ _np(w["wo"]))
        gu = _bf(_bf(rms(x, w["ln2"])) @ _np(w["wgu"]))
        x = x + _bf(_bf(gu[:, :s.inter] / (1 + np.exp(-gu[:, :s.inter])) * gu[:, s.inter:]) @ _np(w["wd"]))
    return _bf(_bf(rms(x, model.lnf)) @ _np(model.lm))


def _slots(table, block_len):
    return np.concatenate([np.arange(block_len[b]) + b * BS for b in table]).astype(np.int64)


def _plain_draw(x, T, k, p, u):
    order = np.argsort(-x, kind="stable")
    w = np.exp((x[order] - x[order[0]]) / float(np.float32(T)))
    w[k:] = 0
    before = np.concatenate(([0.0], np.cumsum(w)[:-1]))
    w[1:][before[1:] >= float(np.float32(p)) * w.sum()] = 0
    full = np.zeros(len(w))
    full[order] = w
    cdf = np.cumsum(full)
    return int(np.searchsorted(cdf, float(u) * cdf[-1], side="right"))


@pytest.mark.gpu
@pytest.mark.parametrize("qk_norm,hq,hkv,d,other", [(True, 8, 2, 128, False), (False, 4, 4, 64, True), (True, 6, 2, 64, True)])
def test_drafted_steps(qk_norm, hq, hkv, d, other):
    rng = np.random.default_rng(hq)
    shape = DecoderShape(layers=2, hidden=256, hq=hq, hkv=hkv, d=d, inter=512, vocab=500, qk_norm=qk_norm)
    model = SyntheticDecoder(shape, seed=hq)
    nb = 160
    bm = tkv.BlockManager(nb, BS, 64)
    root = bm.extend(-1, rng.integers(0, 500, 45).tolist(), True)[0]
    seqs = [bm.extend(root, rng.integers(0, 500, int(n)).tolist(), True)[0] for n in (3, 40, 17)]
    g = torch.Generator(device="cuda").manual_seed(1)
    pools = [[torch.randn((nb, hkv, BS, d), generator=g, device="cuda").bfloat16() for _ in range(2)] for _ in "kv"]
    stream = torch.cuda.Stream() if other else None
    for step in range(2):
        # a tree of drafted tokens under every sequence, in blocks of its own
        parents = [[-1] + [int(rng.integers(max(-1, i - 4), i)) for i in range(1, L)] for L in ((1, 9, 20), (21, 2, 5))[step]]
        drafts = [rng.integers(0, 500, len(p)).tolist() for p in parents]
        kids, dst = [], []
        for q, t in zip(seqs, drafts):
            kid, blk, hit = bm.extend(q, t, False)
            kids.append(kid)
            dst.append(tkv.tkv_extend_slots(blk, hit, len(t)))
        tables, block_len = [bm.table(k) for k in kids], bm.block_len()
        batch = tkv.DraftBatch(tables, parents, block_len)
        for pool in pools[0] + pools[1]:               # the step writes these
            at = torch.from_numpy(np.concatenate(dst)).long().cuda()
            pool[at // BS, :, at % BS] = float("nan")
        tokens = torch.tensor(sum(drafts, []), device="cuda")
        logits = model.verify_draft(tokens, torch.from_numpy(np.concatenate(dst)).cuda(), batch, *pools, stream=stream)
        torch.cuda.synchronize()
        got = _np(logits)
        kp, vp = ([_np(p) for p in ps] for ps in pools)
        want = np.zeros_like(got)
        a = 0
        for r, par in enumerate(parents):
            ctx = _slots(bm.table(seqs[r]), block_len)
            for i in range(len(par)):
                path = [i]
                while par[path[0]] >= 0:
                    path.insert(0, par[path[0]])
                want[a + i] = _path_logits(model, [drafts[r][j] for j in path], len(ctx), kp, vp, ctx)[-1]
                assert batch.depth[a + i] == len(path) - 1
            a += len(par)
        err = np.abs(got - want)
        print(f"    step {step}: {a} drafted tokens, max {err.max():.3e} (|ref| max {np.abs(want).max():.2f}), mean {err.mean():.3e}", flush=True)
        assert np.isfinite(got).all()
        assert err.max() <= 2e-2 * np.abs(want).max() and err.mean() <= 1e-2 * np.abs(want).mean()
        # the next token after every drafted one, from its truncated distribution
        n = len(got)
        T, k, p = np.full(n, 0.8, np.float32), rng.choice([5, 20], n).astype(np.int32), rng.choice([0.5, 0.95], n).astype(np.float32)
        u = rng.random(n, dtype=np.float32)
        dev = lambda x: torch.from_numpy(x).cuda()
        tok, cnt, ng = model.sample_filtered(logits, dev(T), dev(np.arange(n + 1, dtype=np.int32)), dev(u), 1, dev(k), dev(p), stream=stream)
        torch.cuda.synchronize()
        tok = tok.tolist()
        assert ng.tolist() == [1] * n and cnt.tolist() == [1] * n
        assert tok == [_plain_draw(got[i], T[i], int(k[i]), p[i], u[i]) for i in range(n)]
        # walk each tree: drafted children that agree are accepted (one is made to, so that something is)
        a = 0
        for r, par in enumerate(parents):
            L = len(par)
            node, accepted = 0, [0]
            while True:
                nxt = [j for j in range(L) if par[j] == node and (drafts[r][j] == tok[a + node] or len(accepted) < 3)]
                if not nxt:
                    break
                node = nxt[0]
                accepted.append(node)
            new = [drafts[r][j] for j in accepted] + [tok[a + node]]
            dst_new = bm.append(seqs[r], new)
            src = torch.from_numpy(dst[r][accepted]).long().cuda()
            to = torch.from_numpy(dst_new[:-1]).cuda()
            for kpool, vpool in zip(*pools):
                rows = [pool[src // BS, :, src % BS].contiguous() for pool in (kpool, vpool)]
                tkv.tkv_kv_append(to, *rows, kpool, vpool)
                # the last token's K and V come with the next step; here any values do
                end = int(dst_new[-1])
                for pool in (kpool, vpool):
                    pool[end // BS, :, end % BS] = torch.randn((hkv, d), generator=g, device="cuda").bfloat16()
            bm.prune(kids[r])
            bm.seal(seqs[r])
            a += L


@pytest.mark.gpu
def test_a_chain_draft_is_the_decode_step():
    # one drafted token a row: the logits of step() on a plan of the same tables, up to the order of fp32 sums
    shape = DecoderShape(layers=2, hidden=256, hq=4, hkv=2, d=64, inter=512, vocab=1000, qk_norm=True)
    model = SyntheticDecoder(shape, seed=4)
    nb, rows = 64, 5
    tables = [np.r_[0:4, 4 + 2 * r:6 + 2 * r].astype(np.int32) for r in range(rows)]
    block_len = np.full(nb, 16, np.int32)
    g = torch.Generator(device="cuda").manual_seed(5)
    pools = [[torch.randn((nb, 2, 16, 64), generator=g, device="cuda").bfloat16() for _ in range(2)] for _ in "kv"]
    tokens = torch.randint(0, 1000, (rows,), generator=g, device="cuda")
    dst = torch.tensor([16 * (6 + 2 * r) - 1 for r in range(rows)], dtype=torch.int32, device="cuda")
    ptr = np.arange(rows + 1, dtype=np.int32)
    plan = tkv.Plan((4, 2, 64, 16, nb), ptr, 6 * ptr, np.concatenate(tables), block_len)
    want = model.step(tokens, torch.full((rows,), 95, device="cuda"), dst, plan, *pools)
    batch = tkv.DraftBatch(tables, [[-1]] * rows, block_len)
    assert batch.positions.tolist() == [95] * rows
    got = model.verify_draft(tokens, dst, batch, *pools).float()
    err = (got - want).abs()
    assert err.max() <= 2e-2 * want.abs().max() and err.mean() <= 1e-2 * want.abs().mean()


@pytest.mark.gpu
def test_draws_on_another_stream_follow_the_logits_and_come_before_their_use():
    model = SyntheticDecoder(DecoderShape(layers=1, hidden=64, hq=1, hkv=1, d=64, inter=64, vocab=64))
    g = torch.Generator(device="cuda").manual_seed(2)
    n, vocab = 200, 30000
    new = torch.randn((n, vocab), generator=g, device="cuda") * 3
    logits = torch.zeros_like(new)
    T, off, u = torch.ones(n, device="cuda"), torch.arange(n + 1, dtype=torch.int32, device="cuda"), torch.rand(n, generator=g, device="cuda")
    p = torch.full((n,), 0.9, device="cuda")
    want = [t.clone() for t in model.sample_filtered(new, T, off, u, 1, top_p=p)]
    for stream in (torch.cuda.Stream(), torch.cuda.Stream().cuda_stream, 0, None):
        logits.zero_()
        torch.cuda.synchronize()
        torch.cuda._sleep(100_000_000)
        logits.copy_(new)                              # the draws read these
        got = model.sample_filtered(logits, T, off, u, 1, top_p=p, stream=stream)
        got = [t.clone() for t in got]                 # and are complete for the current stream
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_draft_batch_of_bad_lengths():
    # a length outside [0, 16] would count for the positions and not for the attention
    for bad in (17, -1):
        with pytest.raises(ValueError, match="length"):
            tkv.DraftBatch([[0, 1]], [[-1]], np.array([16, bad, 3], np.int32), device="cpu")
    b = tkv.DraftBatch([[0, 2]], [[-1]], np.array([16, 17, 3], np.int32), device="cpu")    # not in a table
    assert b.positions.tolist() == [18]


def test_draft_batch():
    bl = np.array([16, 16, 5, 3, 0], np.int32)
    b = tkv.DraftBatch([[0, 3], [1, 2]], [[-1, 0, 0], [-1, 0, 1, -1]], bl, device="cpu")
    assert b.q_indptr.tolist() == [0, 3, 7] and b.kv_indptr.tolist() == [0, 2, 4] and b.kv_blocks.tolist() == [0, 3, 1, 2]
    assert b.positions.tolist() == [16, 17, 17, 17, 18, 19, 17] and b.depth.tolist() == [0, 1, 1, 0, 1, 2, 0]
    assert b.mask.tolist() == [[1], [3], [5], [1], [3], [7], [8]] and b.block_len.tolist() == bl.tolist()
    assert (b.max_q, b.max_blocks) == (4, 2)
    long = tkv.DraftBatch([[0, 1], [0, 1, 2]], [[-1], list(range(-1, 30))], bl, device="cpu")
    assert long.mask.shape == (32, 1) and long.positions[-1] == 36
    none = tkv.DraftBatch([], [], bl, device="cpu")
    assert none.q_indptr.tolist() == [0] and none.mask.shape[0] == 0
    for tables, parents in (([[0]], []), ([[0]], [[]]), ([[9]], [[-1]]), ([[-1]], [[-1]]), ([[3]], [[-1, 0, 0, 0]])):
        with pytest.raises(ValueError):
            tkv.DraftBatch(tables, parents, bl, device="cpu")
    with pytest.raises(tkv.TkvError):
        tkv.DraftBatch([[0]], [[0]], bl, device="cpu")
