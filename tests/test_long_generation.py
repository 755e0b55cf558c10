"""A long generation as a program runs it: tokens appended, attended and weighed, the next ones drawn under the rules of what was
said, and paths past their budget cut to their first, last and heaviest keys, on the block manager's tables.

Attention and weights are followed in float64 from the device's own inputs; what stays is decided by the device's weights and has to
be what a plain implementation decides from them.  Draws are compared with a plain implementation on float64 logits: a draw whose
uniform lies within 2^-18 of a boundary of the exact distribution may be either neighbour's (an adjusted logit is off by 2^-22 of
its parts, here under 32 in all, a weight then by 2^-17 of itself at most over a temperature of 1, and sums of them by as much,
of which less than half lies on one side).
"""
import numpy as np
import pytest
import torch

import paper_2609_39334_amd as tkv
from paper_2609_39334_amd.model import DecoderShape, SyntheticDecoder
from test_draft_step import _np, _path_logits, _slots
from test_evict_keys import choose

BS = 16


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,other", [(12, 2, 128, False), (4, 4, 64, True)])
def test_steps_under_a_budget(hq, hkv, d, other):
    rng = np.random.default_rng(hq)
    g = torch.Generator(device="cuda").manual_seed(hq)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
    stream = torch.cuda.Stream() if other else None
    nb, R, vocab, budget, slack, sink, recent = 600, 3, 777, 96, 20, 4, 24
    # keys and tokens under block managers of their own: a token stays said when its key is evicted
    cache, spoken = tkv.BlockManager(nb, BS, 64), tkv.BlockManager(nb, BS, 64)
    prompts = [rng.integers(0, vocab, n).tolist() for n in (40, 150, 7)]
    seqs, lines, lost = [], [], [0] * R
    k, v = rand(nb, hkv, BS, d), rand(nb, hkv, BS, d)
    said = torch.full((nb, BS), -1, dtype=torch.int32, device="cuda")
    texts = [list(p) for p in prompts]

    def speak(dst, tokens):
        said.view(-1)[torch.as_tensor(dst).long().cuda()] = torch.as_tensor(tokens, dtype=torch.int32).cuda()

    for p in prompts:
        seqs.append(cache.extend(-1, p, True)[0])
        line, blk, hit = spoken.extend(-1, p, True)
        lines.append(line)
        speak(tkv.tkv_extend_slots(blk, hit, len(p)), p)
    keys = BS * 24
    weights = torch.zeros((R, hkv, keys), device="cuda")
    rules = {"prompt_len": torch.tensor([len(p) for p in prompts], dtype=torch.int32, device="cuda"),
             "repetition": torch.tensor([1.2, 1.0, 1.1], device="cuda"), "presence": torch.tensor([0.5, 0.0, 0.0], device="cuda"),
             "frequency": torch.tensor([0.25, 0.5, 0.0], device="cuda"),
             "bias_indptr": torch.tensor([0, 2, 2, 3], dtype=torch.int32, device="cuda"),
             "bias_token": torch.tensor([5, 9, 100], dtype=torch.int32, device="cuda"),
             "bias_value": torch.tensor([2.0, -4.0, 1.0], device="cuda"),
             "allowed": torch.from_numpy(rng.integers(0, 1 << 32, (2, 25), dtype=np.uint32).view(np.int32)).cuda()}
    draws = 0
    for step in range(70):
        # some tokens each: single ones, or a short chain that was accepted whole
        new = [[int(x) for x in rng.integers(0, vocab, 1 + (step + r) % 3)] if step == 0 else [nxt[r]] + texts[r][:(step + r) % 3]
               for r in range(R)]
        dst = np.concatenate([cache.append(s, t) for s, t in zip(seqs, new)])
        speak(np.concatenate([spoken.append(s, t) for s, t in zip(lines, new)]), sum(new, []))
        for r in range(R):
            texts[r] += new[r]
        n = len(dst)
        tkv.tkv_kv_append(torch.from_numpy(dst).cuda(), rand(n, hkv, d), rand(n, hkv, d), k, v)
        tables, block_len = [cache.table(s) for s in seqs], cache.block_len()
        chains = [list(range(-1, len(t) - 1)) for t in new]
        batch = tkv.DraftBatch(tables, chains, block_len, evicted=lost)
        history = tkv.DraftBatch([spoken.table(s) for s in lines], chains, spoken.block_len())
        assert batch.positions.tolist() == history.positions.tolist()   # eviction moves no positions
        q, o, lse = rand(n, hq, d), torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((n, hq), device="cuda")
        old = weights.clone()
        torch.cuda.synchronize()
        batch.verify(q, k, v, o, lse, stream=stream)
        batch.key_weights(q, k, lse, weights, before=weights, decay=0.9, stream=stream)
        torch.cuda.synchronize()
        a = 0
        for r in range(R):
            L = len(new[r])
            s = torch.from_numpy(_slots(tables[r], block_len)).cuda()
            N = len(s)
            assert N <= keys
            at = np.concatenate([BS * e + np.arange(block_len[b]) for e, b in enumerate(tables[r])])
            x = torch.stack([k[s // BS, h * hkv // hq, s % BS].double() @ q[a:a + L, h].double().t().contiguous() for h in range(hq)]) / d ** 0.5
            i, j = torch.arange(L, device="cuda")[None], torch.arange(N, device="cuda")[:, None]
            x = x.masked_fill(j > N - L + i, -float("inf"))                         # [hq, N, L]
            p = torch.softmax(x, 1)
            for h in range(hq):
                vals = v[s // BS, h * hkv // hq, s % BS].double()
                A = p[h].t() @ vals.abs()
                ref = p[h].t() @ vals
                assert torch.all((o[a:a + L, h].double() - ref).abs() <= 2.0 ** -8 * (A + 2 * ref.abs()) + 2.0 ** -11 * A)
            for m in range(hkv):
                want = p[m * hq // hkv:(m + 1) * hq // hkv].sum((0, 2))
                # (a new key's place may hold anything)
                had = torch.where(torch.arange(N, device="cuda") < N - L, old[r, m, torch.from_numpy(at).cuda()].double() * float(np.float32(0.9)), 0.0)
                # lse is off by 2^-11 at most, and a weight by as much of itself
                assert torch.all((weights[r, m, torch.from_numpy(at).cuda()].double() - want - had).abs() <= 2.0 ** -10 * want + 2.0 ** -20 * had + 2.0 ** -30)
            a += L
        # the next tokens
        logits = torch.randn((n, vocab), generator=g, device="cuda") * 3
        grammar = rng.integers(-1, 2, n).astype(np.int32)
        u = torch.rand(n, generator=g, device="cuda")
        off, one = torch.arange(n + 1, dtype=torch.int32, device="cuda"), torch.ones(n, device="cuda")
        adjusted = history.adjust_logits(said, logits, grammar=torch.from_numpy(grammar).cuda(), stream=stream, **rules)
        torch.cuda.synchronize()
        tok, cnt, groups = tkv.tkv_filter_sample(adjusted, one, off, u, 1)
        assert torch.all(groups == 1) and torch.all(cnt == 1)
        a, nxt = 0, []
        for r in range(R):
            L = len(new[r])
            for i in range(L):
                text = np.array(texts[r][:len(texts[r]) - L + i + 1])
                y = logits[a + i].double().cpu().numpy()
                rep, pres, freq = (float(rules[x][r]) for x in ("repetition", "presence", "frequency"))
                seen = np.isin(np.arange(vocab), text)
                c = np.bincount(text[len(prompts[r]):], minlength=vocab)
                y = np.where(seen, np.where(y > 0, y / rep, y * rep), y) - freq * c - pres * (c > 0)
                y += {0: 2.0 * (np.arange(vocab) == 5) - 4.0 * (np.arange(vocab) == 9), 1: 0.0, 2: 1.0 * (np.arange(vocab) == 100)}[r]
                if grammar[a + i] >= 0:
                    bits = rules["allowed"][int(grammar[a + i])].cpu().numpy().view(np.uint32)
                    y[(bits[np.arange(vocab) // 32] >> (np.arange(vocab) % 32)) & 1 == 0] = -np.inf
                w = np.exp(y - y.max())
                cdf = np.cumsum(w) / w.sum()
                t, z = int(tok[a + i]), float(u[a + i])
                assert (cdf[t - 1] if t else 0.0) - 2.0 ** -18 <= z <= cdf[t] + 2.0 ** -18 and w[t] > 0
                draws += 1
            nxt.append(int(tok[a + L - 1]))
            a += L
        # paths past the budget and its slack
        if max(cache.block_len()[cache.table(s)].sum() for s in seqs) > budget + slack:
            full, lens = [cache.table(s) for s in seqs], [int(cache.block_len()[cache.table(s)].sum()) for s in seqs]
            shorter = [cache.extend(-1, [0] * min(m, budget), False)[0] for m in lens]
            e = tkv.EvictBatch(full, [cache.table(s) for s in shorter], [budget] * R, cache.block_len())
            was_k, was_v, w = k.clone(), v.clone(), weights.clone()
            torch.cuda.synchronize()
            weights, kept, n_kept = e.evict(weights, k, v, sink, recent, stream=stream)
            torch.cuda.synchronize()
            assert n_kept.tolist() == e.n_kept == [min(m, budget) for m in lens]
            for r in range(R):
                at = np.concatenate([BS * i + np.arange(e.block_len.cpu().numpy()[b]) for i, b in enumerate(full[r])])
                src, to = (torch.from_numpy(x).cuda() for x in (_slots(full[r], cache.block_len()), _slots(cache.table(shorter[r]), cache.block_len())))
                for h in range(hkv):
                    pick = choose(w[r, h].cpu().numpy()[at], budget, sink, recent)
                    assert kept[r, h, :len(pick)].tolist() == at[pick].tolist() and torch.all(kept[r, h, len(pick):] == -1)
                    f = src[torch.from_numpy(pick).cuda()]
                    assert torch.equal(k[to // BS, h, to % BS], was_k[f // BS, h, f % BS])
                    assert torch.equal(v[to // BS, h, to % BS], was_v[f // BS, h, f % BS])
                    assert torch.equal(weights[r, h, :len(pick)], w[r, h, torch.from_numpy(at[pick]).cuda()])
                lost[r] += e.evicted[r]
                cache.prune(seqs[r])
            seqs = shorter
    assert draws > 100 and min(lost) > 0


@pytest.mark.gpu
def test_the_model_after_an_eviction():
    # one KV head, so that a row's heads keep the same keys and the float64 model can walk them; positions go on as before
    shape = DecoderShape(layers=2, hidden=256, hq=4, hkv=1, d=64, inter=512, vocab=500, qk_norm=True)
    model, other = SyntheticDecoder(shape, seed=9), torch.cuda.Stream()
    nb, rng = 64, np.random.default_rng(2)
    bm = tkv.BlockManager(nb, BS, 16)
    g = torch.Generator(device="cuda").manual_seed(3)
    pools = [[torch.randn((nb, 1, BS, 64), generator=g, device="cuda").bfloat16() for _ in range(2)] for _ in "kv"]
    seqs = [bm.extend(-1, rng.integers(0, 500, n).tolist(), True)[0] for n in (130, 21)]
    drafts = [rng.integers(0, 500, n).tolist() for n in (5, 3)]
    weights = [torch.zeros((2, 1, BS * 12), device="cuda") for _ in range(2)]

    def verify(seqs, lost, weights):
        kids, dst = [], []
        for s, t in zip(seqs, drafts):
            dst.append(bm.append(s, t))
        batch = tkv.DraftBatch([bm.table(s) for s in seqs], [list(range(-1, len(t) - 1)) for t in drafts], bm.block_len(), evicted=lost)
        for stream in (None, other):
            w = [x.clone() for x in weights]
            got = model.verify_draft(torch.tensor(sum(drafts, []), device="cuda"), torch.from_numpy(np.concatenate(dst)).cuda(), batch,
                                     *pools, weights=w, stream=stream)
        return _np(got), w, batch

    _, weights, _ = verify(seqs, None, weights)
    for w in weights:  # a query's weights add up to 1 for each of the four heads (lse is off by 2^-11 at most)
        assert abs(float(w[0].sum()) - 5 * 4) <= 2.0 ** -9 * 20 and abs(float(w[1].sum()) - 3 * 4) <= 2.0 ** -9 * 12
    new = [bm.extend(-1, [0] * m, False)[0] for m in (40, 24)]
    e = tkv.EvictBatch([bm.table(s) for s in seqs], [bm.table(s) for s in new], [40, 100], bm.block_len())
    assert e.evicted == [95, 0] and e.n_kept == [40, 24]
    before = [float(w.sum()) for w in weights]
    for stream in (other, None):
        short = model.evict(e, weights, *pools, sink=2, recent=8, stream=stream)
    assert all(0 < float(s.sum()) < b for s, b in zip(short, before))
    for args in ((e, weights[:1], *pools), (e, weights, pools[0][:1], pools[1]), (e, weights + weights, *pools)):
        with pytest.raises(ValueError):
            model.evict(*args)
    with pytest.raises(ValueError):
        verify(seqs, None, weights[:1])
    kp, vp = ([_np(p) for p in ps] for ps in pools)
    ctx = [_slots(bm.table(s), bm.block_len()) for s in new]
    got, _, batch = verify(new, e.evicted, short)
    assert batch.positions.tolist() == list(range(135, 140)) + list(range(24, 27))
    want = np.concatenate([_path_logits(model, t, start, kp, vp, c) for t, start, c in zip(drafts, (135, 24), ctx)])
    err = np.abs(got - want)
    assert err.max() <= 2e-2 * np.abs(want).max() and err.mean() <= 1e-2 * np.abs(want).mean()


@pytest.mark.gpu
def test_draws_under_rules_on_another_stream():
    model = SyntheticDecoder(DecoderShape(layers=1, hidden=64, hq=1, hkv=1, d=64, inter=64, vocab=64))
    g = torch.Generator(device="cuda").manual_seed(2)
    n, vocab = 60, 30000
    new = torch.randn((n, vocab), generator=g, device="cuda").bfloat16()
    logits = torch.zeros_like(new)
    said = torch.randint(0, vocab, (n, BS), generator=g, device="cuda", dtype=torch.int32)
    history = tkv.DraftBatch([[r] for r in range(n)], [[-1]] * n, np.full(n, 16, np.int32))
    rules = {"repetition": torch.full((n,), 1.5, device="cuda"), "frequency": torch.full((n,), 0.5, device="cuda")}
    T, off, u = torch.ones(n, device="cuda"), torch.arange(n + 1, dtype=torch.int32, device="cuda"), torch.rand(n, generator=g, device="cuda")
    out = torch.empty((n, vocab), device="cuda")
    want = [t.clone() for t in tkv.tkv_filter_sample(history.adjust_logits(said, new, out=out, **rules), T, off, u, 1)]
    for stream in (torch.cuda.Stream(), torch.cuda.Stream().cuda_stream, 0, None):
        logits.zero_()
        torch.cuda.synchronize()
        torch.cuda._sleep(100_000_000)
        logits.copy_(new)
        got = model.sample_filtered(logits, T, off, u, 1, stream=stream, history=history, said=said, rules=rules)
        got = [t.clone() for t in got]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_numbers_past_32_bits_are_refused():
    dev = lambda *x, dtype=torch.int32: torch.tensor(x, dtype=dtype, device="cuda")
    rows = dict(kv_indptr=dev(0, 2), kv_blocks=dev(0, 1), block_len=dev(16, 4, 0), max_blocks=2)
    k, w = torch.zeros((3, 2, BS, 64), device="cuda").bfloat16(), torch.zeros((1, 2, 32), device="cuda")
    batch = dict(rows, q_indptr=dev(0, 1), mask=dev(1, dtype=torch.int64)[None], max_q=1)
    weigh = dict(batch, q=torch.zeros((1, 2, 64), device="cuda").bfloat16(), k=k, lse=torch.zeros((1, 2), device="cuda"), out=w)
    evict = dict(rows, new_indptr=dev(0, 1), new_blocks=dev(2), budget=dev(4), sink=1, recent=1, weights=w, k=k, v=k.clone(),
                 out=w.clone(), kept=torch.zeros((1, 2, 4), dtype=torch.int32, device="cuda"), n_kept=dev(0))
    adjust = dict(batch, tokens=torch.zeros((3, BS), dtype=torch.int32, device="cuda"), logits=torch.zeros((1, 100), device="cuda"))
    for call, args, names in ((tkv.tkv_key_weights, weigh, ("max_q", "max_blocks")),
                              (tkv.tkv_evict_keys, evict, ("max_blocks", "sink", "recent")),
                              (tkv.tkv_adjust_logits, adjust, ("max_q", "max_blocks"))):
        call(**args)
        for name in names:
            for bad in (1 << 31, -(1 << 31) - 1, (1 << 32) + 2):
                with pytest.raises(ValueError, match="32 bits"):
                    call(**dict(args, **{name: bad}))
    wide = torch.empty((1, (1 << 32) + 100), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="32 bits"):
        tkv.tkv_adjust_logits(**dict(adjust, logits=wide, out=wide))


def test_rules_and_histories_go_together():
    # no draw from logits that silently miss their rules (refused before any device access: no GPU needed)
    model = SyntheticDecoder(DecoderShape(layers=1, hidden=64, hq=1, hkv=1, d=64, inter=64, vocab=64), device="cpu")
    history = tkv.DraftBatch([[0]], [[-1]], np.full(1, 16, np.int32), device="cpu")
    said, rules = torch.zeros((1, BS), dtype=torch.int32), {"repetition": torch.full((1,), 1.5)}
    logits, one, off = torch.zeros((1, 64)), torch.ones(1), torch.tensor([0, 1], dtype=torch.int32)
    for some in (dict(rules=rules), dict(said=said), dict(rules=rules, said=said), dict(history=history),
                 dict(history=history, rules=rules)):
        with pytest.raises(ValueError, match="go together"):
            model.sample_filtered(logits, one, off, one * 0.5, 1, **some)


def test_evict_batch():
    bl = np.array([16, 16, 5, 3, 0, 0, 0], np.int32)
    e = tkv.EvictBatch([[0, 3], [1, 2], []], [[4], [5, 6], []], [10, 1 << 40, 0], bl, device="cpu")  # (a budget of any size)
    assert e.n_kept == [10, 21, 0] and e.evicted == [9, 0, 0] and (e.max_blocks, e.most) == (2, 21)
    assert e.kv_indptr.tolist() == [0, 2, 4, 4] and e.new_indptr.tolist() == [0, 1, 3, 3] and e.budget.tolist() == [10, 21, 0]
    assert e.kv_blocks.tolist() == [0, 3, 1, 2] and e.new_blocks.tolist() == [4, 5, 6] and e.block_len.tolist() == bl.tolist()
    none = tkv.EvictBatch([], [], [], bl, device="cpu")
    assert none.kv_indptr.tolist() == [0] and none.n_kept == [] and none.max_blocks == 1
    for old, new, budget in (([[0]], [], [1]), ([[0]], [[4]], []), ([[0]], [[4]], [-1]), ([[7]], [[4]], [1]), ([[0]], [[-1]], [1]),
                             ([[0, 1]], [[4]], [20]), ([[0]], [[]], [1]),                      # too few blocks
                             ([[0]], [[0]], [1]), ([[0], [1]], [[1], [4]], [1, 1]),            # a block that a path holds
                             ([[0], [1]], [[4], [4]], [1, 1]), ([[0, 1]], [[4, 4]], [20])):    # or that is named twice
        with pytest.raises(ValueError):
            tkv.EvictBatch(old, new, budget, bl, device="cpu")
    for bad in (17, -1):
        with pytest.raises(ValueError, match="length"):
            tkv.EvictBatch([[0, 1]], [[2]], [4], np.array([16, bad, 3], np.int32), device="cpu")


def test_draft_batch_of_evicted_paths():
    bl = np.array([16, 16, 5, 3], np.int32)
    b = tkv.DraftBatch([[0, 3], [1, 2]], [[-1, 0], [-1]], bl, device="cpu", evicted=[100, 0])
    assert b.positions.tolist() == [117, 118, 20]
    for bad in ([1], [1, -1]):
        with pytest.raises(ValueError):
            tkv.DraftBatch([[0, 3], [1, 2]], [[-1, 0], [-1]], bl, device="cpu", evicted=bad)
