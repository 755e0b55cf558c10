"""Truncated sampling against a plain float64 implementation: tokens and counts are equal.

Both sides compare sums of the same 64-bit weights, which differ by their order of addition and the last digits of exp:
below 1e-11 of the total for these sizes, and the histogram's units (2^-43 of the largest weight a token) below 1e-7.  A
draw or an end of top-p that lies closer than that to a border may fall to either side; the plain implementation
reports such rows, of which the fixed seeds here hold none in the first and hardly any in the second sense.
"""
import numpy as np
import pytest
import torch

import paper_2609_39334_amd as tkv


def _plain(x, T, k, p, m, us):
    """(tokens ascending, counts) of one row."""
    x = np.asarray(x, dtype=np.float64) + 0.0
    order = np.argsort(-x, kind="stable")
    if T == 0:
        T, k = 1.0, 1
    T, p, m = (float(np.float32(v)) for v in (T, p, m))
    with np.errstate(over="ignore"):
        w = np.exp((x[order] - x[order[0]]) / T)
    if 0 < k < len(w):
        w[k:] = 0
    if p < 1:
        before = np.concatenate(([0.0], np.cumsum(w)[:-1]))
        w[1:][before[1:] >= p * w.sum()] = 0
    w[1:][w[1:] < m] = 0
    full = np.zeros(len(w))
    full[order] = w
    cdf = np.cumsum(full)
    last = int(np.flatnonzero(full)[-1])
    t = [min(int(np.searchsorted(cdf, float(u) * cdf[-1], side="right")), last) for u in us]
    return np.unique(t, return_counts=True)


def _run(x, T, k, p, m, potential, seed=0, us=None, **other):
    rng = np.random.default_rng(seed)
    off = np.concatenate([[0], np.cumsum(potential)]).astype(np.int32)
    us = rng.random(int(off[-1]), dtype=np.float32) if us is None else np.asarray(us, np.float32)
    dev = lambda a, t: None if a is None else torch.from_numpy(np.asarray(a, t)).cuda()
    tok, cnt, ng = tkv.tkv_filter_sample(x, dev(T, np.float32), dev(off, np.int32), dev(us, np.float32), int(max(potential)),
                                         dev(k, np.int32), dev(p, np.float32), dev(m, np.float32), **other)
    torch.cuda.synchronize()
    return off, us, tok.cpu().numpy(), cnt.cpu().numpy(), ng.cpu().numpy()


def _check(x, T, k, p, m, potential, seed=0, us=None, **other):
    off, us, tok, cnt, ng = _run(x, T, k, p, m, potential, seed, us, **other)
    host = x.float().cpu().numpy()
    n = len(host)
    k, p, m = (np.full(n, d) if a is None else a for a, d in ((k, 0), (p, 1.0), (m, 0.0)))
    for r in range(n):
        a, b = off[r], off[r + 1]
        if a == b:
            assert ng[r] == 0
            continue
        t, c = _plain(host[r], T[r], int(k[r]), p[r], m[r], us[a:b])
        got = (tok[a:a + ng[r]].tolist(), cnt[a:a + ng[r]].tolist())
        assert got == (t.tolist(), c.tolist()), (r, T[r], k[r], p[r], m[r])
        assert np.all(tok[a + ng[r]:b] == -1) and np.all(cnt[a + ng[r]:b] == 0)


def _logits(kind, rows, vocab, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda: torch.randn((rows, vocab), generator=g, device="cuda")
    if kind == "flat":
        x = rand() * 0.1
    elif kind == "wide":
        x = rand() * 9
    elif kind == "peaked":
        rank = torch.argsort(torch.rand((rows, vocab), generator=g, device="cuda"), 1)
        x = 12 - 1.7 * torch.log1p(rank.float()) + 0.2 * rand()
    elif kind == "steps":                             # many equal logits
        x = torch.round(rand() * 2) / 2
    elif kind == "equal":
        x = torch.full((rows, vocab), -3.0, device="cuda")
    elif kind == "masked":                            # most tokens masked, some with the type's lowest value
        x = rand() * 3
        hide = torch.rand((rows, vocab), generator=g, device="cuda")
        x[hide < 0.6] = float("-inf")
        x[hide > 0.9] = torch.finfo(dtype).min
        x[:, vocab // 2] = 1.0
    else:
        x = rand() * 2
    return x.to(dtype)


KINDS = ["normal", "flat", "wide", "peaked", "steps", "equal", "masked"]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [1, 2, 37, 1000, 4099, 32003, 151936])
def test_every_setting(vocab, kind, dtype):
    rng = np.random.default_rng(vocab)
    n = 48 if vocab < 100000 else 24
    T = rng.choice([0.0, 0.3, 0.8, 1.0, 1.7], size=n)
    k = rng.choice([0, 0, 1, 2, 20, 50, 300, 3000, 20000, vocab, vocab + 5], size=n)
    p = rng.choice([1.0, 1.0, 0.999, 0.95, 0.9, 0.5, 0.1, 0.0], size=n)
    m = rng.choice([0.0, 0.0, 0.0, 0.01, 0.1, 0.5, 1.0], size=n)
    potential = rng.choice([0, 1, 1, 2, 5, 70], size=n)
    potential[0] = 3
    _check(_logits(kind, n, vocab, dtype, seed=vocab), T, k, p, m, potential, seed=vocab)


@pytest.mark.gpu
@pytest.mark.parametrize("vocab,rows", [(32000, 300), (600, 2000), (151936, 280)])
def test_one_setting_for_many_rows(vocab, rows):
    for kind, k, p, m in (("peaked", 20, 0.95, None), ("normal", 50, None, None), ("peaked", None, 0.9, None), ("peaked", None, None, 0.05),
                          ("normal", None, None, None)):
        x = _logits(kind, rows, vocab, torch.float32, seed=rows)
        some = slice(0, rows, 7 if vocab < 100000 else 20)
        full = lambda v: None if v is None else np.full(rows, v)
        off, us, tok, cnt, ng = _run(x, np.full(rows, 0.8), full(k), full(p), full(m), [2] * rows)
        host = x.cpu().numpy()
        for r in range(rows)[some]:
            t, c = _plain(host[r], 0.8, k or 0, 1.0 if p is None else p, m or 0.0, us[2 * r:2 * r + 2])
            assert tok[2 * r:2 * r + ng[r]].tolist() == t.tolist() and cnt[2 * r:2 * r + ng[r]].tolist() == c.tolist(), (r, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_go_to_the_lowest_index(dtype):
    # equal weights: top-k and top-p keep the first ones, every cut is exact
    n = 600
    x = torch.zeros((6, n), device="cuda", dtype=dtype)
    x[1::2] = -0.0
    x[2, ::2] = -0.0                                   # -0 equals 0
    us = np.tile((np.arange(8) / 8).astype(np.float32), 6)
    k, p = [100, 0, 200, 0, 600, 7], [1.0, 0.5, 0.25, 0.125, 1.0, 0.0]
    off, _, tok, cnt, ng = _run(x, [1.0] * 6, k, p, [0.0] * 6, [8] * 6, us=us)
    for r, kept in enumerate((100, 300, 50, 75, 600, 1)):
        want = np.unique((np.arange(8) * kept) // 8)
        assert tok[off[r]:off[r] + ng[r]].tolist() == want.tolist(), r
    # a cut inside a run of equal logits below others
    x = torch.zeros((1, n), device="cuda", dtype=dtype)
    x[0, 590], x[0, 7] = 1.0, 2.0
    off, _, tok, cnt, ng = _run(x, [1.0], [12], None, None, [1000], us=np.linspace(0, 0.999, 1000))
    assert tok[:ng[0]].tolist() == list(range(0, 11)) + [590]


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [33, 32003])
def test_slices_and_alignments(vocab):
    for dtype in (torch.float32, torch.bfloat16):
        wide = _logits("normal", 9, vocab + 11, dtype)
        for first in (0, 1, 3, 8, 11):
            x = wide[:, first:first + vocab]
            _check(x, [0.8] * 9, [0, 5, 0, 0, 30, 0, 0, 0, 9], [1, 1, .9, .5, .9, 1, .99, 1, 1], [0] * 7 + [.2, .3], [3] * 9)
        one = wide[4:5, :vocab]
        _check(one, [0.8], [40], [.9], [0.], [50])


@pytest.mark.gpu
def test_most_draws_and_largest_vocabulary():
    vocab = 1 << 21
    x = _logits("normal", 4, vocab, torch.float32)
    x[3, vocab - 1] = 40.0
    _check(x, [0.8, 0.8, 1.0, 1.0], [0, 40, 0, 0], [1.0, 1.0, .7, 1.0], [0.0, 0.0, 0.0, .5], [1024, 1024, 9, 1])


@pytest.mark.gpu
def test_uniforms_at_the_ends():
    # u = 0 is the first kept token, u = 1 (outside the documented range) and the largest below it the last
    x = _logits("normal", 3, 5000, torch.float32)
    x[:, :10], x[:, -10:] = float("-inf"), float("-inf")
    us = [0.0, 1.0, float(np.nextafter(np.float32(1), np.float32(0)))] * 3
    _check(x, [0.8] * 3, [0, 30, 0], [1.0, 1.0, .8], [0.0] * 3, [3] * 3, us=us)


@pytest.mark.gpu
def test_a_uniform_of_zero_and_weights_that_round_to_zero():
    # the first tile's weights are below the smallest 64-bit number each (e^-746), though not as a sum
    for vocab, m in ((9000, None), (100000, None), (100000, 1e-30)):
        x = torch.zeros((2, vocab), device="cuda")
        x[:, :2048] = -746.0
        x[:, 0] = float("-inf")
        x[:, 2048:2050] = torch.tensor([-746.0, -100.0], device="cuda")
        _check(x, [1.0, 1.0], None, None, None if m is None else [m, m], [1, 2], us=[0.0, 0.0, 0.5])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_low_draws_among_tiny_weights_under_a_large_top_k(dtype):
    # logits fall by 0.05 a rank: of 1,000 kept tokens the last 293 weigh less than 2^-51, and no other kept token lies
    # in the first 2,048, where a uniform of 0 and the smallest ones draw
    rng = np.random.default_rng(7)
    vocab, rows = 32003, 4
    x = np.empty((rows, vocab), np.float32)
    for r in range(rows):
        rank = rng.permutation(vocab)
        tiny = np.flatnonzero((rank >= 720) & (rank < 1000))[:200]
        front = rng.permutation(2048)
        others = np.flatnonzero(rank[:2048] < 2500)               # these ranks leave the front
        away = 2048 + np.flatnonzero(rank[2048:] >= 2500)[:len(others)]
        rank[others], rank[away] = rank[away].copy(), rank[others].copy()
        tiny = np.flatnonzero((rank >= 720) & (rank < 1000))[:200]
        rank[front[:200]], rank[tiny] = rank[tiny].copy(), rank[front[:200]].copy()
        assert rank[:2048].min() >= 720 and np.sum(rank[:2048] < 1000) == 200
        x[r] = -0.05 * rank
    us = [0.0, 2.0 ** -149, 2.0 ** -100, 2.0 ** -70, 1.1 * 2.0 ** -60, 2.0 ** -40, 2.0 ** -24, 0.25, 0.9] * rows
    _check(torch.from_numpy(x).to(dtype).cuda(), [1.0] * rows, [1000, 900, 1000, 800], [1.0, 1.0, 1.0, 1.0], [0.0, 0.0, 1e-20, 0.0],
           [9] * rows, us=us)


@pytest.mark.gpu
def test_temperatures_at_the_ends():
    x = _logits("normal", 8, 3001, torch.float32)
    T = [1e-45, 1e-30, 1e-3, 0.05, 100.0, 1e6, 1e30, 3e38]
    for k, p in ((0, 1.0), (10, 1.0), (0, .5), (200, .5)):
        _check(x, T, [k] * 8, [p] * 8, [0.0] * 8, [20] * 8)


@pytest.mark.gpu
def test_magnitudes_at_the_ends():
    for scale in (1e-42, 1e-30, 1e4, 1e30, 1e38):
        x = (_logits("normal", 6, 2000, torch.float32) / 8).clamp(-3, 3) * scale
        _check(x, [0.8, 0.8, 1e30, 1e38, 0.8, 1.0], [0, 7, 0, 40, 0, 0], [1, 1, .9, .9, .5, 1], [0, 0, 0, 0, 0, .1], [9] * 6)


@pytest.mark.gpu
def test_rows_without_a_distribution():
    inf, nan = float("inf"), float("nan")
    for vocab in (300, 40000):
        x = _logits("normal", 14, vocab, torch.float32)
        x[1, 7], x[2, vocab - 1], x[3] = nan, inf, -inf
        x[4, 0], x[4, 1] = inf, -inf
        T, k, p, m = np.full(14, 0.8), np.full(14, 5), np.full(14, 0.9), np.full(14, 0.1)
        T[5], T[6], T[7], k[8], p[9], p[10], p[11], m[12], m[13] = -1.0, nan, inf, -1, 1.5, nan, -0.1, 1.1, nan
        off, us, tok, cnt, ng = _run(x, T, k, p, m, [2] * 14)
        assert ng[0] > 0 and np.all(ng[1:] == -1) and np.all(tok[2:] == -1) and np.all(cnt[2:] == 0)
        off, us, tok, cnt, ng = _run(x, T, k, p, m, [0] * 14)       # no draws: settings are looked at, logits are not
        assert ng.tolist() == [0] * 5 + [-1] * 9


@pytest.mark.gpu
def test_rows_outside_the_arrays():
    x = torch.zeros((5, 100), device="cuda")
    off = torch.tensor([0, 2, 9, 4, 6, -(1 << 31)], dtype=torch.int32, device="cuda")
    u = torch.tensor([0.015, 0.5, 0.25, 0.75, 0.125, 0.995], device="cuda")
    tok, cnt, ng = tkv.tkv_filter_sample(x, torch.ones(5, device="cuda"), off, u, 8)
    assert ng.tolist()[1:3] == [-1, -1] and ng[4] == -1
    assert ng[0] == 2 and tok[0:2].tolist() == [1, 50] and ng[3] == 2 and tok[4:6].tolist() == [12, 99]
    many = torch.tensor([0, 1025], dtype=torch.int32, device="cuda")
    assert tkv.tkv_filter_sample(x[:1], torch.ones(1, device="cuda"), many, torch.rand(1025, device="cuda"), 1024)[2].tolist() == [-1]


@pytest.mark.gpu
def test_rows_of_more_draws_than_max_potential_are_served():
    # as tkv_cd_sample does: the argument's own range is checked, a row is refused past 1,024 draws
    x = _logits("normal", 2, 4000, torch.float32)
    off, u = torch.tensor([0, 3, 103], dtype=torch.int32, device="cuda"), torch.rand(103, device="cuda")
    T = torch.ones(2, device="cuda")
    want = tkv.tkv_filter_sample(x, T, off, u, 100)
    assert want[2].min() > 0 and int(want[1].sum()) == 103
    for most in (0, 2):
        assert all(torch.equal(a, b) for a, b in zip(tkv.tkv_filter_sample(x, T, off, u, most), want))


@pytest.mark.gpu
def test_as_tkv_cd_sample_without_filters():
    # the plain sampler's sums are in 32 bits: a draw in reach of a border may differ
    x = _logits("normal", 40, 32000, torch.float32)
    off = torch.arange(41, dtype=torch.int32, device="cuda") * 3
    u = torch.rand(120, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    a = tkv.tkv_cd_sample(x, 0.8, off, u, 3)
    b = tkv.tkv_filter_sample(x, torch.full((40,), 0.8, device="cuda"), off, u, 3)
    same = sum(int(a[2][r] == b[2][r]) and torch.equal(a[0][3 * r:3 * r + int(a[2][r])], b[0][3 * r:3 * r + int(b[2][r])]) for r in range(40))
    assert same >= 38


@pytest.mark.gpu
def test_other_streams_and_replays():
    x = _logits("peaked", 30, 9000, torch.float32)
    T, k, p = torch.full((30,), 0.8, device="cuda"), torch.full((30,), 20, dtype=torch.int32, device="cuda"), torch.full((30,), .9, device="cuda")
    k[::3], p[1::4] = 0, 1.0
    off, u = torch.arange(31, dtype=torch.int32, device="cuda") * 4, torch.rand(120, device="cuda")
    call = lambda **other: tkv.tkv_filter_sample(x, T, off, u, 4, k, p, **other)
    want = call()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream, 0):
        torch.cuda.synchronize()
        got = call(stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for seed in range(4):
        x.copy_(_logits(KINDS[seed], 30, 9000, torch.float32, seed=seed))
        u.uniform_()
        graph.replay()
        want = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_inputs_dropped_after_a_call_on_another_stream():
    # their memory is not handed out again while that stream may still read it
    side = torch.cuda.Stream()
    off, u = torch.arange(31, dtype=torch.int32, device="cuda") * 4, torch.rand(120, device="cuda")
    kept = dict(x=_logits("peaked", 30, 90000, torch.float32), T=torch.full((30,), 0.8, device="cuda"))
    torch.cuda.synchronize()
    for name in ("x", "T"):
        args = dict(kept, **{name: kept[name].clone()})
        torch.cuda.synchronize()
        at = args[name].data_ptr()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        tkv.tkv_filter_sample(args["x"], args["T"], off, u, 4, stream=side)
        del args
        new = torch.empty_like(kept[name])
        busy = not side.query()
        torch.cuda.synchronize()
        assert busy and new.data_ptr() != at, name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows", [(torch.float32, 335), (torch.bfloat16, 670)])
def test_logits_of_more_than_192_mib(dtype, rows):
    # read past the caches; an odd vocabulary, rows that start at any element
    vocab = 151937
    assert rows * vocab * dtype.itemsize >= 192 << 20
    x = _logits("normal", rows, vocab + 6, dtype, seed=3)[:, 3:3 + vocab]
    x[::2, ::997] += 9
    rng = np.random.default_rng(3)
    T, k = rng.choice([0.3, 0.8, 1.0], rows), rng.choice([0, 0, 1, 50, 1000], rows)
    p, m = rng.choice([1.0, 0.9, 0.5], rows), rng.choice([0.0, 0.0, 0.05], rows)
    off, us, tok, cnt, ng = _run(x, T, k, p, m, [3] * rows, seed=3)
    for r in list(range(0, rows, 17)) + [1, rows - 2, rows - 1]:
        t, c = _plain(x[r].float().cpu().numpy(), T[r], int(k[r]), p[r], m[r], us[3 * r:3 * r + 3])
        assert tok[3 * r:3 * r + ng[r]].tolist() == t.tolist() and cnt[3 * r:3 * r + ng[r]].tolist() == c.tolist(), r


@pytest.mark.gpu
def test_more_rows_read_again_than_workgroups():
    # 1,100 rows whose top-p keeps thousands of tokens, and a top-k past the runs that are looked into
    rows, vocab = 1100, 8200
    x = _logits("normal", rows, vocab, torch.bfloat16)
    k = np.where(np.arange(rows) % 11 == 0, 3500, 0)
    off, us, tok, cnt, ng = _run(x, np.full(rows, 1.0), k, np.full(rows, 0.95), None, [2] * rows)
    host = x.float().cpu().numpy()
    for r in list(range(0, rows, 61)) + list(range(1020, 1100, 7)):
        t, c = _plain(host[r], 1.0, k[r], 0.95, 0.0, us[2 * r:2 * r + 2])
        assert tok[2 * r:2 * r + ng[r]].tolist() == t.tolist() and cnt[2 * r:2 * r + ng[r]].tolist() == c.tolist(), r


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["normal", "peaked", "steps", "masked"])
@pytest.mark.parametrize("vocab", [12000, 32000, 128256])
def test_large_top_k(vocab, kind, dtype):
    n = 20
    k = np.array([512, 513, 700, 1000, 1024, 1500, 2500, 4000, 5000, 11000] * 2)
    p = np.array([1.0] * 7 + [0.95, 0.5, 0.999, 0.9, 0.0, 0.95, 0.99, 1.0, 0.7, 0.9, 1.0, 1.0, 0.95])
    m = np.where(np.arange(n) % 6 == 5, 0.02, 0.0)
    T = np.array([0.8, 1.3, 0.3, 1.0, 30.0] * 4)
    _check(_logits(kind, n, vocab, dtype, seed=vocab + 1), T, k, p, m, [1, 3, 20, 2] * 5, seed=vocab + 1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [2049, 3001, 8200, 12288])
def test_min_p_that_keeps_more_than_a_list_before_top_p(vocab, dtype):
    # at most 384 runs of 32 reach the min-p bound and hold more than 2,048 tokens: the rows turn to top-p's own bound
    rows = 600
    x = _logits("flat", rows, vocab, dtype, seed=vocab)
    p, m = np.tile([0.95, 0.02, 0.5, 0.999], rows // 4), np.tile([0.01, 0.3, 0.02], rows // 3)
    off, us, tok, cnt, ng = _run(x, np.full(rows, 1.0), None, p, m, [3] * rows, seed=vocab)
    host = x.float().cpu().numpy()
    for r in range(rows):
        t, c = _plain(host[r], 1.0, 0, p[r], m[r], us[3 * r:3 * r + 3])
        assert tok[3 * r:3 * r + ng[r]].tolist() == t.tolist() and cnt[3 * r:3 * r + ng[r]].tolist() == c.tolist(), (r, p[r], m[r])


@pytest.mark.gpu
def test_a_workspace_of_the_callers():
    x = _logits("normal", 9, 20000, torch.float32)
    T, p = torch.ones(9, device="cuda"), torch.full((9,), 0.9, device="cuda")
    off, u = torch.arange(10, dtype=torch.int32, device="cuda") * 2, torch.rand(18, device="cuda")
    want = tkv.tkv_filter_sample(x, T, off, u, 2, None, p)
    n = tkv.tkv_filter_sample_workspace_bytes(9, 20000)
    ws = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    for _ in range(2):                                               # what it holds before a call does not matter
        got = tkv.tkv_filter_sample(x, T, off, u, 2, None, p, workspace=ws[16:16 + n])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert bool((ws[:16] == 0xA5).all()) and bool((ws[16 + n:] == 0xA5).all())
    for bad in (ws[:n - 1], ws[1:n + 1], ws[:0]):
        with pytest.raises(tkv.TkvError):
            tkv.tkv_filter_sample(x, T, off, u, 2, None, p, workspace=bad)
    with pytest.raises(ValueError):
        tkv.tkv_filter_sample(x, T, off, u, 2, None, p, workspace=ws.cpu())


@pytest.mark.gpu
def test_two_graphs_replayed_in_turn_and_two_streams_at_once():
    sets = []
    for seed, vocab in ((1, 30000), (2, 30000)):
        x = _logits("normal", 40, vocab, torch.float32, seed=seed)
        T, p = torch.full((40,), 0.9, device="cuda"), torch.full((40,), 0.8, device="cuda")
        off = torch.arange(41, dtype=torch.int32, device="cuda") * 3
        u = torch.rand(120, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
        sets.append((x, T, off, u, 3, None, p))
    want = [tkv.tkv_filter_sample(*a) for a in sets]
    graphs, got = [torch.cuda.CUDAGraph() for _ in sets], []
    for graph, a in zip(graphs, sets):
        with torch.cuda.graph(graph):
            got.append(tkv.tkv_filter_sample(*a))
    for _ in range(3):
        for g in got:
            g[0].zero_()
        for graph in graphs:
            graph.replay()
        eager = tkv.tkv_filter_sample(*sets[0])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got + [eager], want + [want[0]]) for a, b in zip(g, w))
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(5):
        both = [tkv.tkv_filter_sample(*a, stream=s) for a, s in zip(sets, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(both, want) for a, b in zip(g, w))


@pytest.mark.gpu
def test_tensors_are_checked():
    x = torch.zeros((4, 100), device="cuda")
    a = dict(logits=x, temperature=torch.ones(4, device="cuda"), draw_off=torch.arange(5, dtype=torch.int32, device="cuda"),
             uniform=torch.rand(4, device="cuda"), max_potential=1, top_k=torch.ones(4, dtype=torch.int32, device="cuda"))
    assert tkv.tkv_filter_sample(**a)[2].tolist() == [1] * 4
    for name, bad in (("logits", x.double()), ("logits", x.t()), ("logits", x[0]), ("logits", x.cpu()), ("logits", x[:1].expand(4, -1)),
                      ("temperature", a["temperature"][:3]), ("temperature", a["temperature"].double()), ("draw_off", a["draw_off"].long()),
                      ("draw_off", a["draw_off"][:4]), ("uniform", a["uniform"].double()), ("top_k", a["top_k"].long()),
                      ("top_p", a["top_k"]), ("min_p", torch.zeros(8, device="cuda")[::2])):
        with pytest.raises(ValueError):
            tkv.tkv_filter_sample(**dict(a, **{name: bad}))
    for most in (-1, 1025):
        with pytest.raises(tkv.TkvError):
            tkv.tkv_filter_sample(**dict(a, max_potential=most))
    with pytest.raises(tkv.TkvError, match="exceeds"):
        tkv.tkv_filter_sample(**dict(a, logits=torch.zeros((4, (1 << 21) + 1), device="cuda")))
    tok, cnt, ng = tkv.tkv_filter_sample(x[:0], a["temperature"][:0], a["draw_off"][:1], a["uniform"], 1)
    assert ng.numel() == 0


def test_bad_arguments_are_refused():
    # refused before any device access (no GPU needed)
    L, one = tkv.lib(), 16

    def call(n=1, vocab=10, kind=0, logits=one, stride=10, T=one, most=1, n_draws=1, u=one, off=one):
        return L.tkv_filter_sample(n, vocab, kind, logits, stride, T, one, one, one, most, u, off, n_draws, one, one, one, one, 1 << 40, None)

    for bad in (dict(n=-1), dict(vocab=0), dict(vocab=(1 << 21) + 1, stride=1 << 22), dict(kind=2), dict(kind=-1), dict(stride=9),
                dict(logits=None), dict(T=None), dict(most=-1), dict(most=1025), dict(n_draws=-1), dict(u=None), dict(off=None)):
        assert call(**bad) == tkv.TKV_EINVAL, bad
    assert call(n=0) == tkv.TKV_OK and call(n=0, logits=None) == tkv.TKV_OK


def test_more_rows_than_a_launch_takes_are_refused():
    # before any device access: 512 threads a row, under 2^32 in a launch; a wave a tile of 2,048 logits
    L, one = tkv.lib(), 16
    for n, vocab in ((1 << 23, 1), ((1 << 31) - 1, 1), (1 << 22, 16 * 2048)):
        assert L.tkv_filter_sample(n, vocab, 0, one, vocab, one, one, one, one, 1, one, one, 1, one, one, one, one, 1 << 62, None) == tkv.TKV_EINVAL
        assert "too many" in tkv.tkv_last_error()
