"""Logits under their rows' rules, against float64.

Bounds.  In fp32: the repetition's reciprocal, its product, frequency times count, and three additions are rounded once each,
2^-24 of their value, so an adjusted logit is off by at most 2^-22 of |l| max(rep, 1 / rep) + |frequency c| + |presence| + |bias|
(six roundings and the products of them).  A bf16 result is rounded once more, by 2^-8 of it.  Values without a rule pass as they
are, and what is not allowed is -inf.
"""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_39334_amd as tkv
from _rows import BS, Rows, dev


class Case(Rows):
    def __init__(self, rows, vocab, seed=0, in16=False, out16=False, grammar=0.3, bias=0.5, stride=0, out_stride=0, **more):
        super().__init__(rows, seed, **more)
        rng, n, self.vocab = self.rng, int(self.q_ptr[-1]), vocab
        # frequent tokens; some outside the vocabulary
        self.tokens = (vocab * rng.random((self.nb, BS)) ** 3).astype(np.int32)
        odd = rng.random((self.nb, BS)) < 0.02
        self.tokens[odd] = rng.choice([-1, vocab, 2**31 - 1, -2**31], size=int(odd.sum()))
        R = len(rows)
        lens = np.array([len(self.path(r)[0]) for r in range(R)])
        self.rules = {"prompt_len": (lens * rng.uniform(-0.1, 1.2, R)).astype(np.int32),
                      "repetition": rng.choice([1.0, 1.1, 0.9, 2.0], R).astype(np.float32),
                      "presence": rng.choice([0.0, 0.5, -1.5], R).astype(np.float32),
                      "frequency": rng.choice([0.0, 0.1, -0.5], R).astype(np.float32)}
        count = np.where(rng.random(R) < bias, rng.integers(0, 40, R), 0)
        m = int(count.sum())
        # a few tokens, so that many are listed twice, and some outside the vocabulary
        self.rules.update(bias_indptr=np.cumsum(np.concatenate(([0], count))).astype(np.int32),
                          bias_token=rng.integers(-2, min(vocab, 30) + 2, m).astype(np.int32),
                          bias_value=rng.choice([-100.0, 3.0, 0.25, -np.inf], m).astype(np.float32))
        self.rules["grammar"] = np.where(rng.random(n) < grammar, rng.integers(0, 5, n), rng.integers(-3, 0, n)).astype(np.int32)
        words = -(-vocab // 32) + seed % 3
        bits = rng.integers(0, 1 << 32, (5, words), dtype=np.uint32)
        bits[0], bits[1] = 0, 0xFFFFFFFF
        self.rules["allowed"] = bits.view(np.int32)
        g = torch.Generator(device="cuda").manual_seed(seed)
        room = torch.randn((n, vocab + stride), generator=g, device="cuda") * 3
        special = torch.rand(room.shape, generator=g, device="cuda")
        for i, x in enumerate((0.0, -0.0, float("inf"), -float("inf"), float("nan"))):
            room = torch.where((special > i * 0.005) & (special < i * 0.005 + 0.005), x, room)
        self.room = room.to(torch.bfloat16 if in16 else torch.float32)
        self.logits = self.room[:, :vocab]
        self.out = torch.full((n, vocab + out_stride), 7.0, dtype=torch.bfloat16 if out16 else torch.float32, device="cuda")

    def run(self, out=None, without=(), stream=None, **other):
        if out is None:
            self.out.fill_(7)
            out = self.out[:, :self.vocab]
        args = dict(self.arrays(), tokens=dev(self.tokens), logits=self.logits, out=out, stream=stream,
                    **{k: dev(v) for k, v in self.rules.items() if k not in without})
        args.update(other)
        assert tkv.tkv_adjust_logits(**args) is args["out"]
        return args["out"]

    def check(self, out, without=(), rows=None):
        on = {k: v for k, v in self.rules.items() if k not in without}
        for r in range(len(self.L)) if rows is None else rows:
            path = self.tokens.reshape(-1)[self.path(r)[1]].astype(np.int64)
            see, N = self.seen(r), len(path)
            rep, pres, freq = (float(on[k][r]) if k in on else off for k, off in (("repetition", 1), ("presence", 0), ("frequency", 0)))
            prompt = int(on["prompt_len"][r]) if "prompt_len" in on else 0
            bias = np.zeros(self.vocab)
            if "bias_token" in on:
                for e in range(on["bias_indptr"][r], on["bias_indptr"][r + 1]):
                    if 0 <= on["bias_token"][e] < self.vocab:
                        bias[on["bias_token"][e]] = on["bias_value"][e]
            for i in range(self.L[r]):
                q = int(self.q_ptr[r]) + i
                x = self.logits[q].double().cpu().numpy()
                inside = (path >= 0) & (path < self.vocab)
                seen = np.zeros(self.vocab, bool)
                seen[path[see[i] & inside]] = True
                c = np.bincount(path[see[i] & inside & (np.arange(N) >= prompt)], minlength=self.vocab)
                with np.errstate(invalid="ignore", over="ignore"):
                    y = np.where(seen, np.where(x > 0, x / rep, x * rep), x)
                    y = y - freq * c - pres * (c > 0) + bias
                    size = np.where(seen, np.abs(x) * max(rep, 1 / rep), np.abs(x)) + np.abs(freq * c) + abs(pres) * (c > 0) + np.abs(bias)
                    rule = seen | (bias != 0)
                    bound = np.where(rule, 2.0 ** -22 * size, 0.0)
                    if out.dtype == torch.bfloat16 and (self.logits.dtype != torch.bfloat16):
                        bound = bound + 2.0 ** -8 * (np.abs(y) + bound)
                    elif out.dtype == torch.bfloat16:
                        bound = bound + np.where(rule, 2.0 ** -8 * (np.abs(y) + bound), 0.0)
                g = int(on["grammar"][q]) if "grammar" in on else -1
                if g >= 0:
                    y[((on["allowed"].view(np.uint32)[g][np.arange(self.vocab) // 32] >> (np.arange(self.vocab) % 32)) & 1) == 0] = -np.inf
                got = out[q].double().cpu().numpy()
                plain = np.isfinite(y)
                assert np.array_equal(np.isnan(y), np.isnan(got)) and np.array_equal(y[~plain & ~np.isnan(y)], got[~plain & ~np.isnan(y)]), (r, i)
                worst = np.max(np.abs(got[plain] - y[plain]) - bound[plain], initial=0.0)
                assert worst <= 0, (r, i, worst)


TYPES = [(False, False), (True, True), (True, False), (False, True)]


@pytest.mark.gpu
@pytest.mark.parametrize("in16,out16", TYPES)
@pytest.mark.parametrize("vocab", [1, 3, 31, 500, 8191, 8192, 8195, 32003, 151936])
def test_vocabularies_of_many_sizes(vocab, in16, out16):
    c = Case([(200, 1), (0, 1), (90, 3), (700, 1)], vocab, vocab, in16, out16)
    c.check(c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("in16,out16", TYPES)
def test_rows_that_start_anywhere(in16, out16):
    for vocab, stride, out_stride in ((1001, 1, 3), (9001, 7, 0), (8200, 8, 2)):
        c = Case([(50, 2), (300, 5)], vocab, vocab, in16, out16, stride=stride, out_stride=out_stride)
        c.check(c.run())
        assert torch.all(c.out[:, vocab:] == 7)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [[(500, 32), (3, 9), (0, 1)], [(300, 130)], [(10, 1024)], [(0, 5), (1, 1), (2000, 64)]])
@pytest.mark.parametrize("bits", [False, True])
def test_drafted_trees(rows, bits):
    c = Case(rows, 777, 5, bits=bits, extra_words=1)
    c.check(c.run())
    c = Case(rows, 20011, 6, True, bits=bits)
    c.check(c.run())


@pytest.mark.gpu
def test_long_paths():
    for n in (8000, 8192, 30000, 100000):
        c = Case([(n, 1), (n // 3, 4)], 5003, n)
        c.check(c.run())
    # one token everywhere: counts past 16 bits
    c = Case([(90000, 1), (70000, 3)], 100, 3)
    c.tokens[:] = 42
    c.rules["frequency"][:], c.rules["prompt_len"][:] = 0.001, [0, 1000]
    c.check(c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("m", [60000, 70000])
def test_biases_for_every_token(m):
    # many times over: the last one counts
    c = Case([(300, 2), (50, 1)], 9001, 5)
    c.rules["bias_indptr"] = np.array([0, m, m + 10], np.int32)
    c.rules["bias_token"] = c.rng.integers(0, 9001, m + 10).astype(np.int32)
    c.rules["bias_value"] = c.rng.normal(size=m + 10).astype(np.float32)
    c.check(c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("in16,out16", TYPES)
@pytest.mark.parametrize("others", [2, 15])
def test_counts_and_biases_at_the_limit_of_16_bits(others, in16, out16):
    # enough workgroups for numbers of 16 bits: one token 32,752 times over (with the drafted ones), as many biases as they hold
    c = Case([(2047 * BS - 32, 32)] + [(40 + r, 2) for r in range(others)], 151936, others, in16, out16, full_blocks=True, bias=0.0)
    path = c.path(0)[1]
    c.tokens.reshape(-1)[path] = 42
    c.rules["prompt_len"][:], c.rules["frequency"][:] = 0, 0.001
    m = 65534
    c.rules["bias_indptr"][2:] = m
    c.rules["bias_token"] = c.rng.integers(0, 9001, m).astype(np.int32)
    c.rules["bias_value"] = c.rng.normal(size=m).astype(np.float32)
    assert c.max_blocks == 2047
    c.check(c.run(), rows=[0, 1, others])
    off = ("bias_indptr", "bias_token", "bias_value")
    c.check(c.run(without=off), off, rows=[1, others])


@pytest.mark.gpu
def test_rules_that_are_off():
    names = ["prompt_len", "repetition", "presence", "frequency", "bias", "grammar"]
    for off in [names] + [[x] for x in names] + [names[:4], names[4:], names[1:]]:
        without = [y for x in off for y in {"bias": ("bias_indptr", "bias_token", "bias_value"), "grammar": ("grammar", "allowed")}.get(x, (x,))]
        c = Case([(300, 3), (40, 1), (5, 2)], 9001, 11)
        c.check(c.run(without=without), without)
    c = Case([(300, 3)], 501, 1, True)
    got = tkv.tkv_adjust_logits(**c.arrays(), tokens=dev(c.tokens), logits=c.logits)
    assert got.dtype == torch.bfloat16 and torch.equal(got.view(torch.int16), c.logits.contiguous().view(torch.int16))


@pytest.mark.gpu
@pytest.mark.parametrize("in16", [False, True])
def test_in_place_and_rows_between_each_other(in16):
    for rows in ([(200, 1), (90, 3)], [(100, 40)]):
        c = Case(rows, 9001, 4, in16, in16, stride=5)
        want = c.run().clone()
        mine = c.room.clone()
        c.run(out=mine[:, :9001], logits=mine[:, :9001])
        same = lambda a, b: torch.equal(a.nan_to_num(5, 6, 7), b.nan_to_num(5, 6, 7)) and torch.equal(a.isnan(), b.isnan())
        assert same(mine[:, :9001], want) and same(mine[:, 9001:], c.room[:, 9001:])
        both = torch.zeros((len(want), 18010), dtype=c.room.dtype, device="cuda")
        both[:, :9001] = c.logits
        c.run(out=both[:, 9005:18006], logits=both[:, :9001])
        assert same(both[:, 9005:18006], want) and same(both[:, :9001], c.logits)
        for bad in (both[:, 9000:18001], both[:, 1:9002], both[:, 9010:]):
            with pytest.raises((tkv.TkvError, ValueError)):
                c.run(out=bad, logits=both[:, :9001])


@pytest.mark.gpu
def test_prompt_lengths_of_any_size():
    # below 0 is no prompt, past the path's end all of it
    c = Case([(300, 3), (2000, 1), (40, 2), (700, 12), (50, 1)], 501, 4)
    c.rules["frequency"][:], c.rules["presence"][:] = 0.25, 0.5
    c.rules["prompt_len"][:] = [-2**31, -2**31 + 40, -1, 2**31 - 1, -2**31]
    c.check(c.run())


@pytest.mark.gpu
def test_settings_outside_their_ranges():
    c = Case([(100, 2)] * 12, 9001, 2, grammar=0.0)
    want = c.run().clone()
    n = c.q_ptr
    bad = {k: v.copy() for k, v in c.rules.items()}
    for i, x in enumerate((0.0, 1e-39, np.nan, np.inf)):
        bad["repetition"][i] = x
    bad["presence"][4], bad["frequency"][5] = np.inf, np.nan
    bad["grammar"][n[6]] = 5
    got = c.run(**{k: dev(v) for k, v in bad.items()})
    for r in range(12):
        rows = slice(n[r], n[r + 1])
        if r < 6:
            assert torch.all(got[rows].isnan()), r
        elif r == 6:
            assert torch.all(got[n[6]].isnan()) and torch.equal(got[n[6] + 1].nan_to_num(9), want[n[6] + 1].nan_to_num(9))
        else:
            assert torch.equal(got[rows].nan_to_num(9), want[rows].nan_to_num(9)), r
    m = len(c.rules["bias_token"])
    ptr = c.rules["bias_indptr"].copy()
    ptr[0], ptr[-1] = -1, m + 1
    got = c.run(bias_indptr=dev(ptr))
    assert torch.all(got[:2].isnan()) and torch.all(got[-2:].isnan()) and torch.equal(got[2:-2].nan_to_num(9), want[2:-2].nan_to_num(9))
    # the samplers say which rows these are
    R = len(got)
    one = torch.ones(R, device="cuda")
    off = torch.arange(R + 1, dtype=torch.int32, device="cuda")
    clean = torch.where(want.isfinite(), got, -1.0).where(~got.isnan() | want.isfinite(), -1.0)
    clean[:2], clean[-2:] = float("nan"), float("nan")
    _, _, groups = tkv.tkv_filter_sample(clean, one, off, torch.full((R,), 0.5, device="cuda"), 1)
    assert groups.tolist() == [-1] * 2 + [1] * (R - 4) + [-1] * 2


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [9001, 70000])
def test_the_samplers_say_which_rows_are_refused(vocab):
    # the operator's output as it is: every token of a refused row, and the one whose grammar is none, draws nothing
    c = Case([(100, 2)] * 12, vocab, 2, grammar=0.0)
    finite = c.logits.nan_to_num(1.0, 5.0, -5.0)
    u = {k: v.copy() for k, v in c.rules.items()}
    u["bias_value"] = np.where(np.isfinite(u["bias_value"]), u["bias_value"], -4.0).astype(np.float32)
    u["allowed"][1, :] = -1   # all tokens
    u["grammar"][:] = np.where(np.arange(24) % 2, 1, -1)
    u["repetition"][1], u["presence"][4], u["frequency"][7], u["grammar"][17] = np.nan, np.inf, -np.inf, 5
    u["bias_indptr"][-1] += 1
    want = [-1 if i // 2 in (1, 4, 7, 11) or i == 17 else 1 for i in range(24)]
    got = c.run(logits=finite, **{k: dev(v) for k, v in u.items()}, out=torch.empty_like(finite))
    off, half = torch.arange(25, dtype=torch.int32, device="cuda"), torch.full((24,), 0.5, device="cuda")
    tok, _, groups = tkv.tkv_filter_sample(got, torch.ones(24, device="cuda"), off, half, 1)
    assert groups.tolist() == want and [t >= 0 for t in tok.tolist()] == [g == 1 for g in want]
    tok, _, groups = tkv.tkv_cd_sample(got, 1.0, off, half, 1)
    assert groups.tolist() == want
    assert torch.equal(got.isnan().all(1), dev(np.array(want) < 0)) and torch.equal(got.isnan().any(1), got.isnan().all(1))


@pytest.mark.gpu
def test_rows_outside_the_arrays():
    c = Case([(100, 4), (160, 6), (100, 8), (1500, 5), (90, 3), (90, 2)], 900, 3)
    same = lambda x, y: torch.equal(x.nan_to_num(9), y.nan_to_num(9))
    want = c.run().clone()
    a = c.arrays()
    at, n = lambda r: slice(c.q_ptr[r], c.q_ptr[r + 1]), int(c.q_ptr[-1])
    kv = a["kv_indptr"].clone()
    kv[-1] = a["kv_blocks"].numel() + 1
    out = c.run(kv_indptr=kv, max_blocks=50)
    for r in range(6):
        assert torch.all(out[at(r)].isnan()) if r in (3, 5) else same(out[at(r)], want[at(r)])
    real = c.q_ptr.tolist()
    for ptr, kept in (([0, 4, 10, 18, 23, 26, n + 1], [0, 1, 2, 3, 4]), ([-4, 4, 10, 18, 23, 26, n], [1, 2, 3, 4, 5]),
                      ([0, 4, 10, 18, 18, 18, n], [0, 1, 2]), ([0, 4, 10, 1 << 30, -(1 << 31), 26, n], [0, 1, 5])):
        out = c.run(q_indptr=torch.tensor(ptr, dtype=torch.int32, device="cuda"))
        seen = torch.zeros(n, dtype=torch.bool, device="cuda")
        for r in kept:
            if ptr[r] == real[r] and ptr[r + 1] == real[r + 1]:
                assert same(out[at(r)], want[at(r)])
            seen[max(0, ptr[r]):max(0, ptr[r + 1])] = True
        assert torch.all(out[~seen] == 7)
    # fewer rows than tokens
    short = {k: dev(v[:2] if k == "bias_indptr" else v[:1] if len(v) == 6 else v) for k, v in c.rules.items()}
    out = c.run(q_indptr=a["q_indptr"][:2].clone(), kv_indptr=a["kv_indptr"][:2].clone(), **short)
    assert same(out[:4], want[:4]) and torch.all(out[4:] == 7)
    # entries that are no blocks
    c.tables[2][3] = c.nb + 1
    c.block_len[c.tables[3][5]] = 20
    c.check(c.run())


@pytest.mark.gpu
def test_max_q_above_the_rows_lengths():
    # two tokens share a workgroup's counts, or none do where max_q leaves most groups without tokens: the same bits
    c = Case([(50 + 3 * r, 11 - r % 2) for r in range(42)], 151936, seed=2, extra_words=15)
    want = c.run().clone()
    c.check(want, rows=[0, 17, 41])
    for max_q in (64, 400, 1024):
        assert torch.equal(c.run(max_q=max_q).view(torch.int32), want.view(torch.int32)), max_q


@pytest.mark.gpu
def test_many_rows_and_pools_past_four_gib():
    rng = np.random.default_rng(5)
    c = Case([(int(n), int(L)) for n, L in zip(rng.integers(0, 90, 700), rng.integers(1, 3, 700))], 601, 9)
    c.check(c.run(), rows=list(range(0, 700, 23)) + [255, 256, 699])
    big = torch.zeros((70_000_000, BS), dtype=torch.int32, device="cuda")
    off = len(big) - c.nb
    big[off:] = dev(c.tokens)
    lens = torch.zeros(len(big), dtype=torch.int32, device="cuda")
    a = c.arrays()
    lens[off:] = a["block_len"]
    want = c.run().clone()
    got = c.run(tokens=big, block_len=lens, kv_blocks=a["kv_blocks"] + off)
    assert torch.equal(got.nan_to_num(9), want.nan_to_num(9))


@pytest.mark.gpu
def test_logits_past_four_gib():
    c = Case([(30, 1)] * 3, 9001, 9)
    want = c.run().clone()
    stride = (1 << 30) + 7
    room = torch.zeros(2 * stride + 9001, device="cuda")
    x = room.as_strided((3, 9001), (stride, 1))
    x.copy_(c.logits)
    got = c.run(logits=x)
    assert torch.equal(got.nan_to_num(9), want.nan_to_num(9))
    c.run(logits=x, out=x)
    assert torch.equal(x.nan_to_num(9), want.nan_to_num(9))


@pytest.mark.gpu
def test_replays_streams_and_dropped_inputs():
    c = Case([(3000, 3), (400, 1), (50, 9)], 9001, 2)
    same = lambda x, y: torch.equal(x.nan_to_num(9), y.nan_to_num(9))
    want = c.run().clone()
    t = dict(c.arrays(), tokens=dev(c.tokens), logits=c.logits.clone(), out=torch.zeros_like(want), **{k: dev(v) for k, v in c.rules.items()})
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tkv.tkv_adjust_logits(**t)
    side = torch.cuda.Stream()
    for step in range(3):
        t["tokens"].copy_(dev(c.tokens) if step != 1 else dev(c.tokens) + 1)
        t["out"].fill_(7)
        graph.replay()
        eager = c.run(tokens=t["tokens"]).clone()
        torch.cuda.synchronize()
        assert same(t["out"], eager) and same(t["out"], want) == (step != 1)
    for stream in (None, side, side.cuda_stream, 0):
        for out in (t["out"], None):
            t["out"].fill_(7)
            torch.cuda.synchronize()
            got = tkv.tkv_adjust_logits(**dict(t, out=out), stream=stream)
            torch.cuda.synchronize()
            assert same(got, want)
    for name in ("mask", "tokens", "logits", "repetition", "bias_value", "allowed", "out"):
        args = dict(t)
        args[name] = args[name].clone()
        torch.cuda.synchronize()
        at, shape, dtype = args[name].data_ptr(), args[name].shape, args[name].dtype
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        tkv.tkv_adjust_logits(**args, stream=side)
        del args
        new = torch.empty(shape, dtype=dtype, device="cuda")
        busy = not side.query()
        torch.cuda.synchronize()
        assert busy and new.data_ptr() != at, name


@pytest.mark.gpu
def test_tensors_are_checked():
    c = Case([(30, 4), (5, 1)], 700)
    a, u = c.arrays(), {k: dev(v) for k, v in c.rules.items()}
    for name, bad in (("tokens", dev(c.tokens).long()), ("tokens", dev(c.tokens)[:, :8]), ("tokens", dev(c.tokens)[1:]),
                      ("logits", c.logits[1:]), ("logits", c.logits.double()), ("logits", c.logits.t().contiguous().t()),
                      ("logits", c.logits.cpu()), ("out", torch.zeros(5, 699, device="cuda")), ("out", torch.zeros(5, 700, device="cuda").half()),
                      ("mask", a["mask"][1:]), ("q_indptr", a["q_indptr"][:0]), ("kv_indptr", a["kv_indptr"][1:]),
                      ("prompt_len", u["prompt_len"].long()), ("repetition", u["repetition"][1:]), ("presence", u["presence"].double()),
                      ("frequency", u["frequency"].cpu()), ("bias_indptr", u["bias_indptr"][1:]), ("bias_token", None),
                      ("bias_value", u["bias_value"].repeat(2)), ("grammar", u["grammar"][1:]), ("allowed", None),
                      ("allowed", u["allowed"].long())):
        with pytest.raises(ValueError):
            c.run(**{name: bad})
    for name, bad in (("max_q", 0), ("max_q", 65), ("max_q", 1025), ("max_blocks", 0), ("max_blocks", 1 << 28),
                      ("allowed", u["allowed"][:, :20].contiguous())):
        with pytest.raises(tkv.TkvError):
            c.run(**{name: bad})


def test_bad_arguments_are_refused():
    # refused before any device access (no GPU needed)
    L, one, far = tkv.lib(), 16, 1 << 30

    def call(nb=4, tokens=one, n_rows=1, n_qtok=4, max_q=4, n_kv=9, max_blocks=9, words=1, ptr=one, vocab=100, t_in=0, x=one, stride=100,
             t_out=0, y=far, out_stride=100, n_bias=0, bias=None, grammar=None, allowed=None, n_grammars=0, allowed_words=0, rules=True):
        b = tkv.tkv_draft_batch(n_rows, n_qtok, max_q, n_kv, max_blocks, words, ptr, one, one, one, one)
        u = tkv.tkv_logit_rules(None, None, None, None, bias, bias, bias, grammar, allowed, n_bias, n_grammars, allowed_words)
        return L.tkv_adjust_logits(nb, tokens, ctypes.byref(b), ctypes.byref(u) if rules else None, vocab, t_in, x, stride, t_out, y,
                                   out_stride, None)

    for bad in (dict(nb=0), dict(nb=1 << 28), dict(tokens=None), dict(tokens=one + 8), dict(n_rows=-1), dict(n_qtok=-1), dict(max_q=0),
                dict(max_q=1025), dict(max_q=65), dict(n_kv=-1), dict(max_blocks=0), dict(words=0), dict(ptr=None), dict(vocab=0),
                dict(vocab=(1 << 21) + 1, stride=1 << 22, out_stride=1 << 22), dict(t_in=2), dict(t_out=-1), dict(x=None), dict(y=None),
                dict(x=one + 2), dict(y=far + 1), dict(stride=99), dict(out_stride=99), dict(n_bias=-1), dict(n_bias=1),
                dict(n_grammars=-1), dict(n_grammars=1, grammar=one, allowed=None, allowed_words=4),
                dict(n_grammars=1, grammar=one, allowed=one, allowed_words=3), dict(rules=False),
                dict(y=one + 4), dict(y=one, t_out=1), dict(y=one, out_stride=101), dict(y=one + 4 * 399),
                dict(n_rows=1 << 24, n_qtok=1 << 24, max_q=1, y=1 << 50)):
        assert call(**bad) == tkv.TKV_EINVAL, bad
    assert call(n_rows=0) == tkv.TKV_OK and call(n_qtok=0) == tkv.TKV_OK
    assert L.tkv_adjust_logits(4, one, None, None, 100, 0, one, 100, 0, far, 100, None) == tkv.TKV_EINVAL
