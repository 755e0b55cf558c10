"""The attention weight that queries give the keys, against float64.

Bounds.  A weight is c exp(s - z): s = q . k / sqrt(d) from fp32 sums of exact products, off by at most d 2^-23 A with
A = sum |q k| / sqrt(d) (an accumulation may cut where it does not round); the scale, the lse in units of log2 and the difference
are rounded once each, 2^-24 of |s|, |z| and |s - z|, so 2^-23 (|s| + |z|) in all; the exponential and the coefficient add
2^-22.  A key's sum has at most `rows` additions, 2^-24 of the sum each, and the old weight's term 2^-22 of itself.  First order:
twice that covers the products of these.
"""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_39334_amd as tkv
from _rows import BS, Rows, dev

HEADS = [(28, 4, 128), (4, 4, 64), (16, 1, 64), (12, 2, 128), (15, 5, 64), (64, 1, 128), (40, 8, 128), (8, 2, 64)]


def more_entries(c):
    """Entries of no row behind the tables: the work is cut for as many keys as the arrays hold."""
    return {"kv_blocks": torch.cat([c.arrays()["kv_blocks"], torch.zeros(4096, dtype=torch.int32, device="cuda")])}


class Case(Rows):
    def __init__(self, rows, hq, hkv, d, seed=0, extra_keys=0, **more):
        super().__init__(rows, seed, **more)
        self.hq, self.hkv, self.d = hq, hkv, d
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
        n = int(self.q_ptr[-1])
        self.q, self.k = rand(n, hq, d), rand(self.nb, hkv, BS, d)
        for r in range(len(self.L)):   # a key that no token of its row sees may hold anything
            at, slot = self.path(r)
            for s in slot[~self.seen(r).any(0)]:
                self.k[s // BS, :, s % BS] = float("nan")
        dead = torch.arange(BS, device="cuda")[None, :] >= dev(self.block_len)[:, None]
        self.k.masked_fill_(dead[:, None, :, None], float("nan"))
        self.keys = BS * self.max_blocks + extra_keys
        self.coef = (torch.rand(n, generator=g, device="cuda") * 2).where(torch.rand(n, generator=g, device="cuda") < 0.7, 0.0)
        self.before = torch.rand((len(self.L), hkv, self.keys), generator=g, device="cuda") * 4
        self.lse = torch.zeros(n, hq, dtype=torch.float32, device="cuda")
        for r, L in enumerate(self.L):
            a = self.q_ptr[r]
            self.lse[a:a + L] = torch.logsumexp(self.scores(r)[0], -1).permute(2, 0, 1).reshape(L, hq).float()

    def scores(self, r):
        """[hkv, G, L, N] float64: the scores (-inf where hidden) and A."""
        at, slot = self.path(r)
        a, L, G = self.q_ptr[r], self.L[r], self.hq // self.hkv
        slot = dev(slot)
        k = self.k[slot // BS, :, slot % BS].double().transpose(0, 1).nan_to_num(0.0)
        q = self.q[a:a + L].double().view(L, self.hkv, G, self.d).permute(1, 2, 0, 3).reshape(self.hkv, G * L, self.d)
        x, A = (torch.matmul(y, z.transpose(1, 2).contiguous()).view(self.hkv, G, L, len(at)) / self.d ** 0.5
                for y, z in ((q, k), (q.abs(), k.abs())))
        return x.masked_fill(~dev(self.seen(r)), -float("inf")), A

    def run(self, decay=0.75, coef=True, before=True, stream=None, **other):
        out = torch.full((len(self.L), self.hkv, self.keys), 7.0, device="cuda")
        given = lambda x, own: x if torch.is_tensor(x) else own if x else None
        args = dict(self.arrays(), q=self.q, k=self.k, lse=self.lse, out=out, before=given(before, self.before), decay=decay,
                    coef=given(coef, self.coef), stream=stream)
        args.update(other)
        tkv.tkv_key_weights(**args)
        return args["out"]

    def check(self, out, decay=0.75, coef=True, before=True, rows=None):
        for r in range(len(self.L)) if rows is None else rows:
            at, _ = self.path(r)
            a, L, G = self.q_ptr[r], self.L[r], self.hq // self.hkv
            x, A = self.scores(r)
            z = self.lse[a:a + L].double().view(L, self.hkv, G).permute(1, 2, 0)[..., None]
            c = self.coef[a:a + L].double() if coef else torch.ones(L, device="cuda").double()
            p = torch.where(z.isfinite(), c[:, None] * torch.exp(x - torch.where(z.isfinite(), z, 0.0)), 0.0)
            off = p * (self.d * 2.0 ** -23 * A + 2.0 ** -23 * (x.abs().nan_to_num(0, 0, 0) + z.abs().nan_to_num(0, 0, 0)) + 2.0 ** -22)
            want, bound = p.sum((1, 2)), off.sum((1, 2))
            bound += G * L * 2.0 ** -24 * want
            if before:
                had = (decay * self.before[r][:, dev(at)].double()) * (torch.arange(len(at), device="cuda") < len(at) - L)
                want, bound = want + had, bound + 2.0 ** -22 * had.abs() + 2.0 ** -24 * want
            got = out[r][:, dev(at)].double()
            err = (got - want).abs()
            assert torch.all(err <= 2 * bound), (r, L, (err / bound).nan_to_num(9e9).max())
            rest = torch.ones(out.shape[2], dtype=torch.bool, device="cuda")
            rest[dev(at)] = False
            assert torch.all(out[r][:, rest] == 7)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("L", [1, 2, 7, 16, 33, 65, 130])
def test_drafts_of_one_size(hq, hkv, d, L):
    c = Case([(n, L) for n in (0, 1, 15, 16, 17, 100, 700)], hq, hkv, d, seed=L, extra_keys=L)
    c.check(c.run())
    c.check(c.run(**more_entries(c)))


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", HEADS[:4])
def test_ragged_rows_and_any_mask(hq, hkv, d):
    rng = np.random.default_rng(hq)
    rows = [(int(rng.integers(0, 900)), int(rng.integers(1, 90))) for _ in range(17)] + [(3000, 3), (0, 1), (0, 70)]
    for bits in (False, True):
        c = Case(rows, hq, hkv, d, seed=hq, bits=bits, extra_words=1)
        c.check(c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", [(64, 1, 64), (33, 1, 128), (62, 2, 64), (5, 5, 128), (9, 3, 64), (40, 8, 128)])
def test_any_masks_of_groups_of_any_size(hq, hkv, d):
    # tiles of 32 query rows that begin and end inside a token's group, masks looked up for several tiles at once
    c = Case([(5, 60), (300, 40), (0, 257), (77, 33), (1000, 130)], hq, hkv, d, seed=hq, bits=True, extra_words=2)
    c.check(c.run())
    c.check(c.run(**more_entries(c)))


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [[(30000, 1)], [(20000, 40)], [(9000, 9), (10, 1), (0, 2), (17000, 3)], [(4000, 300)],
                                  [(70, 1024)], [(1, 1)] * 3])
def test_long_and_short_paths(rows):
    c = Case(rows, 12, 2, 128, seed=3)
    c.check(c.run())
    c.check(c.run(**more_entries(c)))


@pytest.mark.gpu
def test_few_rows_in_tables_of_a_large_capacity():
    c = Case([(200, 40), (0, 1), (30, 70), (900, 33)], 12, 2, 64, seed=8, extra_keys=16 * 5000)
    c.check(c.run(max_blocks=c.max_blocks + 5000))


@pytest.mark.gpu
def test_old_weights_coefficients_and_decay():
    c = Case([(300, 5), (40, 1), (900, 17)], 8, 2, 64)
    c.check(c.run(decay=1.0, coef=False), 1.0, False)
    c.check(c.run(before=False, coef=False), 0.0, False, False)
    want = c.run()
    own = c.before.clone()          # in place
    tkv.tkv_key_weights(**c.arrays(), q=c.q, k=c.k, lse=c.lse, out=own, before=own, decay=0.75, coef=c.coef)
    for r in range(3):
        at = dev(c.path(r)[0])
        assert torch.equal(own[r][:, at], want[r][:, at])
    # not read where the decay is 0; a new key's old weight never is
    c.before.fill_(float("nan"))
    c.check(c.run(decay=0.0), 0.0, before=False)
    for r in range(3):
        at = dev(c.path(r)[0])[-c.L[r]:]
        assert torch.all(c.run(decay=1.0)[r][:, at].isfinite())
    # coefficients that are not above 0 leave a token out
    c.coef[:] = torch.tensor([0.0, -1.0, float("nan"), 1.0], device="cuda").repeat(6)[:23]
    got = c.run(decay=0.0)
    c.coef[:] = torch.tensor([0.0, 0.0, 0.0, 1.0], device="cuda").repeat(6)[:23]
    assert torch.equal(got, c.run(decay=0.0))


@pytest.mark.gpu
@pytest.mark.parametrize("L", [3, 40])
def test_tokens_that_are_left_out_may_hold_anything(L):
    # padding: no coefficient, or no attention
    c = Case([(300, L), (20, L), (1200, L)], 8, 2, 64)
    out = torch.arange(0, 3 * L, 3, device="cuda")
    for what in ("coef", "lse"):
        if what == "coef":
            c.coef[out] = 0.0
        else:
            c.coef = torch.ones_like(c.coef)
            c.lse[out] = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda").repeat(L)[:len(out), None]
        c.q[out] = 1.0
        want = c.run()
        for x in (float("nan"), float("inf"), -float("inf")):
            c.q[out] = x
            assert torch.equal(c.run(), want)
        if L > 3:  # the kernel for many keys
            c.q[out] = 1.0
            want = c.run(**more_entries(c))
            c.q[out] = float("nan")
            assert torch.equal(c.run(**more_entries(c)), want)


@pytest.mark.gpu
def test_queries_without_keys_give_nothing():
    # masks that hide everything: lse is -inf
    c = Case([(0, 1), (0, 40), (5, 3)], 8, 2, 64, bits=True, seed=5)
    c.masks[0][:] = 0
    c.masks[1][3] = 0
    c.lse[0], c.lse[4] = -float("inf"), -float("inf")
    c.lse[8] = float("nan")
    out = c.run()
    c.check(out)
    assert torch.all(out[0][:, 0] == 0)


@pytest.mark.gpu
def test_sums_of_real_attention():
    # each query's weights add up to 1: a row's to its tokens times its heads, for the lse of every attention entry point
    c = Case([(700, 9), (30, 1), (2000, 40)], 12, 2, 128, seed=8)
    o = torch.empty_like(c.q)
    v = torch.randn_like(c.k)
    k = c.k.nan_to_num(0.0)
    lse = torch.empty_like(c.lse)
    tkv.tkv_draft_verify(**c.arrays(), q=c.q, k=k, v=v, o=o, lse=lse)
    out = c.run(k=k, lse=lse, before=False, coef=False)
    c.lse = lse
    c.check(out, before=False, coef=False)
    for r, L in enumerate(c.L):
        total = out[r][:, dev(c.path(r)[0])].double().sum(1)
        assert torch.all((total - L * 6).abs() <= 2.0 ** -9 * L * 6)   # lse is off by 2^-11 at most
    chain = Case([(300, 5), (60, 1), (500, 30)], 12, 2, 128, seed=9)
    chain.masks = [tkv.tkv_draft_mask(list(range(-1, L - 1)), chain.masks[0].shape[1])[0] for L in chain.L]
    a = chain.arrays()
    plan = tkv.Plan((12, 2, 128, BS, chain.nb), chain.q_ptr, a["kv_indptr"].cpu().numpy(), a["kv_blocks"].cpu().numpy(),
                    chain.block_len)
    k = chain.k.nan_to_num(0.0)
    plan.verify(chain.q, k, torch.randn_like(k), torch.empty_like(chain.q), chain.lse)
    chain.k = k
    out = chain.run(before=False, coef=False)
    chain.check(out, before=False, coef=False)


@pytest.mark.gpu
def test_blocks_that_are_none_and_rows_outside_the_arrays():
    c = Case([(100, 4), (160, 6), (100, 8), (1500, 5), (90, 3), (90, 2)], 8, 2, 64)
    want = c.run()
    bad = Case([(100, 4), (160, 6), (100, 8), (1500, 5), (90, 3), (90, 2)], 8, 2, 64)
    gone = bad.tables[1][2]
    bad.tables[1][2] = bad.nb + 3        # an entry that is no block: its slots keep what they held
    out = bad.run()
    at = slice(16 * 2, 16 * 2 + int(bad.block_len[gone]))
    assert torch.all(out[1][:, at] == 7)
    same = torch.ones(out.shape[2], dtype=torch.bool, device="cuda")
    same[at] = False
    assert torch.equal(out[1][:, same], want[1][:, same]) and torch.equal(out[2:], want[2:])
    bad.tables[1][2] = gone
    bad.block_len[gone] = 17
    assert torch.all(bad.run()[1][:, at] == 7)
    a = c.arrays()
    total, n = a["kv_blocks"].numel(), c.q.shape[0]
    kv = a["kv_indptr"].clone()
    kv[-1] = total + 1
    out = c.run(kv_indptr=kv, max_blocks=40)    # row 3 is longer than max_blocks, the last one runs past the entries
    assert torch.all(out[3] == 7) and torch.all(out[5] == 7) and torch.equal(out[[0, 1, 2, 4]], want[[0, 1, 2, 4]])
    for ptr, kept in (([0, 4, 10, 18, 23, 26, n + 1], [0, 1, 2, 3, 4]), ([-4, 4, 10, 18, 23, 26, n], [1, 2, 3, 4, 5]),
                      ([0, 4, 3, 18, 23, 26, n], [0, 3, 4, 5]), ([0, 4, 10, 18, 18, 18, n], [0, 1, 2]),
                      ([0, 4, 10, 1 << 30, -(1 << 31), 26, n], [0, 1, 5])):
        out = c.run(q_indptr=torch.tensor(ptr, dtype=torch.int32, device="cuda"))
        real = c.q_ptr.tolist()
        for r in range(6):
            if r in kept and ptr[r] == real[r] and ptr[r + 1] == real[r + 1]:
                assert torch.equal(out[r], want[r])
            if not 1 <= ptr[r + 1] - ptr[r] <= c.max_q or ptr[r] < 0 or ptr[r + 1] > n:
                assert torch.all(out[r] == 7)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (14, 2, 64), (10, 2, 128), (9, 3, 64), (6, 2, 64)])
def test_hidden_keys_under_partial_tiles_may_hold_anything(hq, hkv, d):
    # a row's last tile of 32 query rows ends inside; what a call whose masks are all ones leaves on the chip must not count there
    rng, rows = np.random.default_rng(hq), 128 // hkv
    c = Case([(30, int(n)) for n in rng.integers(34, 60, rows)], hq, hkv, d, seed=2)
    infinite = c.k.clone()
    for r, L in enumerate(c.L):
        columns, a = rng.choice(L, 6, replace=False), c.q_ptr[r]
        for j in columns:
            c.masks[r][:, 0] &= ~(np.uint64(1) << np.uint64(j))
        slot = c.path(r)[1][30 + columns]
        for k, x in ((c.k, float("nan")), (infinite, float("inf"))):
            k[dev(slot // BS), :, dev(slot % BS)] = x
        c.lse[a:a + L] = torch.logsumexp(c.scores(r)[0], -1).permute(2, 0, 1).reshape(L, hq).float()
    for more, n in ((lambda x: {}, rows), (more_entries, 2048 // hkv)):   # few keys (the waves share out the tiles), many
        ones = Case([(36, 60)] * n, hq, hkv, d, seed=1)
        for m in ones.masks:
            m[:] = np.uint64(2**64 - 1)
        theirs, mine = dict(ones.arrays(), **more(ones), max_q=60), dict(c.arrays(), **more(c), max_q=60)
        ones.run(**theirs)
        first = c.run(**mine)
        c.check(first)
        assert torch.equal(c.run(**mine), first)
        ones.run(**theirs)
        assert torch.equal(c.run(k=infinite, **mine), first)


@pytest.mark.gpu
@pytest.mark.parametrize("L,more", [(3, lambda c: {}), (40, lambda c: {}), (40, more_entries)], ids=["few", "split", "many"])
def test_rows_without_tokens_are_left_out(L, more):
    # rows that pause among others: in place their weights stay as they are, elsewhere nothing is written for them
    c = Case([(100, 0), (300, L), (0, 0), (77, 0), (500, L), (40, 0)], 8, 2, 64, seed=L)
    out = c.run(**more(c))
    c.check(out, rows=[1, 4])
    assert torch.all(out[[0, 2, 3, 5]] == 7)
    own = c.before.clone()
    c.run(out=own, before=own, **more(c))
    assert torch.equal(own[[0, 2, 3, 5]], c.before[[0, 2, 3, 5]])
    for r in (1, 4):
        at = dev(c.path(r)[0])
        assert torch.equal(own[r][:, at], out[r][:, at])
    none = Case([(30, 0), (5, 0)], 8, 2, 64)
    assert torch.all(none.run() == 7)


@pytest.mark.gpu
def test_the_same_blocks_twice_and_many_rows():
    c = Case([(100, 4), (200, 4), (50, 2)], 12, 2, 128)
    c.tables[0] = np.concatenate([c.tables[1][:3], c.tables[1][:3], c.tables[0]])
    c.tables[2] = c.tables[0][:-1]
    c.max_blocks = max(len(t) for t in c.tables)
    c.keys = BS * c.max_blocks
    c.k = c.k.nan_to_num(0.0)
    c.before = torch.rand((3, 2, c.keys), device="cuda")
    for r, L in enumerate(c.L):
        a = c.q_ptr[r]
        c.lse[a:a + L] = torch.logsumexp(c.scores(r)[0], -1).permute(2, 0, 1).reshape(L, 12).float()
    c.check(c.run())
    rng = np.random.default_rng(5)
    c = Case([(int(n), int(L)) for n, L in zip(rng.integers(0, 90, 400), rng.integers(1, 6, 400))], 12, 2, 128)
    c.check(c.run(), rows=list(range(0, 400, 23)) + [255, 256, 399])


@pytest.mark.gpu
@pytest.mark.parametrize("L", [2, 20])
def test_tables_of_the_largest_capacity(L):
    # maxima and arrays far above what the rows use (a captured call's capacity): hundreds of rows, empty ones among them
    rng = np.random.default_rng(L)
    c = Case([(int(n), L) for n in rng.integers(0, 200, 300)] + [(5000, L), (0, 1)], 12, 2, 64, extra_keys=16 * 3600)
    spare = torch.zeros(3000, dtype=torch.int32, device="cuda")
    a = c.arrays()
    want = c.run()
    c.check(want, rows=list(range(0, 300, 29)) + [255, 256, 300, 301])
    got = c.run(kv_blocks=torch.cat([a["kv_blocks"], spare]), max_blocks=c.max_blocks + 3600, max_q=64)
    for r in range(302):   # (another cut of the work, and for small drafts the other kernel: other orders of additions)
        x, y = got[r], want[r]
        assert torch.all((x - y).abs() <= 2.0 ** -16 * (1 + y.abs()))
    few = c.run(kv_blocks=torch.cat([a["kv_blocks"], spare]), max_blocks=c.max_blocks + 3600)
    c.check(few, rows=list(range(0, 300, 29)) + [255, 256, 300, 301])


@pytest.mark.gpu
def test_pools_and_weights_past_four_gib():
    hkv, d, nb = 8, 128, 140_000
    c = Case([(200, 5)], 16, hkv, d)
    want = c.run()
    big = torch.zeros((nb, hkv, BS, d), dtype=torch.bfloat16, device="cuda")
    ids = torch.arange(nb - c.nb, nb, device="cuda")
    big[ids] = c.k
    lens = torch.zeros(nb, dtype=torch.int32, device="cuda")
    lens[ids] = dev(c.block_len)
    got = c.run(k=big, block_len=lens, kv_blocks=c.arrays()["kv_blocks"] + (nb - c.nb))
    assert torch.equal(got, want)
    keys = 140_000_000   # 8 heads of 560 MB
    far = torch.full((1, hkv, keys), 7.0, device="cuda")
    c.run(out=far, before=None)
    none = c.run(before=False)
    assert torch.equal(far[:, :, :want.shape[2]], none) and torch.all(far[:, :, want.shape[2]:want.shape[2] + 4096] == 7)


@pytest.mark.gpu
def test_replays_streams_and_dropped_inputs():
    c = Case([(3000, 9), (400, 30), (50, 1)], 12, 2, 128)
    want = c.run()
    a, out = c.arrays(), torch.zeros_like(want)
    q, k, lse = c.q.clone(), c.k.clone(), c.lse.clone()

    def call(stream=None):
        tkv.tkv_key_weights(**a, q=q, k=k, lse=lse, out=out, before=c.before, decay=0.75, coef=c.coef, stream=stream)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    side = torch.cuda.Stream()
    for step in range(3):
        q.copy_(c.q * (step != 1))
        out.fill_(7)
        graph.replay()
        eager = c.run(q=q)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(out, want) == (step != 1)
    for stream in (None, side, side.cuda_stream, 0):
        out.fill_(7)
        torch.cuda.synchronize()
        call(stream)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    kept = dict(a, q=q, k=k, lse=lse, out=out, before=c.before, coef=c.coef)
    for name in ("mask", "q", "k", "lse", "out", "before", "coef"):
        args = dict(kept, **{name: kept[name].clone()})
        torch.cuda.synchronize()
        at = args[name].data_ptr()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        tkv.tkv_key_weights(**args, stream=side)
        del args
        new = torch.empty_like(kept[name])
        busy = not side.query()
        torch.cuda.synchronize()
        assert busy and new.data_ptr() != at, name


@pytest.mark.gpu
def test_tensors_are_checked():
    c = Case([(30, 4)], 8, 2, 64)
    a = c.arrays()
    for name, bad in (("q", c.q.float()), ("k", c.k.transpose(1, 2)), ("lse", c.lse[1:]), ("lse", c.lse.double()), ("mask", a["mask"][1:]),
                      ("kv_indptr", a["kv_indptr"][1:]), ("q_indptr", a["q_indptr"][:0]), ("block_len", a["block_len"].cpu()),
                      ("out", c.before[:, :1]), ("out", c.before.double()), ("before", c.before[..., 1:]), ("coef", c.coef[1:]),
                      ("coef", c.coef.double())):
        with pytest.raises(ValueError):
            c.run(**{name: bad})
    for name, bad in (("max_q", 0), ("max_q", 65), ("max_blocks", 0), ("max_blocks", 1000), ("decay", float("nan")),
                      ("decay", float("inf"))):
        with pytest.raises(tkv.TkvError):
            c.run(**{name: bad})


def test_bad_arguments_are_refused():
    # refused before any device access (no GPU needed)
    L, one = tkv.lib(), 16

    def call(sh=(8, 2, 64, 16, 4), n_rows=1, n_qtok=4, max_q=4, n_kv=9, max_blocks=9, words=1, ptr=one, q=one, lse=one, coef=None,
             before=None, out=one, keys=144, decay=1.0):
        b = tkv.tkv_draft_batch(n_rows, n_qtok, max_q, n_kv, max_blocks, words, ptr, one, one, one, one)
        return L.tkv_key_weights(ctypes.byref(tkv.tkv_shape(*sh)), ctypes.byref(b), q, one, lse, coef, decay, before, out, keys, None)

    for sh in ((8, 2, 96, 16, 4), (8, 2, 64, 32, 4), (0, 2, 64, 16, 4), (8, 3, 64, 16, 4), (130, 2, 64, 16, 4), (8, 2, 64, 16, 0)):
        assert call(sh) == tkv.TKV_EINVAL, sh
    for bad in (dict(n_rows=-1), dict(n_qtok=-1), dict(max_q=0), dict(max_q=1025), dict(max_q=65), dict(n_kv=-1), dict(max_blocks=0),
                dict(words=0), dict(ptr=None), dict(q=None), dict(q=one + 8), dict(lse=None), dict(lse=one + 2), dict(coef=one + 1),
                dict(before=one + 2), dict(out=None), dict(out=one + 2), dict(keys=143), dict(keys=-1), dict(decay=float("nan")),
                dict(decay=float("inf")), dict(max_blocks=1 << 28, keys=1 << 40), dict(before=one + 4), dict(before=one + 2 * 144 * 4 - 4),
                dict(out=one + 4, before=one), dict(n_rows=1 << 30), dict(n_rows=1 << 24),
                dict(n_rows=(1 << 31) - 1, max_blocks=(1 << 27) - 1, keys=1 << 31)):
        assert call(**bad) == tkv.TKV_EINVAL, bad
    assert call(n_rows=0) == tkv.TKV_OK and call(n_qtok=0) == tkv.TKV_OK
    assert L.tkv_key_weights(None, None, one, one, one, None, 1.0, None, one, 1, None) == tkv.TKV_EINVAL
