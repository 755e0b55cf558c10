"""Eviction from the paged cache: the kept keys, their order, their rows and their weights are decisions and copies, equal to a
plain implementation's."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_39334_amd as tkv
from _rows import BS, Rows, dev


def choose(w, n, sink, recent):
    """Which of a path's keys stay, by their weights w, in path order."""
    N = len(w)
    n = min(N, n)
    first = min(sink, n)
    last = min(recent, n - first)
    middle = np.arange(first, N - last)
    x = np.where(np.isnan(w[middle]), -np.inf, w[middle].astype(np.float64))
    order = np.lexsort((middle, np.isnan(w[middle]), -x))
    return np.sort(np.concatenate((np.arange(first), middle[order[:n - first - last]], np.arange(N - last, N)))).astype(np.int64)


class Case(Rows):
    def __init__(self, lens, hkv, d, budget, sink=4, recent=8, seed=0, extra_keys=0, spread=True, **more):
        super().__init__([(n, 0) for n in lens], seed, spare=sum(-(-min(n, 4096) // BS) for n in lens) + 7 + sum(lens) // 4, **more)
        self.hkv, self.d, self.sink, self.recent = hkv, d, sink, recent
        self.budget = np.broadcast_to(np.asarray(budget, np.int32), (len(lens),)).copy()
        self.most = int(self.budget.max())
        new = [-(-min(len(self.path(r)[0]), int(b)) // BS) for r, b in enumerate(self.budget)]
        cut = np.cumsum([0] + new)
        assert cut[-1] <= len(self.spare)
        self.new = [self.spare[a:b] for a, b in zip(cut[:-1], cut[1:])]
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.k, self.v = (torch.randn((self.nb, hkv, BS, d), generator=g, device="cuda").bfloat16() for _ in "kv")
        self.keys = BS * self.max_blocks + extra_keys
        w = torch.randn((len(lens), hkv, self.keys), generator=g, device="cuda")
        if spread:
            w = torch.exp(3 * w)
        self.weights = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.1, 0.0, w)

    def arrays(self):
        a = super().arrays()
        return {"kv_indptr": a["kv_indptr"], "kv_blocks": a["kv_blocks"], "block_len": a["block_len"], "max_blocks": self.max_blocks,
                "new_indptr": dev(np.cumsum([0] + [len(x) for x in self.new]).astype(np.int32)),
                "new_blocks": dev(np.concatenate(self.new).astype(np.int32)), "budget": dev(self.budget), "sink": self.sink,
                "recent": self.recent}

    def run(self, **other):
        n = len(self.tables)
        args = dict(self.arrays(), weights=self.weights, k=self.k.clone(), v=self.v.clone(), out=torch.full_like(self.weights, 7.0),
                    kept=torch.full((n, self.hkv, self.most), 9, dtype=torch.int32, device="cuda"),
                    n_kept=torch.full((n,), 9, dtype=torch.int32, device="cuda"))
        args.update(other)
        tkv.tkv_evict_keys(**args)
        return {x: args[x] for x in ("kept", "n_kept", "out", "k", "v")}

    def want(self, out_rows=()):
        """What the call leaves behind; out_rows: those that it leaves out."""
        n = len(self.tables)
        old_k, old_v, w = self.k.view(torch.int16).cpu(), self.v.view(torch.int16).cpu(), self.weights.cpu()
        k, v = old_k.clone(), old_v.clone()
        out = torch.full_like(w, 7.0)
        kept = torch.full((n, self.hkv, self.most), -1, dtype=torch.int32)
        n_kept = torch.zeros(n, dtype=torch.int32)
        for r in range(n):
            if r in out_rows:
                n_kept[r] = -1
                continue
            at, slot = self.path(r)
            for h in range(self.hkv):
                pick = choose(w[r, h, at].numpy(), int(self.budget[r]), self.sink, self.recent)
                m = len(pick)
                n_kept[r] = m
                kept[r, h, :m] = torch.from_numpy(at[pick])
                out[r, h, :m] = w[r, h, at[pick]]
                to, src = np.arange(m), slot[pick]
                to = self.new[r][to // BS].astype(np.int64) * BS + to % BS
                for new, old in ((k, old_k), (v, old_v)):
                    new[to // BS, h, to % BS] = old[src // BS, h, src % BS]
        return {"kept": kept, "n_kept": n_kept, "out": out, "k": k, "v": v}

    def check(self, got, **more):
        want = self.want(**more)
        for name in ("n_kept", "kept", "out", "k", "v"):
            x = got[name].view(torch.int16) if name in "kv" else got[name]
            x, y = x.cpu().view(-1), want[name].view(-1)
            same = (x == y) | ((x != x) & (y != y))
            assert bool(same.all()), (name, int((~same).nonzero()[0]))


@pytest.mark.gpu
@pytest.mark.parametrize("hkv,d", [(2, 64), (4, 128), (1, 128), (8, 64), (5, 128)])
@pytest.mark.parametrize("budget", [1, 15, 16, 17, 64, 300, 1000])
def test_paths_of_many_lengths(hkv, d, budget):
    for sink, recent in ((0, 0), (4, 8), (1, 0), (0, 5), (16, 33), (2000, 1), (3, 2000)):
        c = Case([0, 1, 2, 15, 16, 17, 40, 300, 999, 1000, 1001, 2500], hkv, d, budget, sink, recent, seed=budget, extra_keys=3)
        c.check(c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["equal", "zeros", "two values", "negative", "infinite", "not numbers", "close", "one exponent"])
def test_weights_of_every_kind(kind):
    c = Case([700, 33, 1700, 2100], 2, 64, 128, 4, 16, seed=4)
    g = torch.Generator(device="cuda").manual_seed(2)
    r = torch.rand(c.weights.shape, generator=g, device="cuda")
    c.weights = {"equal": lambda: torch.full_like(r, 0.25), "zeros": lambda: torch.where(r < 0.5, 0.0, -0.0),
                 "two values": lambda: torch.where(r < 0.03, 1.0, 0.5), "negative": lambda: -r,
                 "infinite": lambda: torch.where(r < 0.02, float("inf"), torch.where(r > 0.99, -float("inf"), r - 0.5)),
                 "not numbers": lambda: torch.where(r < 0.97, float("nan"), r),
                 "close": lambda: (torch.full_like(r, 1.0).view(torch.int32) + (r * 50).int()).view(torch.float32),
                 "one exponent": lambda: 1 + r}[kind]()
    c.check(c.run())


@pytest.mark.gpu
def test_budgets_of_their_own_and_long_paths():
    c = Case([5000, 60, 3000, 0, 777, 4100], 4, 128, [2048, 16, 0, 5, 4000, 4096], 4, 256, seed=6)
    c.check(c.run())
    c = Case([40000, 3], 2, 64, [700, 2], 4, 100, seed=7)
    c.check(c.run())
    # more blocks than the lengths that are held beside the kernel's counts
    c = Case([300000], 1, 64, [3000], 70, 20000 % 1000, seed=8, full_blocks=True)
    c.check(c.run())
    c = Case([300000], 1, 64, [3000], 3, 2996, seed=9, full_blocks=True)
    c.check(c.run())


@pytest.mark.gpu
def test_many_rows():
    rng = np.random.default_rng(3)
    c = Case([int(x) for x in rng.integers(0, 200, 300)], 2, 64, [int(x) for x in rng.integers(0, 90, 300)], 2, 9, seed=2)
    c.check(c.run())


@pytest.mark.gpu
def test_rows_that_are_left_out():
    c = Case([100, 160, 300, 1500, 90], 2, 64, 48, seed=1)
    a = c.arrays()
    total = a["kv_blocks"].numel()
    kv = a["kv_indptr"].clone()
    kv[-1] = total + 1
    c.check(c.run(kv_indptr=kv, max_blocks=45), out_rows=(3, 4))
    b = a["budget"].clone()
    b[1], b[2] = -1, 49
    c.check(c.run(budget=b), out_rows=(1, 2))
    new = a["new_blocks"].clone()
    new[4], new[8] = c.nb, -1
    c.check(c.run(new_blocks=new), out_rows=(1, 2))
    ptr = a["new_indptr"].clone()
    ptr[1:] -= 1             # the first row's new table is too short, and the others begin one block early
    got = c.run(new_indptr=ptr)
    assert got["n_kept"].tolist()[0] == -1 and torch.all(got["kept"][0] == -1) and torch.all(got["out"][0] == 7)
    for bad in (-3, 1 << 30):
        ptr = a["new_indptr"].clone()
        ptr[0] = bad
        c.check(c.run(new_indptr=ptr), out_rows=(0,))
        kv = a["kv_indptr"].clone()
        kv[0] = bad
        c.check(c.run(kv_indptr=kv), out_rows=(0,))
    # entries that are no blocks, and blocks whose length is none, count as empty
    c.tables[2][3] = c.nb + 1
    c.block_len[c.tables[3][5]] = 20
    c.check(c.run())
    c.budget[:] = 0
    c.new = [x[:0] for x in c.new]
    c.most = 0
    assert c.run()["n_kept"].tolist() == [0] * 5


@pytest.mark.gpu
def test_evicted_paths_are_attended():
    # the new tables serve attention and the next step's weights
    c = Case([900, 70, 2000], 2, 128, 256, 4, 32, seed=3)
    got = c.run()
    block_len = c.block_len.copy()
    n = got["n_kept"].tolist()
    for r in range(3):
        for j, b in enumerate(c.new[r]):
            block_len[b] = min(BS, n[r] - BS * j)
    batch = tkv.DraftBatch(c.new, [[-1]] * 3, block_len)
    q = torch.randn((3, 12, 128), device="cuda").bfloat16()
    o, lse = torch.empty_like(q), torch.empty((3, 12), device="cuda")
    batch.verify(q, got["k"], got["v"], o, lse)
    w = torch.zeros_like(c.weights)
    tkv.tkv_key_weights(batch.q_indptr, batch.kv_indptr, batch.kv_blocks, batch.block_len, batch.mask, 1, batch.max_blocks, q,
                        got["k"], lse, w, before=got["out"])
    for r in range(3):
        at, slot = c.path(r)
        for h in range(12):
            pick = choose(c.weights[r, h // 6].cpu().numpy()[at], 256, 4, 32)
            s = dev(slot[pick])
            keys, vals = (p[s // BS, h // 6, s % BS].double() for p in (c.k, c.v))
            x = keys @ q[r, h].double() / 128 ** 0.5
            p = torch.softmax(x, 0)
            A = p @ vals.abs()
            assert torch.all((o[r, h].double() - p @ vals).abs() <= 2.0 ** -8 * (A + 2 * (p @ vals).abs()) + 2.0 ** -11 * A)
            assert abs(float(lse[r, h]) - float(torch.logsumexp(x, 0))) <= 2.0 ** -11
        total = w[r, :, :n[r]].double().sum(1) - got["out"][r, :, :n[r] - 1].double().sum(1)
        size = w[r, :, :n[r]].double().abs().sum(1)
        assert torch.all((total - 6).abs() <= 2.0 ** -9 * 6 + 2.0 ** -22 * size)


@pytest.mark.gpu
def test_pools_past_four_gib():
    hkv, d, nb = 8, 128, 140_000
    c = Case([500, 64], hkv, d, 100, seed=5)
    want = c.run()
    big = [torch.zeros((nb, hkv, BS, d), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    off = nb - c.nb
    big[0][off:], big[1][off:] = c.k, c.v
    a = c.arrays()
    lens = torch.zeros(nb, dtype=torch.int32, device="cuda")
    lens[off:] = a["block_len"]
    got = c.run(k=big[0], v=big[1], block_len=lens, kv_blocks=a["kv_blocks"] + off, new_blocks=a["new_blocks"] + off)
    assert torch.equal(got["k"][off:], want["k"]) and torch.equal(got["v"][off:], want["v"]) and torch.equal(got["out"], want["out"])
    assert torch.all(got["k"][:off] == 0) and torch.equal(got["kept"], want["kept"])


@pytest.mark.gpu
def test_replays_streams_and_dropped_inputs():
    c = Case([3000, 400, 50], 2, 128, 300, seed=2)
    want = c.run()
    a = c.arrays()
    t = {"weights": c.weights.clone(), "k": c.k.clone(), "v": c.v.clone(), "out": torch.full_like(c.weights, 7.0),
         "kept": torch.zeros_like(want["kept"]), "n_kept": torch.zeros_like(want["n_kept"])}

    def fill(step):
        t["weights"].copy_(c.weights.flip(2) if step == 1 else c.weights)
        t["k"].copy_(c.k), t["v"].copy_(c.v), t["out"].fill_(7)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tkv.tkv_evict_keys(**a, **t)
    side = torch.cuda.Stream()
    for step in range(3):
        fill(step)
        graph.replay()
        eager = c.run(weights=t["weights"])
        torch.cuda.synchronize()
        assert all(torch.equal(t[x], eager[x]) for x in eager)
        assert torch.equal(t["kept"], want["kept"]) == (step != 1)
    for stream in (None, side, side.cuda_stream, 0):
        fill(0)
        torch.cuda.synchronize()
        tkv.tkv_evict_keys(**a, **t, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(t[x], want[x]) for x in want)
    for name in list(t) + ["new_blocks", "budget"]:
        args = dict(a, **t)
        args[name] = args[name].clone()
        torch.cuda.synchronize()
        at, like = args[name].data_ptr(), args[name]
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        tkv.tkv_evict_keys(**args, stream=side)
        shape, dtype = like.shape, like.dtype
        del args, like
        new = torch.empty(shape, dtype=dtype, device="cuda")
        busy = not side.query()
        torch.cuda.synchronize()
        assert busy and new.data_ptr() != at, name


@pytest.mark.gpu
def test_tensors_are_checked():
    c = Case([300, 40], 2, 64, 32)
    a = c.arrays()
    for name, bad in (("k", c.k.float()), ("k", c.k.transpose(1, 2)), ("v", c.v[1:]), ("weights", c.weights[..., 1:]),
                      ("weights", c.weights.double()), ("out", c.weights[:1]), ("kept", torch.zeros(2, 2, 32, device="cuda")),
                      ("kept", torch.zeros(2, 1, 32, dtype=torch.int32, device="cuda")), ("n_kept", a["budget"][1:]),
                      ("budget", a["budget"].long()), ("new_indptr", a["new_indptr"][1:]), ("new_blocks", a["new_blocks"].cpu()),
                      ("kv_indptr", a["kv_indptr"][:0]), ("block_len", a["block_len"][1:])):
        with pytest.raises(ValueError):
            c.run(**{name: bad})
    for name, bad in (("max_blocks", 0), ("max_blocks", c.max_blocks + 1), ("sink", -1), ("recent", -1), ("out", c.weights)):
        with pytest.raises(tkv.TkvError):
            c.run(**{name: bad})


def test_bad_arguments_are_refused():
    # refused before any device access (no GPU needed)
    L, one = tkv.lib(), 16

    def call(sh=(8, 2, 64, 16, 4), n_rows=1, n_kv=9, max_blocks=9, n_new=4, most=64, sink=1, recent=1, ptr=one, new=one, w=one,
             out=1 << 20, keys=144, k=one, kept=one, n_kept=one):
        b = tkv.tkv_evict_batch(n_rows, n_kv, max_blocks, n_new, most, sink, recent, ptr, one, one, one, new, one)
        return L.tkv_evict_keys(ctypes.byref(tkv.tkv_shape(*sh)), ctypes.byref(b), w, out, keys, k, one, kept, n_kept, None)

    for sh in ((8, 2, 96, 16, 4), (8, 2, 64, 32, 4), (8, 0, 64, 16, 4), (8, 2, 64, 16, 0)):
        assert call(sh) == tkv.TKV_EINVAL, sh
    for bad in (dict(n_rows=-1), dict(n_kv=-1), dict(max_blocks=0), dict(n_new=-1), dict(most=-1), dict(sink=-1), dict(recent=-1),
                dict(ptr=None), dict(new=None), dict(w=None), dict(w=one + 2), dict(out=None), dict(out=one), dict(out=one + 2 * 144 * 4 - 4),
                dict(keys=143), dict(k=None), dict(k=one + 8), dict(kept=None), dict(kept=one + 2), dict(n_kept=None),
                dict(max_blocks=1 << 28, keys=1 << 40), dict(n_rows=1 << 22, out=1 << 50), dict(n_rows=1 << 19, most=1 << 20, n_new=1 << 20, out=1 << 50)):
        assert call(**bad) == tkv.TKV_EINVAL, bad
    assert call(n_rows=0) == tkv.TKV_OK
    assert L.tkv_evict_keys(None, None, one, one, 1, one, one, one, one, None) == tkv.TKV_EINVAL
