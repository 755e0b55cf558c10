"""Rows with block tables, drafted tokens and masks, as the device-side batches take them; and how they are walked on the host."""
import numpy as np
import torch

BS = 16


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def steps(rng, n, most=60):
    """Block lengths of n tokens in steps of up to `most`, each in blocks of its own, the last of them partial."""
    out = []
    while n > 0:
        m = min(n, int(rng.integers(1, most + 1)))
        out += [BS] * ((m - 1) // BS) + [(m - 1) % BS + 1]
        n -= m
    return out


class Rows:
    """Rows (context length, drafted tokens); the draft lies in blocks of its own or continues the last step.  Masks of random
    trees, or random bits."""

    def __init__(self, rows, seed=0, bits=False, extra_words=0, spare=5, full_blocks=False):
        rng = np.random.default_rng([seed, 7])
        self.rng, self.L = rng, [L for _, L in rows]
        lens = []
        for i, (c, L) in enumerate(rows):
            if full_blocks:
                lens.append([BS] * ((c + L) // BS) + ([(c + L) % BS] if (c + L) % BS else []))
            else:
                x = steps(rng, c)
                lens.append(x[:-1] + steps(rng, x[-1] + L, x[-1] + L) if i % 2 and x else x + steps(rng, L, max(L, 1)))
        n = sum(map(len, lens))
        self.nb = n + spare
        ids = rng.permutation(self.nb).astype(np.int32)
        self.spare = ids[n:]
        self.block_len = np.zeros(self.nb, np.int32)
        self.block_len[ids[:n]] = np.concatenate(lens) if n else []
        cut = np.cumsum([0] + [len(x) for x in lens])
        self.tables = [ids[a:b] for a, b in zip(cut[:-1], cut[1:])]
        self.q_ptr = np.cumsum([0] + self.L)
        self.max_q, self.max_blocks = max(self.L + [1]), max([len(t) for t in self.tables] + [1])
        words = -(-self.max_q // 64) + extra_words
        self.masks = []
        for L in self.L:
            m = np.zeros((L, words), np.uint64)
            for i in range(L):
                p = int(rng.integers(max(-1, i - 5), i)) if i else -1
                if p >= 0:
                    m[i] = m[p]
                m[i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
            if bits:
                m = rng.integers(0, 1 << 63, (L, words), dtype=np.uint64) * 2 + rng.integers(0, 2, (L, words), dtype=np.uint64)
            self.masks.append(m)

    def arrays(self):
        """The batch's device arrays and maxima, by the argument names of the entry points."""
        return {"q_indptr": dev(self.q_ptr.astype(np.int32)),
                "kv_indptr": dev(np.cumsum([0] + [len(t) for t in self.tables]).astype(np.int32)),
                "kv_blocks": dev(np.concatenate(self.tables).astype(np.int32)), "block_len": dev(self.block_len),
                "mask": dev(np.concatenate(self.masks).view(np.int64)), "max_q": self.max_q, "max_blocks": self.max_blocks}

    def path(self, r):
        """Row r's keys in order: their places 16 e + s in its table, and their slots in the pool."""
        t = self.tables[r]
        inside = (t >= 0) & (t < self.nb)
        lens = np.where(inside, self.block_len[np.where(inside, t, 0)], 0)
        lens = np.where((lens >= 1) & (lens <= BS), lens, 0)
        at = np.nonzero((np.arange(BS) < lens[:, None]).reshape(-1))[0]
        return at, t[at // BS].astype(np.int64) * BS + at % BS

    def seen(self, r):
        """[L, N]: which of its keys each of row r's tokens sees."""
        N, L = len(self.path(r)[0]), self.L[r]
        s = np.ones((L, N), bool)
        for j in range(L):
            if N - L + j >= 0:
                s[:, N - L + j] = (self.masks[r][:, j // 64] >> np.uint64(j % 64)) & np.uint64(1)
        return s
