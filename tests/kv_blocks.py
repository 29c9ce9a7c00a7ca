"""Attention over the cache where every block of a sequence's tokens is a channel of the output of its own: values are one at that channel and
zero elsewhere, logits are the block's.  What an output channel holds is its block's share of the weights, so that a run, a wavefront's step or
a last token that is lost, taken twice or given another weight is as large an error as that share, however long the sequence is."""
import numpy as np


class Blocks:
    """lengths: tokens per sequence; H, Hq: heads of the cache, of the queries; dead: share of tokens of size 0; everything that is no
    live token holds NaN.  The last token of a sequence has channel D - 1 to itself, blocks share the others, in another order for every
    sequence and head.  Logits are multiples of 1/16 within +-8 (exact in bf16): one of up to four sets for each query head of a group."""

    def __init__(self, lengths, Hq, H, D, P, dead=0.0, seed=1, width=None):
        rng = np.random.default_rng(seed)
        self.lengths, self.Hq, self.H, self.D, self.P = lengths, Hq, H, D, P
        need = [-(-n // P) for n in lengths]
        self.n_pages = sum(need) + 3
        self.width = max(1, max(need)) if width is None else width
        self.table = np.full((len(lengths), self.width), -1, np.int32)
        order = rng.permutation(self.n_pages).astype(np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.sets = min(4, Hq // H, D)
        self.k = np.full((self.n_pages, H, P, D), np.nan, np.float32)
        self.v = np.full((self.n_pages, H, P, D), np.nan, np.float32)
        self.sizes = rng.integers(-3, 9, (self.n_pages, P)).astype(np.int32)
        self.seqs = []                                      # per sequence: live [n], channel [H, n], logits [H, sets, n]
        for s, n in enumerate(lengths):
            j = np.arange(n)
            live = rng.random(n) >= dead
            if n:
                live[-1] = True
            block = j // max(1, -(-n // max(1, D - 1)))
            channel = (block + (s + np.arange(H))[:, None] * 3) % max(1, D - 1)
            if n:
                channel[:, -1] = D - 1
            z = rng.integers(-128, 129, (H, self.sets, block.max() + 1 if n else 0))[:, :, block] / 16.0
            self.seqs.append((live, channel, z))
            if not n:
                continue
            page, row = self.table[s, j // P], j % P
            self.sizes[page, row] = np.where(live, rng.integers(1, 50, n), -rng.integers(0, 3, n))
            page, row, ch, zz = page[live], row[live], channel[:, live], z[:, :, live]
            self.k[page, :, row] = 0.0
            self.v[page, :, row] = 0.0
            for h in range(H):
                self.v[page, h, row, ch[h]] = 1.0
                for c in range(self.sets):
                    self.k[page, h, row, c] = zz[h, c]
        self.q = np.zeros((len(lengths), Hq, D), np.float32)
        self.q[:, np.arange(Hq), np.arange(Hq) % (Hq // H) % self.sets] = 1.0

    def shares(self, s, times=None):
        """[Hq, D] of sequence s; times [n]: how often each token is taken."""
        live, channel, z = self.seqs[s]
        n, out = len(live), np.zeros((self.Hq, self.D))
        if n == 0:
            return out
        w = np.exp(z) * (live if times is None else live * times)                              # [H, sets, n]
        total = w.sum(axis=2)
        group = self.Hq // self.H
        for h in range(self.H):
            sums = np.stack([np.bincount(channel[h], weights=w[h, c], minlength=self.D) for c in range(self.sets)]) / total[h][:, None]
            out[h * group:(h + 1) * group] = sums[np.arange(group) % self.sets]
        return out

    def want(self):
        return np.stack([self.shares(s) for s in range(len(self.lengths))])

    def relative_tolerance(self, dtype, most):
        """Of an output channel, which is a sum of positive terms over another: half a step of the stored value and what fp32 arithmetic adds
        in front of it, in units of 2^-24, above and below the fraction:
          40   a weight: its argument, up to 24 in powers of two, is rounded once (16 units) behind a scale rounded once (12), exp2 (4)
          20   each time what has been summed is scaled to a higher maximum: once in a step of a run, in the joins of 4 wavefronts, of up to
               16 runs of a group, of up to 48 groups
          1    each addition: 96 in a step of a run in bf16 (three products of 32), 16 in fp32; 3 in a join
        A run has `steps` steps at most: all where runs are as long as a call's tokens may be, else a 256th of the steps of all sequences for each head and
        tile of 16 query heads, up to 21 % and 2 more; beyond 1024 sequences 32, or as many as 768 runs of the longest need, and 2^22 runs in all."""
        step = 64 if dtype == "f32" else 128
        all_steps, total = -(-most // step), sum(-(-n // step) for n in self.lengths)
        parts = self.H * -(-(self.Hq // self.H) // 16)
        if len(self.lengths) > 1024:
            steps = max(32, -(-all_steps // 768), (len(self.lengths) * parts * all_steps >> 22) + 1)
        else:
            steps = all_steps if len(self.lengths) * parts * all_steps <= 512 else 1.21 * (1.0001 * total * parts / 256 + 1) + 2
        steps = min(steps, all_steps)
        units = 2 * (40 + 20 * (steps + 70) + (16 if dtype == "f32" else 96) * steps + 3 * 70)
        return (2.0 ** -24 if dtype == "f32" else 2.0 ** -8) + units * 2.0 ** -24 * 1.01


# lengths, query heads, heads, D, dtype, page, dead, bound on the lengths (0: the longest)
CASES = [
    ([40000, 3000, 100, 0], 4, 1, 64, "bf16", 16, 0.0, 0),          # runs joined in groups, next to sequences of a few runs, of one, of none
    ([30000, 2000, 700], 2, 1, 100, "bf16", 64, 0.3, 0),
    ([20000, 11, 9000], 1, 1, 128, "f32", 32, 0.3, 0),
    ([25000], 19, 1, 24, "bf16", 256, 0.0, 0),                      # two tiles of query heads
    ([100001], 7, 1, 128, "bf16", 64, 0.0, 0),
    ([32768], 2, 2, 256, "f32", 16, 0.0, 40000),
    ([5000, 4999, 1, 333, 5001], 8, 4, 256, "bf16", 128, 0.5, 8192),
    ([600, 3, 0, 599], 800, 800, 8, "bf16", 16, 0.0, 0),            # more heads than runs are cut for: one run to a sequence
    ([700, 3], 300, 300, 20, "f32", 16, 0.2, 2000),                 # two or three
    ([300, 77], 1024, 1024, 16, "bf16", 16, 0.0, 0),                # as many heads as there may be
    # more than 1024 sequences: runs of 32 steps, whatever the lengths
    ([9000] + [1, 0, 3, 40] * 257 + [5000, 4097], 2, 1, 40, "bf16", 16, 0.1, 0),
    ([5, 0, 1] * 342 + [4096, 8193, 12000], 6, 2, 64, "bf16", 64, 0.0, 16384),
    ([70001, 2049, 1] + [1, 2] * 520 + [6000], 1, 1, 20, "f32", 64, 0.0, 0),          # 35 runs: in groups
]
