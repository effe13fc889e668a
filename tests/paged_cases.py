"""Seeded sequences in pages for the tests of the paged cache."""
import numpy as np

from paper_2607_28144_amd import synth
from oracle import dit as odit


class Case:
    """A pool full of NaN but for the places of the sequences, whose pages lie in any order; packed queries."""

    def __init__(self, rows, lens, H, heads, D, page, seed=0, lead=0, tail=0, spare=2, sharp=1.0, stale=np.nan):
        rng = np.random.default_rng(seed)
        self.rows, self.lens = np.array(rows, np.int32), np.array(lens, np.int32)
        self.first = (lead + np.concatenate([[0], np.cumsum(rows)])).astype(np.int32)
        self.T = int(self.first[-1]) + tail
        self.H, self.heads, self.D, self.page, self.B = H, heads, D, page, len(rows)
        need = [-(-max(int(n), 0) // page) for n in lens]
        pages = sum(need) + spare
        order = rng.permutation(pages)
        # columns of no sequence name no page
        self.table = np.full((self.B, max(need + [1]) + 1), -1, np.int32)
        self.q = synth.normal_bf16(rng, (self.T, H, D), sharp)
        k, v = (synth.normal_bf16(rng, (pages, heads, page, D)) for _ in range(2))
        nan = np.uint16(0x7fc0) if np.isnan(stale) else (np.float32(stale).view(np.uint32) >> 16).astype(np.uint16)
        keep = np.zeros((pages, page), bool)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            for c in range(n):
                keep[order[at + c], :max(0, min(page, int(lens[b]) - c * page))] = True
            at += n
        self.keep = keep
        mask = keep[:, None, :, None]
        self.k, self.v = np.where(mask, k, nan).astype(np.uint16), np.where(mask, v, nan).astype(np.uint16)

    def wide(self):
        """q, k, v as float64."""
        return [odit.widen(x).astype(np.float64) for x in (self.q, self.k, self.v)]
