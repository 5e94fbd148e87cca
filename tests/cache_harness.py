"""Quantised caches for the tests: paged codes and scales with shuffled pages, the
tensors of a batch of tail_harness, and what each row of it sees."""
import numpy as np
import torch

from oracle import cache as oc
from paper_2607_17652_amd import binding as fb
from tail_harness import TORCH, Batch, f64

EPS = 2.0 ** -24


def table(bt, ps, seed, spare=2, reach=0):
    """A page table whose rows cover each request's window, in shuffled pages, and reach
    `reach` keys at least; what it does not need holds a page id out of range."""
    rng = np.random.default_rng(seed)
    w = bt.state["R"] - bt.state["L"]
    need = -(-(bt.o + w * bt.bl) // ps)
    pages = int(need.sum()) + spare
    ids = rng.permutation(pages)
    t = np.full((bt.B, max(int(need.max()) + 1, -(-reach // ps))), pages + 7, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = ids[at:at + n]
        at += n
    return t, pages


class Cache:
    """A cache of `bits` for the batch, filled with codes and scales that are anything
    the format can hold (no NaN), a power of two around 2^spread."""

    def __init__(self, bt, Hq, Hkv, d, ps, bits, dtype, seed=0, spread=0, reach=0):
        rng = np.random.default_rng(seed)
        self.bt, self.bits, self.Hq, self.Hkv, self.d, self.ps = bt, bits, Hq, Hkv, d, ps
        self.dtype = dtype
        self.table, self.pages = table(bt, ps, seed, reach=reach)
        shape = (self.pages, Hkv, ps)
        n = d * bits // 8
        self.host = []
        for _ in "kv":
            codes = rng.integers(0, 256, size=shape + (n,), dtype=np.uint8)
            if bits == 8:                       # codes 127 and 255 are NaN; keep to 15 exponents less
                codes = np.where((codes & 127) > 0x48, codes & 0x87 | 0x40, codes).astype(np.uint8)
            lo = 125 if bits == 4 else 126
            self.host += [codes, (rng.integers(lo - 2, lo + 2, size=shape + (d // 32,)) +
                                  spread).astype(np.uint8)]

    def cuda(self):
        self.dev = [torch.from_numpy(x.copy()).cuda() for x in self.host]
        self.tab = torch.from_numpy(self.table).cuda()
        self.mx = fb.make_mx_cache(self.bits, *self.dev)
        self.shape = fb.make_shape(self.Hq, self.Hkv, self.d, self.dtype, self.ps,
                                   self.table.shape[1], self.pages)
        return self

    def gather(self, b, n, host=None):
        h = self.host if host is None else host
        return tuple(oc.gather(h[i], h[i + 1], self.table[b], n, self.bits) for i in (0, 2))

    def read_back(self):
        return [x.cpu().numpy() for x in self.dev]


def seen(bt):
    """Keys that each live row sees, and its request: arrays over the live rows."""
    pos = np.full(bt.row_cap, -1)
    pos[:len(bt.packed["row_pos"])] = bt.packed["row_pos"]
    b = bt.row_req[bt.live]
    s = (pos[bt.live] - bt.o[b]) // bt.bl
    return bt.o[b] + (s + 1) * bt.bl, b


def status(pack):
    s = fb.fb_pack_read_status(pack)
    return s["code"], s["request"]


__all__ = ["Batch", "Cache", "EPS", "TORCH", "f64", "seen", "status", "table"]
