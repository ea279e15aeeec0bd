"""Small caches for the tests of the cache operators: numpy arrays for the
oracle, the same bytes on the device for the kernels."""
import numpy as np
import torch

from oracle import cache as oc

NAN = 0x7F  # the e4m3 code of NaN


class Case:
    """B sequences of `lengths` tokens, pages scattered over the pool. Rows
    behind a sequence's last token, and pages of no sequence, hold NaN."""

    def __init__(self, lengths, H=4, hkv=2, d=64, ps=16, dtype="bf16",
                 spare=2, seed=0, spread=1.0, extra_pages=3, k_size=1.0):
        g = np.random.default_rng(seed)
        self.rng = g
        self.B, self.H, self.hkv, self.d, self.ps = len(lengths), H, hkv, d, ps
        self.dtype = dtype
        used = [-(-n // ps) for n in lengths]
        self.max_pages = max(max(used), 1) + spare
        num = sum(used) + extra_pages
        place = g.permutation(num)
        self.free = place[sum(used):]
        table = np.full((self.B, self.max_pages), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(used):
            table[b, :n] = place[at:at + n]
            at += n
        shape = (num, hkv, ps, d)
        self.c = c = dict(
            k=np.full(shape, NAN, np.uint8), v=np.full(shape, NAN, np.uint8),
            k_scale=np.full((num, hkv), np.nan, np.float32),
            v_scale=np.full((num, hkv), np.nan, np.float32),
            bounds=np.zeros((num, hkv, 2, d), np.int8), table=table,
            lengths=np.array(lengths, np.int32))
        for b, n in enumerate(lengths):
            for p in range(used[b]):
                rows = min(ps, n - p * ps)
                i = table[b, p]
                for x in "kv":
                    val = g.standard_normal((hkv, rows, d)) * np.exp(
                        spread * g.standard_normal((hkv, 1, 1)))
                    if x == "k":
                        val = val * k_size
                    for h in range(hkv):
                        e = oc._page(val[h])
                        c[x][i, h, :rows] = oc.encode(val[h] / 2.0 ** e)
                        c[x + "_scale"][i, h] = 2.0 ** e
                        if x == "k":
                            hi, lo = oc._extremes(c["k"][i, h, :rows])
                            c["bounds"][i, h] = np.stack([hi, lo])

    def rows(self, heads, T, size=1.0):
        """Random rows [B, heads, T, d] that the type holds: (numpy float64,
        device tensor)."""
        x = torch.tensor(self.rng.standard_normal((self.B, heads, T, self.d))
                         * size, dtype=torch.float32)
        if self.dtype == "bf16":
            x = x.to(torch.bfloat16)
        return x.double().numpy(), x.cuda()

    def device(self, E, impl=0, **over):
        """The cache on the device (its tensors under `.tensors`)."""
        t = {x: torch.tensor(self.c[x]).cuda() for x in self.c}
        return E.make_cache(t["k"], t["v"], t["k_scale"], t["v_scale"],
                            t["bounds"], t["table"], t["lengths"], H=self.H,
                            dtype=self.dtype, impl=impl, **over)

    def same_bytes(self, cache):
        """The device's pages hold what the oracle's arrays hold, byte for
        byte (-0 counts as 0)."""
        bad = []
        for x in ("k", "v", "k_scale", "v_scale", "bounds"):
            a = cache.tensors[x].cpu()
            a = a.view(torch.uint8).numpy() if x in "kv" else a.numpy()
            b = self.c[x]
            if x in "kv":
                a, b = oc.E4M3[a], oc.E4M3[b]
            if not np.array_equal(a, b, equal_nan=x != "bounds"):
                bad.append(x)
        return bad


def int_tensor(x):
    return torch.tensor(x, dtype=torch.int32).cuda()
