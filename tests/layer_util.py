"""Inputs shared by the GPU tests of the operators between a layer's products."""
import numpy as np
import torch

from oracle import layer_oracle as LO

ACT = {"f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}          # half an ulp of the type, relative
LEAST = {"f16": 2.0 ** -25, "bf16": 2.0 ** -133}        # half a step of its smallest numbers


def wtype(kv):
    from paper_2504_12984_amd import binding as B
    return B.WType(B.QG_INT, 8) if kv == "i8" else B.WType(B.QG_FLOAT, 8, 4, 3)


class Sequences:
    """A cache with random content, and sequences laid over it.

    new, length: new rows and tokens (new ones included) of each sequence.  Blocks lie in random order; entries of the table
    past a sequence's end are -1."""

    def __init__(self, seed, new, length, kv_heads, dim, kv, extra=2, missing=(), blocks=None):
        from paper_2504_12984_amd import binding as B
        r = self.rng = np.random.default_rng(seed)
        self.new, self.length, self.H, self.D, self.kv = list(new), list(length), kv_heads, dim, kv
        used = [max(0, -(-n // 64)) for n in length]
        total = sum(used) + extra if blocks is None else blocks
        order = r.permutation(total)
        width = max(max(used), 1) + 1
        table = np.full((len(new), width), -1, np.int32)
        at = 0
        for b, n in enumerate(used):
            table[b, :n] = order[at:at + n]
            at += n
        for b, i in missing:
            table[b, i] = -1 if i % 2 else total
        self.table, self.total = table, total
        codes = r.integers(0, 256, (2, total, kv_heads, 64 * dim), dtype=np.uint8)
        if kv == "i8":
            codes[codes == 0] = 1
        else:
            codes[(codes & 0x7F) == 0x7F] = 0x3A
        self.codes = {"k": codes[0], "v": codes[1]}
        self.scale = {n: np.exp(r.normal(size=(total, kv_heads)) * 0.7 - (5.0 if kv == "i8" else 5.5)).astype(np.float32) for n in "kv"}
        self.start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.rows = int(self.start[-1])
        self.B = B
        self.t = wtype(kv)

    def upload(self):
        d = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        self.cache = self.B.KvCache(d(self.codes["k"]), d(self.codes["v"]), d(self.scale["k"]), d(self.scale["v"]), self.t, self.D)
        self.args = (d(self.start), d(np.array(self.length, np.int32)), d(self.table))
        return self

    def download(self):
        c = self.cache
        return ({"k": c.k.cpu().numpy(), "v": c.v.cpu().numpy()}, {"k": c.k_scale.cpu().numpy(), "v": c.v_scale.cpu().numpy()})

    def values(self, name, b, codes=None, scale=None):
        return LO.sequence_values((codes or self.codes)[name], (scale or self.scale)[name], self.table[b], max(self.length[b], 0), name,
                                  self.kv, self.D)
