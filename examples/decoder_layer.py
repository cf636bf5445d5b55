"""Decoder layers with 4-bit weights, int8 activations and an 8-bit paged attention cache.

    python examples/decoder_layer.py [--layers 2] [--hidden 4096] [--inner 14336] [--prompt 1000] [--steps 32] [--batch 4]

Random weights.  Between the matrix products a step of a layer is

    qg_rmsnorm_a8 -> qgemm_a8 (q, k, v) -> qg_kv_append -> qg_kv_attention -> qgemm (o) ->
    qg_rmsnorm_a8 -> qgemm_a8 (gate, up) -> qg_silu_a8 -> qgemm_a8 (down)

Each norm adds what the product before it brought to the residual; activations are int8 wherever one row's
scale is at hand, and 16-bit from the attention to its projection.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2504_12984_amd import binding as B  # noqa: E402

GROUP = 128
U4 = B.WType(B.QG_UINT, 4)


def linear(K, N, generator, a8=True):
    """A random uint4 weight [K, N] with group scales and zero-points: (packed, scales, zeros, codes)."""
    codes = torch.randint(0, 16, (K, N), generator=generator, device="cuda", dtype=torch.uint8)
    scales = ((0.7 + 0.6 * torch.rand(K // GROUP, N, generator=generator, device="cuda")) * (0.22 * K ** -0.5)).half()
    zeros = torch.full((K // GROUP, N), 8, dtype=torch.uint8, device="cuda")
    layout = B.QG_LAYOUT_TILE128x64_I8 if a8 else B.QG_LAYOUT_TILE128x64
    return B.repack(B.qg_pack_codes(codes, 4), U4, K, N, layout=layout), scales, zeros, codes


class Layer:
    def __init__(self, hidden, inner, heads, kv_heads, dim, blocks, kv_type, generator):
        self.heads, self.kv_heads, self.dim, self.N = heads, kv_heads, dim, (heads + 2 * kv_heads) * dim
        self.hidden, self.inner = hidden, inner
        self.norm1, self.norm2 = ((1 + 0.1 * torch.randn(hidden, generator=generator, device="cuda")).half() for _ in range(2))
        self.qkv = linear(hidden, self.N, generator)
        self.o = linear(heads * dim, hidden, generator, a8=False)
        self.gate_up = linear(hidden, 2 * inner, generator)
        self.down = linear(inner, hidden, generator)
        self.cache = B.KvCache.empty(blocks, kv_heads, dim, kv_type)

    def __call__(self, x, residual, seq, cos, sin):
        """x: what the layer before brought to `residual` (updated in place); seq: (row_start, kv_len, table, max_rows, max_kv)."""
        row_start, kv_len, table, max_rows, max_kv = seq

        def product(a8, scale, w, N):
            return B.qgemm_a8(a8, scale, *w[:3], U4, GROUP, N)
        a8, scale, residual = B.qg_rmsnorm_a8(x, self.norm1, 1e-5, residual=residual, sum_out=residual)
        rows = product(a8, scale, self.qkv, self.N).view(x.shape[0], -1, self.dim)
        q, k, v = rows.split((self.heads, self.kv_heads, self.kv_heads), 1)
        q = B.qg_kv_append(k, v, self.cache, row_start, kv_len, table, max_rows, q=q, cos=cos, sin=sin)
        a = B.qg_kv_attention(q, self.cache, row_start, kv_len, table, self.dim ** -0.5, max_rows, max_kv)
        x = B.qgemm(a.view(x.shape[0], -1), *self.o[:3], U4, GROUP, self.hidden)
        a8, scale, residual = B.qg_rmsnorm_a8(x, self.norm2, 1e-5, residual=residual, sum_out=residual)
        a8, scale = B.qg_silu_a8(product(a8, scale, self.gate_up, 2 * self.inner))
        return product(a8, scale, self.down, self.hidden)


def run(layers, x, seq, cos, sin):
    """All layers; the stream's end is residual + what the last one brought."""
    residual = torch.zeros_like(x)
    for layer in layers:
        x = layer(x, residual, seq, cos, sin)
    return residual + x


def tables(positions, dim, base=500000.0):
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * base ** (
        -torch.arange(dim // 2, device="cuda", dtype=torch.float64) / (dim // 2))
    return torch.cos(angle).float(), torch.sin(angle).float()


def sequences(new, length, table):
    """The arrays of a step with new[b] rows that make sequence b length[b] tokens long."""
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    return (torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.tensor(length, dtype=torch.int32, device="cuda"), table,
            max(new), max(length))


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("layers", 2), ("hidden", 4096), ("inner", 14336), ("heads", 32), ("kv_heads", 8), ("dim", 128), ("prompt", 1000),
                        ("steps", 32), ("batch", 4)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--cache", choices=("int8", "e4m3"), default="int8")
    a = ap.parse_args()
    g = torch.Generator("cuda").manual_seed(0)
    kv_type = B.WType(B.QG_INT, 8) if a.cache == "int8" else B.WType(B.QG_FLOAT, 8, 4, 3)
    width = -(-(a.prompt + a.steps) // B.KV_BLOCK)
    layers = [Layer(a.hidden, a.inner, a.heads, a.kv_heads, a.dim, a.batch * width, kv_type, g) for _ in range(a.layers)]
    table = torch.randperm(a.batch * width, generator=g, device="cuda").to(torch.int32).view(a.batch, width)
    cos, sin = tables(a.prompt + a.steps, a.dim)

    def timed(new, length):
        x = torch.randn(sum(new), a.hidden, generator=g, device="cuda").half()
        seq = sequences(new, length, table)
        torch.cuda.synchronize()
        t = time.perf_counter()
        out = run(layers, x, seq, cos, sin)
        torch.cuda.synchronize()
        assert torch.isfinite(out).all()
        return time.perf_counter() - t
    timed([a.prompt] * a.batch, [a.prompt] * a.batch)                       # loads the kernels
    t = timed([a.prompt] * a.batch, [a.prompt] * a.batch)
    print(f"prompts: {a.batch} x {a.prompt} tokens through {a.layers} layers in {t * 1e3:.2f} ms")
    t = [timed([1] * a.batch, [a.prompt + 1 + i] * a.batch) for i in range(a.steps)]
    print(f"single tokens: {a.batch} sequences, {sorted(t)[len(t) // 2] * 1e6 / a.layers:.0f} us a layer and step")


if __name__ == "__main__":
    main()
