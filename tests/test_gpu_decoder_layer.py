"""The operators between a layer's products run together with the products: the example's layer against fp64, and its steps
against one another."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import layer_oracle as LO

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu

HIDDEN, INNER, HEADS, KV, DIM = 512, 1024, 8, 2, 64


@pytest.fixture(scope="module")
def E():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import decoder_layer
    return decoder_layer


def make(E, kv, blocks=6):
    from paper_2504_12984_amd import binding as B
    g = torch.Generator("cuda").manual_seed(3)
    t = B.WType(B.QG_INT, 8) if kv == "i8" else B.WType(B.QG_FLOAT, 8, 4, 3)
    layer = E.Layer(HIDDEN, INNER, HEADS, KV, DIM, blocks, t, g)
    x = torch.randn(150, HIDDEN, generator=g, device="cuda").half()
    return layer, x, torch.tensor([[4, 0, 5]], dtype=torch.int32, device="cuda")


def f64(t):
    return t.double().cpu().numpy()


def weight(w):
    packed, scales, zeros, codes = w
    s = np.repeat(f64(scales), 128, 0)
    return (f64(codes) - 8) * s


def exact(layer, x, cos, sin):
    x = f64(x)
    residual, y = LO.norm(x, np.zeros_like(x), f64(layer.norm1), 1e-5)
    rows = (y @ weight(layer.qkv)).reshape(len(x), -1, DIM)
    pos = np.arange(len(x))
    q, k = (LO.rotate(r, f64(cos), f64(sin), pos, False) for r in (rows[:, :HEADS], rows[:, HEADS:HEADS + KV]))
    a, _, _ = LO.attention(q, k, rows[:, HEADS + KV:], np.ones(len(x), bool), 0, DIM ** -0.5, True, 0)
    residual, y = LO.norm(a.reshape(len(x), -1) @ weight(layer.o), residual, f64(layer.norm2), 1e-5)
    gu = y @ weight(layer.gate_up)
    return residual + LO.gate(gu[:, :INNER], gu[:, INNER:]) @ weight(layer.down)


@pytest.mark.parametrize("kv,most", [
    # Rounding to int8 with a step of amax / 127 leaves rms errors of amax / 127 / sqrt(12), about 0.01 of a row's rms with amax near
    # 4.5 of it: three products' inputs and (with a block's larger amax) keys and values; they add in squares to below 0.03 of what
    # the layer brings, and no output is taken for more than itself.  e4m3: half a step of 2^-4, rms 0.02 to 0.03 for keys and for values.
    ("i8", 0.04), ("e4m3", 0.06)])
def test_layer_against_fp64(E, kv, most):
    layer, x, table = make(E, kv)
    cos, sin = E.tables(150, DIM)
    out = E.run([layer], x, E.sequences([150], [150], table), cos, sin)
    want = exact(layer, x, cos, sin)
    brought = np.linalg.norm(want - f64(x))
    assert np.linalg.norm(f64(out) - want) <= most * brought


@pytest.mark.parametrize("kv", ["i8", "e4m3"])
def test_prompt_in_pieces_and_token_by_token(E, kv):
    """The same tokens as one prompt, in chunks, and the last ones one at a time: the last row's output is the same up to the
    cache's rounding (blocks' scales that grow leave another half step)."""
    cos, sin = E.tables(150, DIM)
    got = []
    for pieces in ([150], [70, 1, 9, 70], [140] + [1] * 10):
        layer, x, table = make(E, kv)
        at = 0
        for n in pieces:
            out = E.run([layer], x[at:at + n], E.sequences([n], [at + n], table), cos, sin)
            at += n
        got.append(f64(out[-1]))
    brought = np.linalg.norm(got[0] - f64(x[-1]))
    for g in got[1:]:
        assert np.linalg.norm(g - got[0]) <= (0.04 if kv == "i8" else 0.06) * brought


def test_several_sequences_do_not_touch_each_other(E):
    cos, sin = E.tables(150, DIM)
    layer, x, _ = make(E, "i8", blocks=9)
    table = torch.tensor([[3, 1], [8, 0], [2, 5]], dtype=torch.int32, device="cuda")
    both = E.run([layer], x[:120], E.sequences([70, 20, 30], [70, 20, 30], table), cos, sin)
    for lo, n, b in ((0, 70, 0), (70, 20, 1), (90, 30, 2)):
        alone = E.run([layer], x[lo:lo + n], E.sequences([n], [n], table[b:b + 1].contiguous()), cos, sin)
        assert (both[lo:lo + n].double() - alone.double()).abs().max() <= 2.0 ** -7 * alone.double().abs().max()
