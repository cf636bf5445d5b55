"""Pins of the fp64 reference of the operators between a layer's products (CPU)."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as LO


@pytest.mark.parametrize("D", [64, 128])
def test_cache_orders_are_permutations_and_match_their_formulas(D):
    for name in ("k", "v"):
        at = LO.order(name, D)
        assert sorted(at.ravel().tolist()) == list(range(64 * D))
    # hand-worked places
    assert LO.key_byte(0, 17, D) == 256 + 1 and LO.key_byte(1, 0, D) == 16 and LO.key_byte(16, 0, D) == 1024 * (D // 64)
    assert LO.value_byte(0, 1, D) == 16 and LO.value_byte(4, 0, D) == 256 and LO.value_byte(16, 0, D) == 4 and LO.value_byte(0, 16, D) == 1024
    # sixteen neighbouring bytes are one lane's load: one token's dimensions, or one dimension's tokens
    assert len({LO.key_byte(5, d, D) // 16 for d in range(16)}) == 1
    assert len({LO.value_byte(16 * t + 4 + r, 3, D) // 16 for t in range(4) for r in range(4)}) == 1


def test_numbers_of_bytes():
    e4m3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(LO.table("e4m3"), e4m3, equal_nan=True)
    assert LO.table("i8")[[1, 128, 255]].tolist() == [-127.0, 0.0, 127.0]


def test_half_step_bounds_the_nearest_number():
    r = np.random.default_rng(0)
    for kv in ("i8", "e4m3"):
        numbers = LO.table(kv)
        numbers = numbers[np.isfinite(numbers) & (np.abs(numbers) <= LO.QMAX[kv])]
        x = r.uniform(-1, 1, 4000) * LO.QMAX[kv] * 10.0 ** r.uniform(-4, 0, 4000)
        off = np.min(np.abs(x[:, None] - numbers[None, :]), axis=1)
        assert np.all(off <= LO.half_step(x, kv))


def test_scale_rule():
    assert LO.scale_of(np.array([-254.0, 3.0])) == 2.0 and LO.scale_of(np.zeros(4)) == LO.FLOOR
    assert LO.scale_of(np.array([448.0]), "e4m3") == 1.0
    assert np.isnan(LO.scale_of(np.array([np.inf]))) and np.isnan(LO.scale_of(np.array([np.nan, 1.0])))


def test_norm_and_gate_against_torch():
    r = np.random.default_rng(1)
    x, res, w = r.normal(size=(3, 40)), r.normal(size=(3, 40)), r.normal(size=40)
    h, y = LO.norm(x, res, w, 1e-5)
    ref = torch.nn.functional.rms_norm(torch.from_numpy(x + res), (40,), torch.from_numpy(w), 1e-5)
    assert np.allclose(y, ref.numpy(), atol=1e-13) and np.array_equal(h, x + res)
    ref = torch.nn.functional.silu(torch.from_numpy(x)) * torch.from_numpy(res)
    assert np.allclose(LO.gate(x, res), ref.numpy(), atol=1e-13)


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotation_is_a_rotation(neighbours):
    r = np.random.default_rng(2)
    x = r.normal(size=(5, 2, 64))
    angle = r.uniform(0, 6, (9, 16))
    y = LO.rotate(x, np.cos(angle), np.sin(angle), [0, 3, 8, 8, 20], neighbours)
    assert np.allclose(np.linalg.norm(x, axis=-1), np.linalg.norm(y, axis=-1)) and np.array_equal(x[..., 32:], y[..., 32:])
    z = x[..., 0:32:2] + 1j * x[..., 1:32:2] if neighbours else x[..., :16] + 1j * x[..., 16:32]
    z = z * np.exp(1j * angle[[0, 3, 8, 8, 8]])[:, None]
    got = y[..., 0:32:2] + 1j * y[..., 1:32:2] if neighbours else y[..., :16] + 1j * y[..., 16:32]
    assert np.allclose(z, got)


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 3), (False, 4)])
def test_attention_against_torch(causal, window):
    r = np.random.default_rng(3)
    q, k, v = r.normal(size=(4, 6, 64)), r.normal(size=(9, 2, 64)), r.normal(size=(9, 2, 64))
    out, weight, _ = LO.attention(q, k, v, np.ones(9, bool), 5, 0.2, causal, window)
    pos, t = np.arange(5, 9)[:, None], np.arange(9)[None]
    see = np.ones((4, 9), bool)
    if causal:
        see &= t <= pos
    if window:
        see &= t > pos - window
    qt, kt, vt = (torch.from_numpy(np.moveaxis(a, 1, 0).copy()) for a in (q, np.repeat(k, 3, 1), np.repeat(v, 3, 1)))
    ref = torch.nn.functional.scaled_dot_product_attention(qt, kt, vt, attn_mask=torch.from_numpy(see), scale=0.2)
    assert np.allclose(np.moveaxis(out, 1, 0), ref.numpy(), atol=1e-12) and np.all(weight >= np.abs(out) - 1e-12)


def test_attention_rows_that_see_nothing_are_zero():
    r = np.random.default_rng(4)
    q, k = r.normal(size=(3, 2, 64)), r.normal(size=(1, 2, 64))
    out, _, _ = LO.attention(q, k, k, np.ones(1, bool), -2, 1.0, True, 0)         # rows at places -2, -1, 0
    assert np.all(out[:2] == 0) and np.allclose(out[2], k[0])
