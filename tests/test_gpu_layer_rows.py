"""Norm and gated activation to int8 rows, against fp64."""
import numpy as np
import pytest
import torch

from layer_util import ACT, LEAST, ROUND
from oracle import layer_oracle as LO

pytestmark = pytest.mark.gpu

# Sums of N squares in fp32, a tree over lanes of at most 32 each: below 64 roundings, and half of that in the root; the factors around
# it, the exponential and the reciprocal add a few (the exponential 2^-24 |g| too, |g| < 32 here)
REL = 2.0 ** -17


def f64(t):
    return t.detach().double().cpu().numpy()


def check_rows(A8, a_scale, y):
    code, scale = A8.cpu().numpy().astype(np.float64), f64(a_scale)
    want = np.array([LO.scale_of(r) for r in y])
    assert np.array_equal(np.isnan(want), np.isnan(scale))
    fine = ~np.isnan(want)
    assert np.all(np.abs(scale[fine] - want[fine]) <= REL * want[fine])
    assert np.abs(code).max(initial=0) <= 127
    # half a step, and what REL of a number of up to 127 steps comes to
    off = np.abs(code[fine] * scale[fine, None] - y[fine]) / scale[fine, None]
    assert off.max(initial=0) <= 0.5 + 2 * 127 * REL


def norm_inputs(seed, M, N, act, extra=0, residual=True):
    r = np.random.default_rng(seed)
    channel = np.exp(r.normal(size=N) * 0.7)

    def rows(std):
        wide = torch.zeros((M, N + extra), dtype=ACT[act])
        wide[:, :N] = torch.from_numpy(r.normal(size=(M, N)) * std * channel).to(ACT[act])
        return wide.cuda()[:, :N]
    return rows(1.0), rows(3.0) if residual else None, torch.from_numpy(1 + 0.2 * r.normal(size=N)).to(ACT[act]).cuda()


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,extra,residual", [
    (1, 512, 0, True), (5, 512, 8, True), (7, 8, 0, True), (1, 4096, 0, False), (3, 5120, 64, True), (2, 8192, 0, True),
    (2, 13824, 0, True), (2, 28672, 0, False), (1, 32776, 0, True),                     # up to and past what stays in registers
    (3, 1, 0, True), (2, 77, 0, True), (2, 1000, 3, True), (1, 40001, 0, False)])       # widths and strides that are no vectors
def test_norm(act, M, N, extra, residual):
    from paper_2504_12984_amd import binding as B
    x, res, w = norm_inputs(M * 7 + N, M, N, act, extra, residual)
    A8, scale, total = B.qg_rmsnorm_a8(x, w, 1e-5, residual=res)
    h, y = LO.norm(f64(x), None if res is None else f64(res), f64(w), 1e-5)
    check_rows(A8, scale, y)
    if residual:
        assert np.all(np.abs(f64(total) - h) <= (ROUND[act] + 2.0 ** -23) * np.abs(h) + LEAST[act])
    else:
        assert total is x


@pytest.mark.parametrize("N", [4096, 1001])
def test_norm_sum_in_place_and_without(N):
    from paper_2504_12984_amd import binding as B
    x, res, w = norm_inputs(3, 4, N, "bf16")
    A8, scale, total = B.qg_rmsnorm_a8(x, w, 1e-6, residual=res)
    inplace = res.clone()
    got = B.qg_rmsnorm_a8(x, w, 1e-6, residual=inplace, sum_out=inplace)
    assert got[2] is inplace and torch.equal(inplace, total) and torch.equal(got[0], A8) and torch.equal(got[1], scale)
    inplace = x.clone()
    got = B.qg_rmsnorm_a8(inplace, w, 1e-6, residual=res, sum_out=inplace)
    assert torch.equal(inplace, total) and torch.equal(got[0], A8)


@pytest.mark.parametrize("N", [512, 4096, 999])
def test_norm_of_zeros_and_of_what_is_not_finite(N):
    from paper_2504_12984_amd import binding as B
    x, _, w = norm_inputs(4, 5, N, "f16", residual=False)
    x[1] = 0
    x[2, N // 2] = float("nan")
    x[3, N - 1] = float("inf")
    A8, scale, _ = B.qg_rmsnorm_a8(x, w, 1e-5)
    assert scale[1].item() == LO.FLOOR and not A8[1].any()
    assert torch.isnan(scale[2:4]).all()
    _, y = LO.norm(f64(x), None, f64(w), 1e-5)
    check_rows(A8[[0, 4]], scale[[0, 4]], y[[0, 4]])


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,fused", [(1, 512, True), (3, 14336, True), (2, 28672, True), (4, 8, False), (1, 33000, True),
                                       (2, 77, True), (3, 1000, False), (1, 1, True)])
def test_gate(act, M, N, fused):
    from paper_2504_12984_amd import binding as B
    r = np.random.default_rng(N)
    gu = torch.from_numpy(r.normal(size=(M, 2 * N)) * 2).to(ACT[act]).cuda()
    g, u = gu[:, :N], gu[:, N:]
    A8, scale = B.qg_silu_a8(gu) if fused else B.qg_silu_a8(g.contiguous(), u)
    check_rows(A8, scale, LO.gate(f64(g), f64(u)))


def test_gate_of_large_and_small_numbers():
    from paper_2504_12984_amd import binding as B
    g = torch.tensor([[-3e4, -100.0, -20.0, 0.0, 20.0, 100.0, 3e4, 1.0]] * 2, dtype=torch.bfloat16).cuda()
    u = torch.ones_like(g)
    u[1] = 0
    A8, scale = B.qg_silu_a8(g, u)
    check_rows(A8[:1], scale[:1], LO.gate(f64(g), f64(u))[:1])
    assert scale[1].item() == LO.FLOOR and not A8[1].any()
    u[0, 3] = float("nan")
    assert torch.isnan(B.qg_silu_a8(g, u)[1][0])


def test_rows_feed_the_int8_product():
    from paper_2504_12984_amd import binding as B
    x, res, w = norm_inputs(9, 5, 512, "f16")
    A8, scale, _ = B.qg_rmsnorm_a8(x, w, 1e-5, residual=res)
    r = np.random.default_rng(1)
    codes = r.integers(0, 16, (512, 128), dtype=np.uint8)
    t = B.WType(B.QG_UINT, 4)
    packed = B.repack(B.qg_pack_codes(torch.from_numpy(codes).cuda(), 4), t, 512, 128, layout=B.QG_LAYOUT_TILE128x64_I8)
    ws = torch.full((4, 128), 0.01, dtype=torch.float16).cuda()
    C = B.qgemm_a8(A8, scale, packed, ws, torch.full((4, 128), 8, dtype=torch.uint8).cuda(), t, 128, 128)
    ref = (f64(A8) * f64(scale)[:, None]) @ ((codes.astype(np.float64) - 8) * f64(ws[0, 0]))
    assert np.all(np.abs(f64(C) - ref) <= 1e-2 + 5e-3 * np.abs(ref))


def test_rows_refuse_what_is_not_theirs():
    from paper_2504_12984_amd import binding as B
    x, res, w = norm_inputs(1, 2, 64, "f16")
    for bad in (lambda: B.qg_rmsnorm_a8(x.float(), w, 1e-5), lambda: B.qg_rmsnorm_a8(x, w.float(), 1e-5),
                lambda: B.qg_rmsnorm_a8(x, w[:32], 1e-5), lambda: B.qg_rmsnorm_a8(x.t(), w, 1e-5),
                lambda: B.qg_rmsnorm_a8(x, w, 1e-5, residual=res[:1]), lambda: B.qg_rmsnorm_a8(x.cpu(), w, 1e-5),
                lambda: B.qg_silu_a8(x[:, :63]), lambda: B.qg_silu_a8(x, res.bfloat16())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.QgError):
        B.qg_rmsnorm_a8(x[:1].expand(4, 64), w, 1e-5)        # rows on top of one another


def test_rows_on_another_stream():
    from paper_2504_12984_amd import binding as B
    x, res, w = norm_inputs(11, 300, 4096, "bf16")
    want = B.qg_rmsnorm_a8(x, w, 1e-5, residual=res)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = B.qg_rmsnorm_a8(x, w, 1e-5, residual=res)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
