"""Attention over the paged 8-bit cache: all tiles of a head cut into equal shares, against fp64 on the same codes."""
import numpy as np
import pytest
import torch

from layer_util import LEAST, ROUND, Sequences
from test_gpu_kv_attention import CASES, check, f64, queries

pytestmark = pytest.mark.gpu


@pytest.fixture
def shares():
    from paper_2504_12984_amd import binding as B

    def force(dim, least):
        B.qg_set_knob(4, 0 if dim is None else 3 if dim == 128 else 2)
        B.qg_set_knob(5, -least)
    yield force
    force(None, 0)


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_shares(case, shares):
    from paper_2504_12984_amd import binding as B
    new, length, H, Hq, D, kv, act, causal, window = case
    S = Sequences(sum(length) + Hq, new, length, H, D, kv).upload()
    q = queries(S, Hq, act)
    for least in (1, 2, 5):
        shares(D, least)
        try:
            out = B.qg_kv_attention(q, S.cache, *S.args, D ** -0.5, max(new), max(length), causal=causal, window=window)
        except B.QgError:
            assert max(length) <= 64 * least                                # nothing that could be shared
            continue
        check(S, q, out, act, causal, window, D ** -0.5)


@pytest.mark.parametrize("dim", [64, 128])
def test_one_tile_in_more_pieces_than_a_wavefront_has_lanes(dim, shares):
    from paper_2504_12984_amd import binding as B
    S = Sequences(50, [70], [5000], 1, dim, "i8").upload()
    q = queries(S, 1, "bf16")
    for least in (1, 3):
        shares(dim, least)
        check(S, q, B.qg_kv_attention(q, S.cache, *S.args, 0.1, 70, 5000), "bf16", True, 0, 0.1)


def test_more_tiles_than_a_wavefront_counts_at_once(shares):
    """Short and long sequences in turn, some without rows: shares of several whole tiles and of parts."""
    from paper_2504_12984_amd import binding as B
    new = [(0, 1, 5, 2, 40)[i % 5] for i in range(150)]
    length = [n + (i * 37) % 300 for i, n in enumerate(new)]
    for dim, kv in ((64, "e4m3"), (128, "i8")):
        S = Sequences(51, new, length, 1, dim, kv).upload()
        q = queries(S, 4, "f16")
        for least in (1, 8, 100):
            shares(dim, least)
            check(S, q, B.qg_kv_attention(q, S.cache, *S.args, 0.1, 40, max(length)), "f16", True, 0, 0.1)


@pytest.mark.parametrize("kv", ["i8", "e4m3"])
def test_where_they_can_go_wrong(kv, shares):
    """Blocks that are not there, large scores, scales far apart."""
    from paper_2504_12984_amd import binding as B
    S = Sequences(52, [150, 20], [400, 129], 2, 128, kv, missing=[(0, 1), (0, 4), (1, 0)])
    for i, e in ((0, -4), (2, -34), (3, 0), (5, -14)):
        S.scale["v"][S.table[0, i]] = 2.0 ** e
    S.upload()
    for std in (1.0, 20.0):
        q = queries(S, 6, "bf16", std=std)
        for least in (1, 3):
            shares(128, least)
            check(S, q, B.qg_kv_attention(q, S.cache, *S.args, 0.1, 150, 400), "bf16", True, 0, 0.1)


def test_they_repeat_also_in_a_graph(shares):
    """The order in which pieces come does not matter, and the counters are left as they were."""
    from paper_2504_12984_amd import binding as B
    S = Sequences(53, [300, 120, 5], [3000, 2700, 900], 2, 128, "i8").upload()
    q = queries(S, 8, "f16")
    out = torch.empty_like(q)

    def step():
        B.qg_kv_attention(q, S.cache, *S.args, 0.09, 300, 3000, out=out)
    step()
    whole = out.clone()
    shares(128, 4)
    step()
    want = out.clone()
    assert (want.double() - whole.double()).abs().max() <= 2.0 ** -9 * whole.double().abs().max()
    for _ in range(20):
        step()
        assert torch.equal(out, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()                                                              # makes this stream's workspace
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for k in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), k
        step()                                                              # eager, in between
        assert torch.equal(out, want), k


@pytest.mark.parametrize("dim", [64, 128])
def test_chosen_where_tiles_fill_the_gpu_once_and_a_bit(dim):
    """Chunks of prompts on long histories: sampled rows."""
    from oracle import layer_oracle as LO
    from paper_2504_12984_amd import binding as B
    S = Sequences(54, [400, 333, 290, 350], [2400, 2333, 2800, 1500], 8, dim, "i8").upload()
    q = queries(S, 64, "bf16")
    out = B.qg_kv_attention(q, S.cache, *S.args, dim ** -0.5, 400, 2800)
    for b, (n, m) in enumerate(zip(S.new, S.length)):
        k, there = S.values("k", b)
        v, _ = S.values("v", b)
        for j in (0, 1, 31, 32, n // 2, n - 1):
            row = int(S.start[b]) + j
            want, weight, reach = LO.attention(f64(q[row:row + 1]), k, v, there, m - n + j, dim ** -0.5, True, 0)
            rel = 2 * reach * (dim + 16) * 2.0 ** -24 + 2.0 ** -11 + 2.0 ** -12
            tol = ROUND["bf16"] * np.abs(want) * (1 + rel) + weight * rel + m * 2.0 ** -25 * np.abs(v).max() + LEAST["bf16"]
            assert np.all(np.abs(f64(out[row:row + 1]) - want) <= tol), (b, j)


def test_refused_where_there_are_none(shares):
    from paper_2504_12984_amd import binding as B
    S = Sequences(55, [40], [900], 1, 64, "i8").upload()
    q = queries(S, 4, "f16")
    shares(128, 2)                                                          # 256-row tiles: heads of 128
    with pytest.raises(B.QgError):
        B.qg_kv_attention(q, S.cache, *S.args, 0.1, 40, 900)
    shares(64, 1000)                                                        # one share would take it all
    with pytest.raises(B.QgError):
        B.qg_kv_attention(q, S.cache, *S.args, 0.1, 40, 900)
