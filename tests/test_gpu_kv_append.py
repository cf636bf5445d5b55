"""Append to the paged 8-bit cache, against fp64."""
import numpy as np
import pytest
import torch

from layer_util import ACT, LEAST, ROUND, Sequences
from oracle import layer_oracle as LO

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().double().cpu().numpy()


def rows_of(r, rows, heads, D, act, spread=1.0):
    x = r.normal(size=(rows, heads, D)) * np.exp(spread * r.normal(size=(rows, 1, 1)))
    return torch.from_numpy(x).to(ACT[act]).cuda()


def tables(positions, rot):
    angle = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(rot // 2) / max(rot // 2, 1))
    return (torch.from_numpy(f(angle)).float().cuda().contiguous() for f in (np.cos, np.sin))


def check_append(S, k, v, q, q_out, cos, sin, neighbours, before, after, act):
    """What the call left, against what it found."""
    kv, D = S.kv, S.D
    (codes0, scale0), (codes1, scale1) = before, after
    c, s = (None, None) if cos is None else (f64(cos), f64(sin))
    pos = np.concatenate([np.arange(m - n, m) for n, m in zip(S.new, S.length)]) if S.rows else np.zeros(0, int)
    if q is not None:
        want = LO.rotate(f64(q), c, s, pos, neighbours)
        # two products and a sum in fp32 of numbers that are as large as the pair, then one rounding
        size = np.abs(f64(q)).max() * 2
        assert np.all(np.abs(f64(q_out) - want) <= (ROUND[act] + 2.0 ** -22) * np.abs(want) + 2.0 ** -22 * size + LEAST[act])
    new = {"k": LO.rotate(f64(k), c, s, pos, neighbours), "v": f64(v)}
    untouched = {n: np.ones(codes0["k"].shape[:1], bool) for n in "kv"}
    for name in "kv":
        at = 0
        for b, (n, m) in enumerate(zip(S.new, S.length)):
            first = m - n
            for blk in range(max(first, 0) // 64, -(-m // 64) if n else 0):
                ident = S.table[b, blk]
                if not 0 <= ident < S.total:
                    continue
                untouched[name][ident] = False
                lo, hi = max(first, 0, blk * 64), min(m, blk * 64 + 64)
                mine = new[name][at + lo - first:at + hi - first]                      # [tokens, heads, D]
                kept = lo - blk * 64
                old = LO.block_values(codes0[name][ident], scale0[name][ident], name, kv, D)[:kept]
                got = LO.block_values(codes1[name][ident], scale1[name][ident], name, kv, D)
                for h in range(S.H):
                    want = LO.scale_of(mine[:, h], kv)
                    was, now = float(scale0[name][ident, h]), float(scale1[name][ident, h])
                    if kept and not want * (1 - 2.0 ** -20) > was:
                        assert now == was or abs(now - want) <= 2.0 ** -20 * want
                    else:
                        assert abs(now - want) <= 2.0 ** -20 * want
                    # the new tokens: half a step (and fp32's error of a number of QMAX steps, twice)
                    steps = mine[:, h] / now
                    off = np.abs(got[kept:kept + hi - lo, h] / now - steps)
                    assert np.all(off <= LO.half_step(steps, kv) + 2.0 ** -20 * LO.QMAX[kv])
                    # those that were there: the same bytes while the scale stays, else half a step of the new scale
                    if kept and now == was:
                        assert np.array_equal(codes0[name][ident, h][LO.order(name, D)][:kept], codes1[name][ident, h][LO.order(name, D)][:kept])
                    elif kept:
                        steps = old[:, h] / now
                        assert np.all(np.abs(got[:kept, h] / now - steps) <= LO.half_step(steps, kv) + 2.0 ** -20 * LO.QMAX[kv])
            at += n
        assert np.array_equal(codes0[name][untouched[name]], codes1[name][untouched[name]])
        assert np.array_equal(scale0[name][untouched[name]], scale1[name][untouched[name]])


CASES = [
    # new rows, lengths, kv heads, query heads, dim, kv, act, rot, neighbours
    ([1, 1, 1], [1, 64, 130], 2, 4, 128, "i8", "f16", 128, False),
    ([1, 1, 1, 1], [65, 3, 200, 64], 1, 8, 64, "e4m3", "bf16", 64, True),
    ([1], [33], 8, 8, 128, "e4m3", "f16", 0, False),
    ([5, 0, 70, 64, 1], [5, 12, 100, 128, 257], 2, 2, 128, "i8", "bf16", 64, False),
    ([200, 3], [300, 3], 3, 15, 64, "i8", "f16", 32, True),
    ([64, 128, 63, 65], [64, 128, 63, 65], 1, 1, 128, "e4m3", "bf16", 128, True),
    ([7, 90], [70, 91], 2, 4, 64, "e4m3", "f16", 22, False),           # pairs that are no vectors
    ([7, 90], [70, 91], 2, 4, 128, "i8", "bf16", 10, True),
    ([4], [2], 1, 2, 64, "i8", "f16", 64, False),                       # more rows than tokens: the first two are nowhere
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("fused", [True, False])
def test_append(case, fused):
    from paper_2504_12984_amd import binding as B
    new, length, H, Hq, D, kv, act, rot, neighbours = case
    S = Sequences(sum(length) + H, new, length, H, D, kv).upload()
    r = np.random.default_rng(17)
    if fused:                                    # as a fused projection leaves them
        qkv = rows_of(r, S.rows, Hq + 2 * H, D, act)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    else:
        q, k, v = (rows_of(r, S.rows, n, D, act) for n in (Hq, H, H))
    cos, sin = tables(max(length) + 3, rot) if rot else (None, None)
    before = S.download()
    out = B.qg_kv_append(k, v, S.cache, *S.args, max(new), q=q, cos=cos, sin=sin, neighbours=neighbours)
    torch.cuda.synchronize()
    if min(m - n for n, m in zip(new, length)) >= 0:
        check_append(S, k, v, q, out, cos, sin, neighbours, before, S.download(), act)
    else:
        codes, scale = S.download()
        got = LO.block_values(codes["v"][S.table[0, 0]], scale["v"][S.table[0, 0]], "v", kv, D)[:2]
        assert np.all(np.abs(got - f64(v)[2:]) <= scale["v"][S.table[0, 0]][None, :, None] * 0.5001)


def test_append_token_by_token_keeps_within_the_growing_scale():
    """Token after token into one block: each later scale adds at most half a step of itself."""
    from paper_2504_12984_amd import binding as B
    for kv in ("i8", "e4m3"):
        S = Sequences(5, [1], [64], 2, 64, kv).upload()
        r = np.random.default_rng(3)
        k, v = rows_of(r, 64, 2, 64, "f16"), rows_of(r, 64, 2, 64, "f16")
        budget, last = np.zeros((64, 2)), None
        for n in range(1, 65):
            args = (S.args[0], torch.tensor([n], dtype=torch.int32).cuda(), S.args[2])
            B.qg_kv_append(k[n - 1:n], v[n - 1:n], S.cache, *args, 1)
            now = S.cache.v_scale[int(S.table[0, 0])].double().cpu().numpy()
            grew = np.ones(2, bool) if last is None else now != last
            assert last is None or np.all(now >= last)
            budget[:n - 1][:, grew] += 0.501 * now[grew] if kv == "i8" else 0.0
            budget[n - 1] = 0.501 * now
            last = now
        got = B.qg_kv_dequant(S.cache, torch.tensor([0, 64], dtype=torch.int32).cuda(), torch.tensor([64], dtype=torch.int32).cuda(),
                              S.args[2], 64, torch.float16)[1]
        off = np.abs(f64(got) - f64(v)).max(-1)
        if kv == "i8":
            assert np.all(off <= budget + 2.0 ** -11 * np.abs(f64(v)).max(-1))
        else:                                    # a power of two apart from re-coding: relative steps add up, few times
            assert np.all(off <= 0.5 * np.abs(f64(v)).max(-1))


def test_append_at_once_equals_the_scale_of_all():
    from paper_2504_12984_amd import binding as B
    S = Sequences(6, [64], [64], 2, 128, "i8").upload()
    r = np.random.default_rng(4)
    k, v = rows_of(r, 64, 2, 128, "bf16"), rows_of(r, 64, 2, 128, "bf16")
    B.qg_kv_append(k, v, S.cache, *S.args, 64)
    at = int(S.table[0, 0])
    assert torch.equal(S.cache.v_scale[at].cpu(), (v.float().abs().amax((0, 2)) / 127).cpu())
    assert torch.equal(S.cache.k_scale[at].cpu(), (k.float().abs().amax((0, 2)) / 127).cpu())


def test_append_twice_is_appending_once():
    from paper_2504_12984_amd import binding as B
    S = Sequences(7, [10, 40], [75, 40], 2, 64, "e4m3").upload()
    r = np.random.default_rng(5)
    k, v = rows_of(r, 50, 2, 64, "bf16"), rows_of(r, 50, 2, 64, "bf16")
    B.qg_kv_append(k, v, S.cache, *S.args, 40)
    first = S.download()
    B.qg_kv_append(k, v, S.cache, *S.args, 40)
    again = S.download()
    for a, b in zip(first, again):
        assert all(np.array_equal(a[n], b[n]) for n in "kv")


def test_append_of_zeros_and_of_what_is_not_finite():
    from paper_2504_12984_amd import binding as B
    for kv in ("i8", "e4m3"):
        S = Sequences(8, [2, 2, 2], [2, 2, 40], 2, 64, kv).upload()
        k, v = (torch.zeros(6, 2, 64, dtype=torch.float16).cuda() for _ in range(2))
        v[2, 0, 5], v[4, 1, 6] = float("inf"), float("nan")
        was = S.cache.v_scale[int(S.table[2, 0]), 0].item()
        B.qg_kv_append(k, v, S.cache, *S.args, 2)
        at = [int(S.table[b, 0]) for b in range(3)]
        assert (S.cache.v_scale[at[0]] == LO.FLOOR).all() and (S.cache.k_scale[at[0]] == LO.FLOOR).all()
        assert torch.isnan(S.cache.v_scale[at[1], 0]) and S.cache.v_scale[at[1], 1].item() == LO.FLOOR
        assert torch.isnan(S.cache.v_scale[at[2], 1]) and S.cache.v_scale[at[2], 0].item() == was
        if kv == "e4m3":                                            # no code is NaN, whatever the input
            assert not ((S.cache.v[at] & 0x7F) == 0x7F)[:2].any()
        B.qg_kv_append(torch.ones_like(k), torch.ones_like(v), S.cache, *S.args, 2)
        assert torch.isnan(S.cache.v_scale[at[2], 1])                # what was there stays spoilt
        assert torch.isfinite(S.cache.v_scale[at[1]]).all()          # a block that is begun again is not


def test_append_without_blocks_and_past_the_table():
    """Entries outside the cache, and tokens past the table's width, are dropped."""
    from paper_2504_12984_amd import binding as B
    S = Sequences(9, [130, 70], [130, 70], 1, 64, "i8", missing=[(0, 1), (1, 0)]).upload()
    r = np.random.default_rng(6)
    k, v = rows_of(r, 200, 1, 64, "f16"), rows_of(r, 200, 1, 64, "f16")
    before = S.download()
    B.qg_kv_append(k, v, S.cache, *S.args, 130)
    check_append(S, k, v, None, None, None, None, False, before, S.download(), "f16")
    narrow = (S.args[0], S.args[1], S.args[2][:, :1].contiguous())
    S2 = Sequences(9, [130, 70], [130, 70], 1, 64, "i8").upload()
    before = S2.download()
    B.qg_kv_append(k, v, S2.cache, narrow[0], narrow[1], S2.args[2][:, :1].contiguous(), 130)
    after = S2.download()
    beyond = [int(x) for x in S2.table[:, 1:].ravel() if x >= 0]
    assert all(np.array_equal(before[0][n][beyond], after[0][n][beyond]) for n in "kv")


def test_append_many_sequences():
    """More sequences than a wavefront has lanes, some without rows."""
    from paper_2504_12984_amd import binding as B
    r = np.random.default_rng(10)
    new = [int(x) for x in r.integers(0, 4, 150)]
    new[17] = 100
    length = [n + int(x) for n, x in zip(new, r.integers(0, 150, 150))]
    S = Sequences(10, new, length, 1, 64, "i8").upload()
    q, k, v = rows_of(r, S.rows, 2, 64, "bf16"), rows_of(r, S.rows, 1, 64, "bf16"), rows_of(r, S.rows, 1, 64, "bf16")
    cos, sin = tables(max(length), 64)
    before = S.download()
    out = B.qg_kv_append(k, v, S.cache, *S.args, 100, q=q, cos=cos, sin=sin)
    check_append(S, k, v, q, out, cos, sin, False, before, S.download(), "bf16")


def test_append_q_in_place():
    from paper_2504_12984_amd import binding as B
    for neighbours, rot in ((False, 128), (True, 128), (False, 22)):
        S = Sequences(11, [9], [30], 1, 128, "i8").upload()
        r = np.random.default_rng(7)
        q, k = rows_of(r, 9, 5, 128, "f16"), rows_of(r, 9, 1, 128, "f16")
        cos, sin = tables(40, rot)
        want = B.qg_kv_append(k, k, S.cache, *S.args, 9, q=q, cos=cos, sin=sin, neighbours=neighbours)
        got = B.qg_kv_append(k, k, S.cache, *S.args, 9, q=q, cos=cos, sin=sin, neighbours=neighbours, q_out=q)
        assert got is q and torch.equal(q, want)


@pytest.mark.parametrize("D,kv,act", [(64, "i8", "f16"), (128, "e4m3", "bf16"), (128, "i8", "bf16"), (64, "e4m3", "f16")])
def test_dequant(D, kv, act):
    from paper_2504_12984_amd import binding as B
    new = [3, 0, 100, 64]
    S = Sequences(12, new, [70, 5, 100, 200], 2, D, kv, missing=[(2, 1)]).upload()
    k, v = B.qg_kv_dequant(S.cache, *S.args, S.rows, ACT[act])
    for name, got in (("k", k), ("v", v)):
        want = np.concatenate([S.values(name, b)[0][m - n:m] for b, (n, m) in enumerate(zip(new, S.length))])
        assert np.all(np.abs(f64(got) - want) <= (ROUND[act] + 2.0 ** -23) * np.abs(want) + LEAST[act])


def test_append_refuses_what_does_not_fit():
    from paper_2504_12984_amd import binding as B
    S = Sequences(13, [2], [2], 2, 64, "i8").upload()
    k = torch.zeros(2, 2, 64, dtype=torch.float16).cuda()
    cos = torch.zeros(8, 32).cuda()
    for bad in (lambda: B.qg_kv_append(k.float(), k, S.cache, *S.args, 2), lambda: B.qg_kv_append(k, k[:, :1], S.cache, *S.args, 2),
                lambda: B.qg_kv_append(k, k.bfloat16(), S.cache, *S.args, 2), lambda: B.qg_kv_append(k, k[..., :32], S.cache, *S.args, 2),
                lambda: B.qg_kv_append(k, k, S.cache, *S.args, 2, cos=cos), lambda: B.qg_kv_append(k, k, S.cache, *S.args, 2, cos=cos, sin=cos.half()),
                lambda: B.qg_kv_append(k, k, S.cache, S.args[0].long(), *S.args[1:], 2),
                lambda: B.qg_kv_append(k, k, S.cache, S.args[0][:1], *S.args[1:], 2),
                lambda: B.KvCache(S.cache.k, S.cache.v, S.cache.k_scale.half(), S.cache.v_scale, S.t, 64),
                lambda: B.KvCache(S.cache.k, S.cache.v, S.cache.k_scale, S.cache.v_scale, S.t, 128)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.QgError):
        B.qg_kv_append(k, k, S.cache, *S.args, 2, cos=torch.zeros(8, 33).cuda(), sin=torch.zeros(8, 33).cuda())
