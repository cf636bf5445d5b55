"""Attention over the paged 8-bit cache, against fp64 on the same codes."""
import numpy as np
import pytest
import torch

from layer_util import ACT, LEAST, ROUND, Sequences

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().double().cpu().numpy()


def queries(S, Hq, act, seed=1, std=1.5, extra=0):
    r = np.random.default_rng(seed)
    x = torch.from_numpy(r.normal(size=(S.rows, Hq + extra, S.D)) * std).to(ACT[act]).cuda()
    return x[:, :Hq]


def check(S, q, out, act, causal, window, scale, heads=None):
    from oracle import layer_oracle as LO
    got = f64(out)
    for b, (n, m) in enumerate(zip(S.new, S.length)):
        if not n:
            continue
        k, there = S.values("k", b)
        v, _ = S.values("v", b)
        lo = S.start[b]
        want, weight, reach = LO.attention(f64(q[lo:lo + n]), k, v, there, m - n, scale, causal, window)
        # scores: D products added in fp32 and a few factors, 2^-24 each of at most `reach`; every probability is off by that (twice:
        # numerator and sum) and by fp16's 2^-11, or 2^-25 of the reference where it is below fp16's normal numbers; the exponential and
        # the sums add less than 2^-12.  Then one rounding.
        rel = 2 * reach * (S.D + 16) * 2.0 ** -24 + 2.0 ** -11 + 2.0 ** -12
        top = np.abs(v).max() if m > 0 else 0.0
        tol = ROUND[act] * np.abs(want) * (1 + rel) + weight * rel + max(m, 0) * 2.0 ** -25 * top + LEAST[act]
        off = np.abs(got[lo:lo + n] - want)
        assert np.all(off <= tol), f"sequence {b}: {np.max(off / tol)} of the tolerance at {np.unravel_index(np.argmax(off / tol), off.shape)}"


CASES = [
    # new rows, lengths, kv heads, query heads, dim, kv, act, causal, window
    ([1], [1], 1, 1, 64, "i8", "f16", True, 0),
    ([1, 1, 1, 1, 1], [63, 64, 65, 1, 300], 2, 8, 128, "i8", "f16", True, 0),
    ([1, 1], [700, 129], 2, 16, 128, "e4m3", "bf16", True, 0),
    ([1, 0, 1], [0, 0, 5], 1, 16, 64, "e4m3", "f16", True, 0),             # a row without tokens, a sequence without rows
    ([1, 1], [1000, 90], 8, 8, 64, "i8", "bf16", True, 100),
    ([2, 5, 1], [200, 5, 64], 2, 10, 128, "i8", "bf16", True, 0),          # several tokens of a sequence, groups of 5
    ([3, 3], [190, 2], 1, 7, 64, "e4m3", "bf16", True, 0),                 # rows before the first token
    ([4], [333], 1, 16, 128, "e4m3", "f16", True, 40),                     # four row tiles
    ([1], [150], 1, 40, 128, "i8", "f16", False, 0),
    ([6], [100], 1, 4, 128, "i8", "bf16", False, 70),
    ([65], [65], 1, 1, 128, "i8", "f16", True, 0),                         # prompts
    ([300], [300], 2, 4, 128, "i8", "bf16", True, 0),
    ([129, 0, 17, 70], [129, 50, 400, 70], 1, 8, 64, "e4m3", "f16", True, 0),
    ([130], [257], 1, 5, 128, "e4m3", "bf16", True, 33),
    ([90, 100], [90, 20], 1, 3, 64, "i8", "bf16", True, 0),                # more rows than tokens
    ([80], [200], 2, 2, 128, "e4m3", "f16", False, 0),
    ([80], [200], 1, 2, 64, "i8", "f16", False, 50),
    ([257], [600], 1, 1, 128, "e4m3", "bf16", True, 128),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_attention(case):
    from paper_2504_12984_amd import binding as B
    new, length, H, Hq, D, kv, act, causal, window = case
    S = Sequences(sum(length) + Hq, new, length, H, D, kv).upload()
    q = queries(S, Hq, act)
    out = B.qg_kv_attention(q, S.cache, *S.args, D ** -0.5, max(new), max(length), causal=causal, window=window)
    check(S, q, out, act, causal, window, D ** -0.5)


@pytest.fixture
def forced():
    from paper_2504_12984_amd import binding as B

    def force(kernel, blocks=0):
        B.qg_set_knob(4, kernel)
        B.qg_set_knob(5, blocks)
    yield force
    force(0)


KERNELS = [1, 2, 3]          # streaming, 128-row tiles, 256-row tiles


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_attention_by_each_kernel(case, kernel, forced):
    from paper_2504_12984_amd import binding as B
    new, length, H, Hq, D, kv, act, causal, window = case
    if kernel == 3 and D == 64:
        pytest.skip("tiles of 256 rows: heads of 128")
    S = Sequences(sum(length) + Hq, new, length, H, D, kv).upload()
    q = queries(S, Hq, act)
    for blocks in (0, 1, 2):                                                # as it comes, and cut into parts of so many
        forced(kernel, blocks)
        out = B.qg_kv_attention(q, S.cache, *S.args, D ** -0.5, max(new), max(length), causal=causal, window=window)
        check(S, q, out, act, causal, window, D ** -0.5)


@pytest.mark.parametrize("kernel", [2, 3])
@pytest.mark.parametrize("kv", ["i8", "e4m3"])
def test_tiled_kernel_where_it_can_go_wrong(kernel, kv, forced):
    """Blocks that are not there, codes past the end that are NaN, a spoilt block, large scores, scales far apart."""
    from paper_2504_12984_amd import binding as B
    from oracle import layer_oracle as LO
    S = Sequences(40, [150, 20], [400, 129], 2, 128, kv, missing=[(0, 1), (0, 4), (1, 0)])
    for i, e in ((0, -4), (2, -34), (3, 0), (5, -14)):
        S.scale["v"][S.table[0, i]] = 2.0 ** e
    if kv == "e4m3":
        for b in (0, 1):
            last = S.table[b, (S.length[b] - 1) // 64]
            for name in "kv":
                S.codes[name][last][:, LO.order(name, 128)[S.length[b] % 64:].ravel()] = 0x7F
    S.upload()
    S.codes = {n: np.where((c & 0x7F) == 0x7F, 0, c) if kv == "e4m3" else c for n, c in S.codes.items()}
    for std in (1.0, 20.0):
        q = queries(S, 6, "bf16", std=std)
        for blocks in (0, 1, 3):
            forced(kernel, blocks)
            check(S, q, B.qg_kv_attention(q, S.cache, *S.args, 0.1, 150, 400), "bf16", True, 0, 0.1)
    S = Sequences(41, [150], [200], 2, 128, kv)
    for name in "kv":
        S.scale[name][S.table[0, 2], 1] = np.nan
        S.upload()
        q = queries(S, 4, "f16")
        for blocks in (0, 1):
            forced(kernel, blocks)
            bad = torch.isnan(B.qg_kv_attention(q, S.cache, *S.args, 0.1, 150, 200, window=30)).all(-1).cpu().numpy()
            pos = 50 + np.arange(150)
            sees = (pos >= 128) & (pos - 30 < 191)
            assert np.array_equal(bad[:, 2:], np.repeat(sees[:, None], 2, 1)) and not bad[:, :2].any()
        S.scale[name][S.table[0, 2], 1] = 0.01


def test_kernels_agree_and_repeat(forced):
    from paper_2504_12984_amd import binding as B
    S = Sequences(42, [300, 5], [900, 700], 2, 128, "i8").upload()
    q = queries(S, 8, "f16")
    got = []
    for kernel in KERNELS:
        for blocks in (0, 2):
            forced(kernel, blocks)
            out = B.qg_kv_attention(q, S.cache, *S.args, 0.09, 300, 900)
            assert torch.equal(out, B.qg_kv_attention(q, S.cache, *S.args, 0.09, 300, 900))
            got.append(out)
    for out in got:
        assert (out.double() - got[0].double()).abs().max() <= 2.0 ** -9 * got[0].double().abs().max()


def test_automatic_choice_of_the_tiled_kernel():
    """Enough rows that tiles are chosen: of 128 (heads of 64) and of 256 rows."""
    from paper_2504_12984_amd import binding as B
    for D, H, Hq, rows in ((64, 8, 8, 2100), (128, 8, 64, 2050)):
        S = Sequences(43, [rows], [rows + 30], H, D, "i8").upload()
        q = queries(S, Hq, "bf16")
        out = B.qg_kv_attention(q, S.cache, *S.args, D ** -0.5, rows, rows + 30)
        k, there = S.values("k", 0)
        v, _ = S.values("v", 0)
        from oracle import layer_oracle as LO
        for j in (0, 1, 63, 64, 1000, rows - 1):
            want, weight, reach = LO.attention(f64(q[j:j + 1]), k, v, there, 30 + j, D ** -0.5, True, 0)
            rel = 2 * reach * (D + 16) * 2.0 ** -24 + 2.0 ** -11 + 2.0 ** -12
            tol = ROUND["bf16"] * np.abs(want) * (1 + rel) + weight * rel + (rows + 30) * 2.0 ** -25 * np.abs(v).max() + LEAST["bf16"]
            assert np.all(np.abs(f64(out[j:j + 1]) - want) <= tol)


def test_a_forced_kernel_that_does_not_exist(forced):
    from paper_2504_12984_amd import binding as B
    S = Sequences(44, [2], [2], 2, 64, "i8").upload()
    q = torch.zeros(2, 4, 64, dtype=torch.float16).cuda()
    for kernel in (3, 4, -1):
        forced(kernel)
        with pytest.raises(B.QgError):
            B.qg_kv_attention(q, S.cache, *S.args, 0.1, 2)


@pytest.mark.parametrize("rows", [1, 3, 40])
@pytest.mark.parametrize("kv", ["i8", "e4m3"])
def test_blocks_that_are_not_there_are_not_seen(rows, kv):
    from paper_2504_12984_amd import binding as B
    S = Sequences(20, [rows, rows], [300, 100], 1, 64, kv, missing=[(0, 0), (0, 1), (0, 3), (1, 0), (1, 1)]).upload()
    q = queries(S, 4, "f16")
    out = B.qg_kv_attention(q, S.cache, *S.args, 0.125, rows, 300)
    check(S, q, out, "f16", True, 0, 0.125)
    assert not out[rows:].any()                                            # the second sequence has none at all


@pytest.mark.parametrize("rows", [1, 100])
def test_what_lies_past_the_end_does_not_matter(rows):
    """Codes past the last token may be NaN, scales of other blocks too."""
    from paper_2504_12984_amd import binding as B
    from oracle import layer_oracle as LO
    S = Sequences(21, [rows], [rows + 69], 2, 128, "e4m3")
    end, last = S.length[0], S.table[0, (S.length[0] - 1) // 64]
    for name in "kv":
        places = LO.order(name, 128)[end % 64:].ravel()
        S.codes[name][last][:, places] = 0x7F
        others = [i for i in range(S.total) if i not in S.table[0]]
        S.scale[name][others] = np.nan
        S.codes[name][others] = 0xFF
    S.upload()
    q = queries(S, 4, "bf16")
    out = B.qg_kv_attention(q, S.cache, *S.args, 0.09, rows, end)
    assert torch.isfinite(out).all()
    S.codes = {n: np.where((c & 0x7F) == 0x7F, 0, c) for n, c in S.codes.items()}
    check(S, q, out, "bf16", True, 0, 0.09)


@pytest.mark.parametrize("rows,window", [(1, 0), (150, 0), (150, 30)])
def test_a_spoilt_block_reaches_those_who_see_it_and_no_others(rows, window):
    from paper_2504_12984_amd import binding as B
    for name in "kv":
        S = Sequences(22, [rows], [200], 2, 64, "i8")
        S.scale[name][S.table[0, 2], 1] = np.nan                           # tokens 128 .. 191 of the second head
        S.upload()
        q = queries(S, 4, "f16")
        out = B.qg_kv_attention(q, S.cache, *S.args, 0.1, rows, 200, window=window)
        bad = torch.isnan(out).all(-1).cpu().numpy()
        assert np.array_equal(bad, torch.isnan(out).any(-1).cpu().numpy())
        pos = 200 - rows + np.arange(rows)
        sees = (pos >= 128) & ((pos - window < 191) if window else True)
        assert np.array_equal(bad[:, 2:], np.repeat(sees[:, None], 2, 1)) and not bad[:, :2].any()


def test_a_spoilt_query_spoils_itself():
    from paper_2504_12984_amd import binding as B
    for rows in (1, 90):
        for act in ("f16", "bf16"):
            S = Sequences(23, [rows], [200], 1, 64, "i8").upload()
            q = queries(S, 3, act)
            want = B.qg_kv_attention(q, S.cache, *S.args, 0.1, rows, 200)
            q2 = q.clone()
            q2[0, 1, 7] = float("nan")
            got = B.qg_kv_attention(q2, S.cache, *S.args, 0.1, rows, 200)
            assert torch.isnan(got[0, 1]).all()
            got[0, 1] = want[0, 1]
            assert torch.equal(got, want)


@pytest.mark.parametrize("act", ["f16", "bf16"])
def test_large_scores_and_wide_ranges(act):
    """One token takes all the weight; scales of neighbouring blocks are 2^30 apart; a block of zeros is among them."""
    from paper_2504_12984_amd import binding as B
    for rows in (1, 70):
        S = Sequences(24, [rows], [400], 1, 128, "i8")
        for i, e in enumerate((0, -30, 0, -40, 0, -10)):
            S.scale["v"][S.table[0, i]] = 2.0 ** e
        S.codes["v"][S.table[0, 3]] = 128
        S.upload()
        q = queries(S, 4, act, std=20.0)
        out = B.qg_kv_attention(q, S.cache, *S.args, 0.1, rows, 400)
        check(S, q, out, act, True, 0, 0.1)
        q = queries(S, 4, act, std=1e-3)
        out = B.qg_kv_attention(q, S.cache, *S.args, 0.1, rows, 400)
        check(S, q, out, act, True, 0, 0.1)


def test_bf16_queries_beyond_fp16():
    from paper_2504_12984_amd import binding as B
    for rows in (1, 70):
        S = Sequences(25, [rows], [130], 1, 64, "i8").upload()
        q = queries(S, 2, "bf16") * 2.0 ** 60
        out = B.qg_kv_attention(q, S.cache, *S.args, 0.125 * 2.0 ** -60, rows, 130)
        check(S, q, out, "bf16", True, 0, 0.125 * 2.0 ** -60)


@pytest.mark.parametrize("std", [1.0, 6.0])
def test_long_histories_in_parts(std):
    """Enough blocks that they are cut among workgroups; the same bits every time, and from a later call."""
    from paper_2504_12984_amd import binding as B
    S = Sequences(26, [1, 1, 2], [9000, 130, 5001], 1, 128, "e4m3").upload()
    q = queries(S, 8, "bf16", std=std)
    first = B.qg_kv_attention(q, S.cache, *S.args, 0.0884, 2, 9000)
    check(S, q, first, "bf16", True, 0, 0.0884)
    for _ in range(3):
        assert torch.equal(first, B.qg_kv_attention(q, S.cache, *S.args, 0.0884, 2, 9000))
    # the call's longest length only decides the cut: wider, unknown and too short ones are served too
    for max_kv in (0, 9100, 700, 64):
        check(S, q, B.qg_kv_attention(q, S.cache, *S.args, 0.0884, 2, max_kv), "bf16", True, 0, 0.0884)
    window = B.qg_kv_attention(q, S.cache, *S.args, 0.0884, 2, 9000, window=2500)
    check(S, q, window, "bf16", True, 2500, 0.0884)


@pytest.mark.parametrize("extra,offset", [(3, 0), (0, 1)])
def test_queries_with_a_stride_and_off_their_alignment(extra, offset):
    from paper_2504_12984_amd import binding as B
    for new, length in (([1, 1], [100, 70]), ([100], [150])):
        S = Sequences(27, new, length, 2, 64, "i8").upload()
        if offset:
            flat = torch.zeros(S.rows * 4 * 64 + 8, dtype=torch.float16).cuda()
            q = flat[offset:offset + S.rows * 256].view(S.rows, 4, 64)
            q.copy_(queries(S, 4, "f16"))
        else:
            q = queries(S, 4, "f16", extra=extra)
        out = B.qg_kv_attention(q, S.cache, *S.args, 0.125, max(new), max(length))
        check(S, q, out, "f16", True, 0, 0.125)


def test_blocks_beyond_32_bits():
    """A cache of more than 4 GiB for the keys alone, sequences in its last blocks."""
    from paper_2504_12984_amd import binding as B
    blocks, H, D = 67000, 8, 128
    cache = B.KvCache.empty(blocks, H, D, B.WType(B.QG_INT, 8))
    S = Sequences(28, [1, 70], [200, 70], H, D, "i8")
    to = torch.arange(blocks - S.total, blocks).cuda()
    small = S.upload().cache
    for a, b in ((cache.k, small.k), (cache.v, small.v), (cache.k_scale, small.k_scale), (cache.v_scale, small.v_scale)):
        a[to] = b
    table = torch.where(S.args[2] >= 0, S.args[2] + (blocks - S.total), -1).to(torch.int32)
    r = np.random.default_rng(5)
    for rows, args in ((1, (S.args[0][:2].contiguous(), S.args[1][:1], table[:1].contiguous())), (70, (S.args[0], S.args[1], table))):
        q = torch.from_numpy(r.normal(size=(71 if rows == 70 else 1, 16, D))).half().cuda()
        k = torch.from_numpy(r.normal(size=(q.shape[0], H, D))).half().cuda()
        small_args = (args[0], args[1], S.args[2][:args[1].shape[0]].contiguous())
        B.qg_kv_append(k, k, cache, *args, rows)
        B.qg_kv_append(k, k, small, *small_args, rows)
        assert torch.equal(B.qg_kv_attention(q, cache, *args, 0.09, rows, 200), B.qg_kv_attention(q, small, *small_args, 0.09, rows, 200))
    used = table[table >= 0].long()
    assert torch.equal(cache.v[used], small.v[used - (blocks - S.total)])


def test_blocks_shared_between_sequences():
    from paper_2504_12984_amd import binding as B
    S = Sequences(29, [1, 1], [200, 190], 1, 64, "e4m3")
    S.table[1, :2] = S.table[0, :2]                                         # a common beginning
    S.upload()
    q = queries(S, 4, "bf16")
    check(S, q, B.qg_kv_attention(q, S.cache, *S.args, 0.125, 1, 200), "bf16", True, 0, 0.125)


def test_append_then_attend_on_another_stream_and_in_a_graph():
    from paper_2504_12984_amd import binding as B
    S = Sequences(30, [1] * 4, [3000, 70, 2, 1500], 2, 128, "i8").upload()
    r = np.random.default_rng(2)
    qkv = torch.from_numpy(r.normal(size=(4, 12, 128))).to(torch.bfloat16).cuda()
    out = torch.empty(4, 8, 128, dtype=torch.bfloat16).cuda()
    q_out = torch.empty_like(out)
    cos, sin = (torch.from_numpy(f(r.uniform(0, 6, (3000, 64)))).float().cuda() for f in (np.cos, np.sin))

    def step():
        B.qg_kv_append(qkv[:, 8:10], qkv[:, 10:], S.cache, *S.args, 1, q=qkv[:, :8], cos=cos, sin=sin, q_out=q_out)
        B.qg_kv_attention(q_out, S.cache, *S.args, 0.0884, 1, 3000, out=out)
    step()
    want = out.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        out.zero_()
        step()                                                              # makes this stream's workspace
        side.synchronize()
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for k in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), k
        step()
        torch.cuda.synchronize()


def test_a_captured_call_without_a_workspace_runs_whole():
    from paper_2504_12984_amd import binding as B
    S = Sequences(31, [1], [4000], 1, 64, "i8").upload()
    q = queries(S, 4, "f16")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.qg_kv_attention(q, S.cache, *S.args, 0.125, 1, 64, out=out)       # one part: loads the kernel, makes no workspace
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.qg_kv_attention(q, S.cache, *S.args, 0.125, 1, 4000, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check(S, q, out, "f16", True, 0, 0.125)


def test_attention_refuses_what_does_not_fit():
    from paper_2504_12984_amd import binding as B
    S = Sequences(32, [2], [2], 2, 64, "i8").upload()
    q = torch.zeros(2, 4, 64, dtype=torch.float16).cuda()
    for bad in (lambda: B.qg_kv_attention(q.float(), S.cache, *S.args, 0.1, 2), lambda: B.qg_kv_attention(q[..., :32], S.cache, *S.args, 0.1, 2),
                lambda: B.qg_kv_attention(q, S.cache, *S.args, 0.1, 2, out=q.bfloat16()), lambda: B.qg_kv_attention(q.cpu(), S.cache, *S.args, 0.1, 2),
                lambda: B.qg_kv_attention(q[:, :, ::2], S.cache, *S.args, 0.1, 2)):
        with pytest.raises(ValueError):
            bad()
    for bad in (dict(scale=0.0), dict(scale=-1.0), dict(window=-5), dict(max_kv=-1)):
        kw = dict(scale=0.1, max_rows=2) | bad
        with pytest.raises(B.QgError):
            B.qg_kv_attention(q, S.cache, *S.args, **kw)
    with pytest.raises(B.QgError):
        B.qg_kv_attention(q[:, :3].contiguous(), S.cache, *S.args, 0.1, 2)  # heads that are no multiple
