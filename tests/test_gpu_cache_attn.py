"""GPU: attention over the 8-bit cache against softmax attention in 64 bits over the values that its codes stand for."""
import numpy as np
import pytest
import torch

from tests import serve_testlib as sl

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, usp, seed, lens, news, hq, hk, hs, page, causal=True, o_dtype=sl.BF16, drop=0.0, strided=False, tail=0, wide=False):
        rng = np.random.default_rng(seed)
        self.usp, self.hq, self.page, self.causal, self.o_dtype = usp, hq, page, causal, o_dtype
        self.lens, self.cu = np.asarray(lens), np.concatenate([[0], np.cumsum(news)])
        pages = sum(-(-max(x, 0) // page) for x in lens) + 2
        self.cache = sl.Cache(usp, rng, pages, page, hk, hs)
        self.table = sl.ragged_table(rng, [max(x, 0) for x in lens], page, pages, max(1, max(-(-max(x, 0) // page) for x in lens)))
        if wide:        # room for more than 4096 tokens: units are cut between workgroups
            more = np.full((len(lens), 4096 // page + 1), 0x7fffff02, dtype=np.int32)
            self.table = np.concatenate([self.table, more], 1)
        if drop:
            self.table[rng.random(self.table.shape) < drop] = -1
        self.total = int(self.cu[-1]) + tail
        q = torch.from_numpy(rng.standard_normal((self.total, hq, hs))).bfloat16().cuda()
        if strided:
            wide = torch.zeros(self.total, hq + 5, hs, dtype=q.dtype, device="cuda")
            wide[:, :hq] = q
            q = wide[:, :hq]
        self.q = q

    def run(self, max_q=None, workspace=None, scale=0.0, table=None):
        hs, n = self.cache.hs, len(self.lens)
        table = sl.ints(self.table) if table is None else table
        o = torch.full((self.total, self.hq, hs), 7.0, dtype=sl.torch_dtype(self.o_dtype), device="cuda")
        lse = torch.full((self.hq, self.total), 7.0, device="cuda")
        max_q = int(np.diff(self.cu).max()) if max_q is None else max_q
        ws = workspace
        if ws is None:      # what stood in it before must not matter
            ws = torch.full((self.usp.usp_cache_attn_workspace_bytes(self.cache.c, self.hq, max_q),), 0xff, dtype=torch.uint8, device="cuda")
        self.usp.usp_cache_attn(self.cache.c, self.q, self.q.stride(0), sl.ints(self.cu), sl.ints(self.lens), table, table.shape[1],
                                n, self.total, max_q, self.hq, scale, self.causal, o, lse, self.o_dtype, ws)
        return o, lse

    def reference(self, scale=None):
        k, v = self.cache.values()
        return sl.attention(sl.f64(self.q), k, v, self.cu, self.lens, self.table, self.page, self.cache.pages, self.causal, scale)

    def check(self, **kw):
        o, lse = self.run(**kw)
        ref = self.reference()
        sl.check_attention(sl.f64(o), sl.f64(lse), ref, self.o_dtype)
        assert bool((o[~torch.from_numpy(ref[3])] == 7.0).all()) and bool((lse[:, ~torch.from_numpy(ref[3])] == 7.0).all())
        return o, lse


HEADS = [(32, 8), (4, 4), (8, 1), (6, 2), (71, 1)]


@pytest.mark.parametrize("hs,page", [(128, 64), (128, 16), (64, 32), (64, 128)])
@pytest.mark.parametrize("hq,hk", HEADS)
@pytest.mark.parametrize("wide", [False, True])
def test_single_tokens(usp, hs, page, hq, hk, wide):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 500, 1003, 0]
    Case(usp, hq + hs + page, lens, [1] * len(lens), hq, hk, hs, page, wide=wide).check()


@pytest.mark.parametrize("steps", [1, 2, 3, 5, 8, 13, 40, 300, 700])
@pytest.mark.parametrize("wide", [False, True])
def test_one_unit_cut_among_waves_and_workgroups(usp, steps, wide):
    """One KV head and few steps or many: shares of none, one and several steps to a wave, with whole units between cut ones."""
    if wide or steps <= 64:
        Case(usp, steps, [64 * steps - 5], [1], 4, 1, 128, 64, wide=wide).check()
    lens = [64 * steps, 1, 100, 64 * steps - 63, 64, 65]
    if wide or steps <= 64:
        Case(usp, steps + 1, lens, [1, 1, 2, 1, 1, 0], 4, 2, 64, 32, wide=wide).check()


@pytest.mark.parametrize("hs,page,length", [(128, 64, 40000), (64, 16, 70001), (128, 128, 9999)])
@pytest.mark.parametrize("o_dtype", [sl.BF16, sl.FP32])
def test_one_long_request(usp, hs, page, length, o_dtype):
    Case(usp, length, [length], [1], 8, 2, hs, page, o_dtype=o_dtype).check()


@pytest.mark.parametrize("hs,page", [(128, 64), (64, 16), (128, 32)])
@pytest.mark.parametrize("hq,hk", [(32, 8), (4, 4), (6, 2), (8, 1)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("most", [1, 1000])
def test_ragged_rows(usp, hs, page, hq, hk, causal, most):
    """No row, one and many; fewer keys than rows (rows that see nothing); lengths of zero; rows behind the last request."""
    news = [1, 0, 3, 8, 17, 40, 64, 5, 130]
    lens = [77, 50, 3, 5, 17, 700, 64, 0, 1000]
    for wide in (False, True):          # (most: whether the kernel for few rows or the one for many has them)
        Case(usp, hq * hs + causal, lens, news, hq, hk, hs, page, causal=causal, strided=True, tail=3, wide=wide).check(max_q=most)


@pytest.mark.parametrize("hs", [64, 128])
@pytest.mark.parametrize("news", [[4], [8], [5, 2, 8], [16, 1]])
def test_a_few_rows(usp, hs, news):
    """One to four tiles of 16 rows and more, full and not; tables of up to 8192 tokens and beyond."""
    case = Case(usp, sum(news) + hs, [300 + 200 * i for i in range(len(news))], news, 8, 2, hs, 32)
    case.check()
    case.table = np.concatenate([case.table, np.full((len(news), 8192 // 32), 0x7fffff03, dtype=np.int32)], 1)
    case.check()


@pytest.mark.parametrize("hs", [64, 128])
def test_a_piece_of_a_prompt(usp, hs):
    Case(usp, hs, [2600], [700], 8, 2, hs, 64).check()
    Case(usp, hs + 1, [333, 0, 900], [333, 1, 100], 4, 4, hs, 16, o_dtype=sl.FP32).check()


@pytest.mark.parametrize("n", [64, 257, 700])
def test_many_requests(usp, n):
    rng = np.random.default_rng(n)
    lens = np.where(rng.random(n) < 0.1, 0, np.exp(rng.uniform(0, 6.5, n)).astype(int))
    for wide in (False, True):
        for most in (2, 100):
            Case(usp, n, lens.tolist(), rng.choice([0, 1, 1, 1, 2], n).tolist(), 4, 2, 64, 16, wide=wide).check(max_q=most)


def test_as_many_requests_as_there_may_be(usp):
    rng = np.random.default_rng(8192)
    lens = rng.integers(0, 40, 8192)
    Case(usp, 81, lens.tolist(), rng.choice([0, 1, 1, 2], 8192).tolist(), 2, 1, 64, 16, o_dtype=sl.FP32).check(max_q=2)


@pytest.mark.parametrize("most", [1, 1000])
def test_requests_that_share_pages(usp, most):
    """A prefix that several requests have in common, and a table row that names one page again and again."""
    case = Case(usp, 82, [200, 180, 130], [1, 40, 3], 8, 2, 128, 16)
    case.table[1, :8] = case.table[0, :8]
    case.table[2, :] = case.table[2, 0]
    case.check(max_q=most)


def test_the_most_rows_are_a_hint(usp):
    """max_q below and above what the requests have: the same attention."""
    case = Case(usp, 3, [500, 90, 1200], [1, 30, 9], 8, 2, 128, 64)
    outs = [case.check(max_q=m) for m in (0, 1, 2, 30, 5000)]
    assert all(torch.equal(outs[0][0], o) or float((outs[0][0].float() - o.float()).abs().max()) < 2e-2 for o, _ in outs)


@pytest.mark.parametrize("causal", [True, False])
def test_pages_of_other_ranks_and_their_merge(usp, causal):
    """Two ranks hold alternate pages of every request; usp_lse_merge of what each gives is attention over all."""
    for news in ([1, 1, 1], [1, 40, 200]):
        case = Case(usp, 21, [700, 41, 300], news, 8, 2, 128, 16, causal=causal, o_dtype=sl.FP32)
        whole, table, parts = case.reference(), case.table.copy(), []
        for rank in range(2):
            case.table = np.where(np.arange(table.shape[1]) % 2 == rank, table, -1 if rank else 2 ** 30).astype(np.int32)
            parts.append(case.check())
        o = torch.empty(case.total, 8, 128, device="cuda")
        lse = torch.empty(8, case.total, device="cuda")
        usp.usp_lse_merge([p[0] for p in parts], [p[1] for p in parts], o, lse, 1, case.total, 8, 128, usp.USP_FP32, usp.USP_FP32)
        sl.check_attention(sl.f64(o), sl.f64(lse), whole, sl.FP32)


def test_pages_dropped_at_random(usp):
    Case(usp, 22, [900, 64, 128, 1], [1, 2, 70, 1], 4, 2, 64, 16, drop=0.4, o_dtype=sl.FP32).check()
    Case(usp, 23, [900, 64], [1, 2], 4, 2, 128, 32, drop=1.1).check()      # none left


def test_what_stands_behind_the_length_has_no_influence(usp):
    """NaN codes and exponents of NaN behind kv_len, in the last page and in pages that no request names."""
    for hs, page, news in ((128, 64, [1, 1]), (64, 16, [1, 20]), (128, 32, [3, 70])):
        case = Case(usp, 31, [70, 201], news, 8, 2, hs, page)
        want = case.check()
        named = set()
        rows = sl.v_rows(case.cache.v_codes)
        for i, length in enumerate(case.lens):
            for b in range(-(-int(length) // page)):
                named.add(int(case.table[i, b]))
                tail = int(length) - b * page
                if tail < page:
                    case.cache.k_codes[case.table[i, b], :, tail:] = 0x7f
                    rows[case.table[i, b], :, tail:] = 0xff
        for other in set(range(case.cache.pages)) - named:
            case.cache.k_codes[other], rows[other] = 0xff, 0x7f
            case.cache.k_scale[other], case.cache.v_scale[other] = 255, 255
        case.cache.v_codes = sl.v_tiles(rows)
        case.cache.to_device()
        got = case.run()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("news", [[6], [40], [90]])
@pytest.mark.parametrize("hs", [64, 128])
def test_nan_reaches_the_rows_that_see_it_alone(usp, news, hs):
    """A NaN key makes the rows that see it NaN, a NaN value its column of theirs; earlier rows of the same tile stay clean."""
    case = Case(usp, 41, [150], news, 4, 2, hs, 32)
    rows = sl.v_rows(case.cache.v_codes)
    at = 150 - news[0] + news[0] // 2                       # a token of this step, in the middle
    rows[case.table[0, at // 32], 1, at % 32, 3] = 0x7f
    rows[case.table[0, 149 // 32], 0, 149 % 32, 40] = 0xff
    case.cache.v_codes = sl.v_tiles(rows)
    case.cache.to_device()
    o, lse = case.check()
    assert int(torch.isnan(o).sum()) == 2 * (news[0] - news[0] // 2) + 2
    assert not bool(torch.isnan(lse).any())
    case.cache.k_codes[case.table[0, at // 32], 0, at % 32, 7] = 0x7f
    case.cache.to_device()
    o, lse = case.check()
    assert int(torch.isnan(lse).sum()) == 2 * (news[0] - news[0] // 2)


def test_rows_of_nan_and_infinity(usp):
    case = Case(usp, 43, [100, 64], [3, 1], 4, 2, 64, 16)
    case.q[1, 2, 5] = float("nan")
    case.q[3, 0, 9] = float("inf")                          # scores of +inf and -inf: NaN, as inf - inf is
    o, lse = case.run()
    assert torch.isnan(o[1, 2]).all() and torch.isnan(o[3, 0]).all()
    o[1, 2], o[3, 0], lse[2, 1], lse[0, 3] = 0, 0, 0, 0
    ref = case.reference()
    ref[0][1, 2], ref[0][3, 0], ref[2][1, 2], ref[2][3, 0], ref[1][2, 1], ref[1][0, 3] = 0, 0, 0, 0, 0, 0
    sl.check_attention(sl.f64(o), sl.f64(lse), ref, sl.BF16)


def test_scale_and_far_exponents(usp):
    case = Case(usp, 44, [333], [2], 4, 2, 128, 64, o_dtype=sl.FP32)
    o, lse = case.run(scale=0.25)
    sl.check_attention(sl.f64(o), sl.f64(lse), case.reference(0.25), sl.FP32, 48.0)
    # the smallest and largest exponents that usp_cache_append writes, and one page far above the others
    case.cache.k_scale[:] = 10
    case.cache.v_scale[:] = 10
    case.cache.v_scale[case.table[0, 1]] = 214
    case.cache.to_device()
    case.check()
    case.cache.k_scale[:] = 121
    case.cache.v_scale[:] = 215
    case.cache.to_device()
    o, lse = case.run()
    k, v = case.cache.values()
    ref = sl.attention(sl.f64(case.q), k, v * 2.0 ** -100, case.cu, case.lens, case.table, 64, case.cache.pages, True)
    sl.check_attention(sl.f64(o) * 2.0 ** -100, sl.f64(lse), ref, sl.FP32)


def test_two_streams_two_workspaces_and_graphs(usp):
    """Results are those of a call alone, bit for bit: side by side on two streams, and replayed while other calls run between."""
    a, b = Case(usp, 51, [3000, 500], [1, 1], 8, 2, 128, 64), Case(usp, 52, [900, 2000], [30, 1], 8, 2, 128, 32)
    want = a.run(), b.run()
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        outs = []
        for case, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                outs.append(case.run())
        torch.cuda.synchronize()
        for got, w in zip(outs, want):
            assert torch.equal(got[0], w[0]) and torch.equal(got[1], w[1])
    ws = torch.empty(usp.usp_cache_attn_workspace_bytes(a.cache.c, 8, 1), dtype=torch.uint8, device="cuda")
    o, lse = torch.empty(a.total, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(8, a.total, device="cuda")
    cu, lens, table = sl.ints(a.cu), sl.ints(a.lens), sl.ints(a.table)
    call = lambda: usp.usp_cache_attn(a.cache.c, a.q, a.q.stride(0), cu, lens, table, a.table.shape[1], 2, a.total, 1, 8, 0.0, True, o, lse, sl.BF16, ws)  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for shorter in (0, 100, 2000, 2999):                    # the lengths stand on the device: a replay goes by what is there then
        lens.copy_(sl.ints(np.maximum(a.lens - shorter, 0)))
        o.zero_()
        graph.replay()
        b.run()
        torch.cuda.synchronize()
        again = o.clone(), lse.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(o, again[0]) and torch.equal(lse, again[1])
        k, v = a.cache.values()
        ref = sl.attention(sl.f64(a.q), k, v, a.cu, np.maximum(a.lens - shorter, 0), a.table, 64, a.cache.pages, True)
        sl.check_attention(sl.f64(o), sl.f64(lse), ref, sl.BF16)


@pytest.mark.parametrize("hs", [64, 128])
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [3, 1, 8, 2]])
def test_tables_whose_steps_pass_32_bits(usp, hs, news):
    """Rows of the table for 2^31 tokens: steps are counted in 64 bits, whatever the lengths are."""
    case = Case(usp, 71 + hs, [3000, 77, 900, 1], news, 16, 16, hs, 128)
    want = case.check()
    table = torch.full((4, 1 << 24), -1, dtype=torch.int32, device="cuda")
    table[:, :case.table.shape[1]] = sl.ints(case.table)
    o, lse = case.run(table=table)
    sl.check_attention(sl.f64(o), sl.f64(lse), case.reference(), sl.BF16)
    assert float((o.float() - want[0].float()).abs().max()) < 2e-2


def test_a_cache_beyond_32_bits(usp):
    """Codes at byte offsets of 2^32 and more: the pages that are named lie at the end of a cache of 5 GiB per tensor."""
    page, hk, hs = 128, 8, 128
    pages = (5 << 30) // (page * hk * hs)
    rng = np.random.default_rng(61)
    small = sl.Cache(usp, rng, 6, page, hk, hs)
    k_codes, v_codes = (torch.zeros(pages, hk * page * hs, dtype=torch.uint8, device="cuda") for _ in range(2))
    k_scale, v_scale = (torch.full((pages, hk), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
    where = [pages - 1, pages - 7, 0, 1 << 15, (1 << 15) - 1, pages // 2]
    for i, w in enumerate(where):
        k_codes[w], v_codes[w] = small.dev[0][i].flatten(), small.dev[1][i].flatten()
        k_scale[w], v_scale[w] = small.dev[2][i], small.dev[3][i]
    case = Case(usp, 62, [700], [2], 8, 8, hs, page)
    case.cache, case.table = small, np.arange(6, dtype=np.int32)[None]
    ref = case.reference()
    small.c, case.table = usp.cache(k_codes, v_codes, k_scale, v_scale, pages, page, hk, hs), np.array([where], dtype=np.int32)
    small.pages = pages
    o, lse = case.run()
    sl.check_attention(sl.f64(o), sl.f64(lse), ref, sl.BF16)
    # and a row written there
    x = torch.from_numpy(rng.standard_normal((1, hk, hs))).bfloat16().cuda()
    usp.usp_cache_append(small.c, x, x, sl.ints([(pages - 7) * page]), 1, hk * hs, hk * hs, sl.BF16)
    codes, scale = small.k_codes[1:2].copy(), small.k_scale[1:2].copy()
    sl.append(codes, scale, sl.f64(x), [0], page)
    assert sl.same_codes(k_codes[pages - 7].cpu().numpy(), codes.flatten())
    assert np.array_equal(k_scale[pages - 7].cpu().numpy(), scale[0])
