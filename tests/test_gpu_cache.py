"""GPU: block tables and slots (whole numbers, equal) and rows written to the 8-bit cache (codes and exponents, equal) against plain
loops on the host."""
import numpy as np
import pytest
import torch

from tests import serve_testlib as sl

pytestmark = pytest.mark.gpu


def extend(usp, cu, before, total, table, page, pages, free, max_pages=None):
    n = len(before)
    max_pages = max_pages or np.shape(table)[1]
    t, f = sl.ints(table), sl.ints(free)
    after, slots, positions, taken = (torch.full((x,), 77, dtype=torch.int32, device="cuda") for x in (n, total, total, 2))
    usp.usp_cache_extend(sl.ints(cu), sl.ints(before), n, total, t, max_pages, page, pages, f, len(free), after, slots, positions, taken)
    got = [x.cpu().numpy() for x in (t, after, slots, positions, taken)]
    want = sl.extend(list(cu), list(before), total, table, page, pages, list(free))
    for name, a, b in zip(("table", "len_after", "slots", "positions", "taken"), got, want):
        assert np.array_equal(a.reshape(-1), np.asarray(b, dtype=np.int64).reshape(-1)), name
    return got


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n,most", [(1, 1), (1, 5000), (3, 1), (255, 3), (256, 1), (257, 90), (1000, 2), (2100, 40), (6100, 1), (8192, 3)])
def test_extend(usp, page, n, most):
    rng = np.random.default_rng(n + most + page)
    before = np.where(rng.random(n) < 0.2, 0, rng.integers(0, 700, n))
    before[rng.integers(0, n)] = page                       # a full page: the next token begins another
    new = rng.integers(0, most + 1, n)
    new[rng.integers(0, n)] = most
    cu = np.concatenate([[0], np.cumsum(new)])
    held = -(-before // page)
    need = -(-(before + new) // page) - held
    pages = int(held.sum() + need.sum()) + 3
    order = rng.permutation(pages)
    table = np.full((n, int((held + need).max()) + 1), -1)
    at = 0
    for i in range(n):
        table[i, :held[i]] = order[at:at + held[i]]
        at += held[i]
    for spare in (0, 3):                                    # rows of no request behind the last one
        extend(usp, cu, before, int(cu[-1]) + spare, table, page, pages, order[at:])
    # a list of free pages that ends on the way, and rows of the table too short for some
    extend(usp, cu, before, int(cu[-1]), table, page, pages, order[at:at + int(need.sum()) // 2])
    if held.max() < table.shape[1] - 1:
        short = table[:, :max(int(held.max()), 1)]
        extend(usp, cu, before, int(cu[-1]), short, page, pages, order[at:])


def test_extend_of_nothing_and_of_numbers_that_lie(usp):
    got = extend(usp, [0], [], 4, np.zeros((0, 3)), 16, 8, [1, 2], max_pages=3)
    assert got[2].tolist() == [-1] * 4 and got[4].tolist() == [0, 0]
    got = extend(usp, [0, 0, 0], [5, 32], 0, [[1, -1], [2, 3]], 16, 8, [])
    assert got[1].tolist() == [5, 32] and got[4].tolist() == [0, 0]
    # lengths below zero and beyond the table; free pages that are none; a page that another rank holds
    got = extend(usp, [0, 1, 2, 3, 5], [-4, 2 ** 31 - 1, 16, 20], 5, [[1, 2], [3, 4], [5, -1], [6, -1]], 16, 8, [900, -1])
    assert got[2].tolist() == [-1] * 5 and got[1].tolist() == [-4, 2 ** 31 - 1, 17, 22]


def append_case(usp, page, hk, hs, dtype, olds, news, seed, strided=False, spread=0.0, special=False):
    rng = np.random.default_rng(seed)
    n, rows = len(olds), int(sum(news))
    lens = [o + m for o, m in zip(olds, news)]
    pages = sum(-(-x // page) for x in lens) + 2
    cache = sl.Cache(usp, rng, pages, page, hk, hs)
    cache.k_scale[:], cache.v_scale[:] = rng.integers(112, 122, cache.k_scale.shape), rng.integers(112, 122, cache.k_scale.shape)
    cache.to_device()
    table = sl.ragged_table(rng, lens, page, pages, max(-(-x // page) for x in lens))
    slots = np.concatenate([[table[i, p // page] * page + p % page for p in range(olds[i], lens[i])] for i in range(n)]).astype(np.int64)
    t = sl.torch_dtype(dtype)
    size = 2.0 ** (spread * rng.standard_normal((rows, hk, 1)))
    k, v = (torch.from_numpy(rng.standard_normal((rows, hk, hs)) * size).to(t).cuda() for _ in range(2))
    if special:
        for x in (k, v):
            x[0, 0, 0] = x[rows - 1, 1, 2] = float("nan")
            if special == "infinite":
                x[rows // 2, hk - 1, hs - 1], x[rows - 1, 0, 3] = float("inf"), float("-inf")
            x[rows // 3] = 0.0
    if strided:
        both = torch.zeros(rows, 3 * hk, hs, dtype=t, device="cuda")
        both[:, hk:2 * hk], both[:, 2 * hk:] = k, v
        k, v = both[:, hk:2 * hk], both[:, 2 * hk:]
    usp.usp_cache_append(cache.c, k, v, sl.ints(slots), rows, k.stride(0), v.stride(0), dtype)
    got = [x.cpu().numpy() for x in cache.dev]
    kr, vr = cache.k_codes.copy(), sl.v_rows(cache.v_codes)
    ks, vs = cache.k_scale.copy(), cache.v_scale.copy()
    sl.append(kr, ks, sl.f64(k), slots.tolist(), page)
    sl.append(vr, vs, sl.f64(v), slots.tolist(), page)
    assert np.array_equal(got[2], ks) and np.array_equal(got[3], vs)
    assert sl.same_codes(got[0], kr)
    assert sl.same_codes(got[1], sl.v_tiles(vr))
    return cache


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("hs,dtype", [(128, sl.BF16), (64, sl.BF16), (128, sl.FP32), (64, sl.FP32)])
def test_append(usp, page, hs, dtype):
    # first and last places of a page, tiles begun and ended inside, one token and many
    append_case(usp, page, 2, hs, dtype, [0, 1, 15, 16, 17, page - 1, page, 3, 40], [1, 1, 1, 1, 1, 1, 1, 200, 2 * page], page + hs, spread=2.0)
    append_case(usp, page, 3, hs, dtype, [0], [1], 3)
    append_case(usp, page, 1, hs, dtype, [5, 0], [page - 5, 3 * page + 7], 4, strided=True)


@pytest.mark.parametrize("rows", [2048, 2049, 5000, 8192, 8200, 20000])
def test_append_of_many_rows(usp, rows):
    """Waves that look at one row each, and at several."""
    rng = np.random.default_rng(rows)
    news = []
    while sum(news) < rows:
        news.append(int(min(rng.choice([1, 1, 2, 30, 130]), rows - sum(news))))
    append_case(usp, 32, 1, 64, sl.BF16, rng.integers(0, 90, len(news)).tolist(), news, rows, spread=1.0)


@pytest.mark.parametrize("dtype", [sl.BF16, sl.FP32])
def test_append_of_nan_infinity_and_zero(usp, dtype):
    for special in ("nan", "infinite"):
        append_case(usp, 32, 2, 128, dtype, [3, 0, 0], [4, 50, 1], 5, special=special)
        append_case(usp, 128, 2, 64, dtype, [0, 60], [128, 10], 6, special=special)


def test_exponents_at_their_ends(usp):
    """The largest and smallest values of 32 bits, and the first value above a power's reach."""
    rng = np.random.default_rng(11)
    cache = sl.Cache(usp, rng, 8, 16, 1, 64)
    f = np.finfo(np.float32)
    heads = [f.max, f.tiny, f.smallest_subnormal, 448.0, np.nextafter(np.float32(448), np.float32(500)), 2.0 ** -109 * 1.75, 0.0, 2.0 ** 127]
    x = np.zeros((8, 1, 64), dtype=np.float32)
    for i, h in enumerate(heads):
        x[i, 0] = np.float32(h) * rng.uniform(-1, 1, 64).astype(np.float32)
        x[i, 0, i] = h
    k = torch.from_numpy(x).cuda()
    slots = np.arange(8) * 16
    usp.usp_cache_append(cache.c, k, k, sl.ints(slots), 8, 64, 64, sl.FP32)
    kr, ks = cache.k_codes.copy(), cache.k_scale.copy()
    sl.append(kr, ks, x.astype(np.float64), slots.tolist(), 16)
    assert np.array_equal(cache.dev[2].cpu().numpy(), ks), (cache.dev[2].flatten().tolist(), ks.flatten().tolist())
    assert sl.same_codes(cache.dev[0].cpu().numpy(), kr)


def test_slots_that_are_none_and_stretches_of_one_page(usp):
    """Padding is skipped; rows of a page that do not follow on one another, or name a place twice, count one after the other."""
    rng = np.random.default_rng(12)
    cache = sl.Cache(usp, rng, 6, 16, 2, 128)
    slots = [-1, 20, 21, 25, 25, 17, 18, 19, -1, -7, 96, 2 ** 31 - 1, 50, 3, 4, 48]
    x = (rng.standard_normal((len(slots), 2, 128)) * 2.0 ** np.arange(len(slots))[:, None, None]).astype(np.float32)
    k = torch.from_numpy(x).cuda()
    usp.usp_cache_append(cache.c, k, k, sl.ints(slots), len(slots), 256, 256, sl.FP32)
    for codes, scale, dev in ((cache.k_codes.copy(), cache.k_scale.copy(), (0, 2)), (sl.v_rows(cache.v_codes), cache.v_scale.copy(), (1, 3))):
        want = slots[:12] + [50] + slots[13:15] + [48]
        sl.append(codes, scale, x.astype(np.float64), want, 16)
        got = cache.dev[dev[0]].cpu().numpy()
        got = sl.v_rows(got) if got.ndim == 5 else got
        # page 3 is named twice, by rows that do not stand together: its values are undefined
        keep = [0, 1, 2, 4, 5]
        assert np.array_equal(cache.dev[dev[1]].cpu().numpy()[keep], scale[keep])
        assert sl.same_codes(got[keep], codes[keep])


def test_codes_grow_with_their_page(usp):
    """One token after the other, each larger than all before: the page's codes are rounded again at every step, as on the host."""
    rng = np.random.default_rng(13)
    for hs, page in ((128, 32), (64, 64)):
        cache = sl.Cache(usp, rng, 3, page, 2, hs)
        kr, ks, vr, vs = cache.k_codes.copy(), cache.k_scale.copy(), sl.v_rows(cache.v_codes), cache.v_scale.copy()
        for i in range(page):
            x = (rng.standard_normal((1, 2, hs)) * 2.0 ** (i / 3 - 5)).astype(np.float32)
            d = torch.from_numpy(x).cuda()
            usp.usp_cache_append(cache.c, d, d, sl.ints([page + i]), 1, 2 * hs, 2 * hs, sl.FP32)
            sl.append(kr, ks, x.astype(np.float64), [page + i], page)
            sl.append(vr, vs, x.astype(np.float64), [page + i], page)
        got = [x.cpu().numpy() for x in cache.dev]
        assert np.array_equal(got[2], ks) and np.array_equal(got[3], vs)
        assert sl.same_codes(got[0], kr) and sl.same_codes(sl.v_rows(got[1]), vr)
