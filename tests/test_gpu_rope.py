"""GPU: rotary positions, forward and backward, against the formula in 64 bits (angles in extended precision)."""
import numpy as np
import pytest
import torch

from oracle import usp_oracle as orc
from tests import serve_testlib as sl

pytestmark = pytest.mark.gpu


def made(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape)).to(sl.torch_dtype(dtype)).cuda()


def check(got, x, positions, freq, pairs, magnitude, backward, dtype):
    y, size = sl.rope(sl.f64(x), positions, freq, pairs, magnitude, backward)
    tol = sl.rope_tolerance(y, size, dtype, positions, freq)
    far = np.abs(sl.f64(got) - y)
    assert np.all(far <= tol), (float((far / tol).max()), np.argwhere(far > tol)[0])


@pytest.mark.parametrize("dtype", [sl.BF16, sl.FP32])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("hs,d", [(128, 128), (128, 32), (128, 112), (64, 64), (64, 16)])
@pytest.mark.parametrize("rows,hq,hk", [(1, 32, 8), (7, 4, 4), (131, 3, 1), (1000, 32, 8)])
def test_rows(usp, dtype, pairs, hs, d, rows, hq, hk):
    rng = np.random.default_rng(rows * 7 + hs + d + pairs)
    pos = np.concatenate([[0], rng.integers(0, 300000, rows)])[:rows]
    r = usp.rope(hs, d, int(pairs), 500000.0, usp.USP_ROPE_BY_PARTS, 8.0, 1.0, 32.0, 8192, 1.2)
    q, k = made(rng, (rows, hq, hs), dtype), made(rng, (rows, hk, hs), dtype)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    for backward in (False, True):
        usp.usp_rope_rows(r, q, k, qo, ko, sl.ints(pos), rows, hq, hk, hs, hq * hs, hk * hs, hq * hs, hk * hs, dtype, backward)
        for got, x in ((qo, q), (ko, k)):
            check(got, x, pos, r.freq[:d // 2], pairs, r.magnitude, backward, dtype)
            assert torch.equal(got[..., d:], x[..., d:])


@pytest.mark.parametrize("dtype", [sl.BF16, sl.FP32])
def test_positions_over_the_whole_range(usp, dtype):
    """Far positions, whose angles 32 bits do not hold; negative ones are turned the other way."""
    rng = np.random.default_rng(5)
    pos = np.array([0, 1, -1, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 212991, 1 << 20, 12345678])
    r = usp.rope(64, 64, 0, 10000.0)
    q = made(rng, (len(pos), 5, 64), dtype)
    out = torch.empty_like(q)
    usp.usp_rope_rows(r, q, None, out, None, sl.ints(pos), len(pos), 5, 0, 64, 320, 0, 320, 0, dtype, False)
    check(out, q, pos, r.freq[:32], False, 1.0, False, dtype)


@pytest.mark.parametrize("dtype", [sl.BF16, sl.FP32])
def test_in_place_in_the_columns_of_a_qkv_product(usp, dtype):
    rng = np.random.default_rng(6)
    rows, hq, hk, hs = 77, 6, 2, 128
    qkv = made(rng, (rows, hq + 2 * hk, hs), dtype)
    was = qkv.clone()
    pos = rng.integers(0, 5000, rows)
    r = usp.rope(hs, 96, 1, 10000.0)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hk]
    usp.usp_rope_rows(r, q, k, q, k, sl.ints(pos), rows, hq, hk, hs, *[qkv.stride(0)] * 4, dtype, False)
    check(q, was[:, :hq], pos, r.freq[:48], True, 1.0, False, dtype)
    check(k, was[:, hq:hq + hk], pos, r.freq[:48], True, 1.0, False, dtype)
    assert torch.equal(qkv[:, hq + hk:], was[:, hq + hk:])
    # K alone, out of the columns into a tensor of its own
    out = torch.empty(rows, hk, hs, dtype=qkv.dtype, device="cuda")
    usp.usp_rope_rows(r, None, was[:, hq:], None, out, sl.ints(pos), rows, 0, hk, hs, 0, was.stride(0), 0, hk * hs, dtype, True)
    check(out, was[:, hq:hq + hk], pos, r.freq[:48], True, 1.0, True, dtype)


@pytest.mark.parametrize("bs,L,U,R,zigzag", [(1, 256, 2, 2, True), (2, 240, 1, 4, True), (1, 1000, 4, 2, False), (2, 96, 2, 3, True), (1, 64, 8, 1, True),
                                             (3, 7, 1, 1, False)])
@pytest.mark.parametrize("dtype,backward", [(sl.BF16, False), (sl.FP32, True)])
def test_shards(usp, bs, L, U, R, zigzag, dtype, backward):
    """Each rank's shard at the oracle's Algorithm 2 positions; ranks that are not asked for stay as they were."""
    rng = np.random.default_rng(L)
    N, n, hc, hk, hs = U * R, L // (U * R), 16, 8, 64
    p = usp.problem(bs, L, hc, hk, hs, U, R, True, usp.USP_SPLIT_ZIGZAG if zigzag else usp.USP_SPLIT_CONTIG, dtype)
    r = usp.rope(hs, 64, 0, 10000.0, magnitude=0.75)
    q, k = made(rng, (N, bs, n, hc, hs), dtype), made(rng, (N, bs, n, hk, hs), dtype)
    for begin, end in ((0, N), (N - 1, N), (N // 2, N // 2 + 1)):
        qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
        usp.usp_rope_shards(p, r, q, k, qo, ko, backward, begin, end)
        for rank in range(N):
            pos = orc.zigzag_positions(L, R, U, rank // U, rank % U, zigzag)
            for got, x in ((qo, q), (ko, k)):
                if begin <= rank < end:
                    check(got[rank], x[rank], pos, r.freq[:32], False, 0.75, backward, dtype)
                else:
                    assert bool((got[rank] == 7.0).all())
    inplace = q.clone()
    usp.usp_rope_shards(p, r, inplace, None, inplace, None, backward, 0, N)
    usp.usp_rope_shards(p, r, q, None, qo, None, backward, 0, N)
    assert torch.equal(inplace, qo)


def test_backward_is_the_gradient(usp):
    """Against differences: the rotation is linear, so <dy, f(x + h) - f(x)> / h is <backward(dy), h-direction> exactly, up to rounding."""
    rng = np.random.default_rng(8)
    rows, h, hs = 40, 3, 128
    r = usp.rope(hs, 64, 1, 10000.0, usp.USP_ROPE_LINEAR, 2.0, magnitude=1.5)
    pos = sl.ints(rng.integers(0, 100000, rows))
    run = lambda x, backward: (usp.usp_rope_rows(r, x, None, out := torch.empty_like(x), None, pos, rows, h, 0, hs, h * hs, 0, h * hs, 0, sl.FP32, backward), out)[1]  # noqa: E731
    x, step, dy = (made(rng, (rows, h, hs), sl.FP32) for _ in range(3))
    change = (run(x + step, False).double() - run(x, False).double())
    a, b = float((dy.double() * change).sum()), float((run(dy, True).double() * step.double()).sum())
    # the three results, and x + step, are rounded to 24 bits: at most 4 * 2^-24 of sums of rows * h * hs terms of size 1.5 * 2 * 3 * 3
    assert abs(a - b) <= 4 * 2.0 ** -24 * rows * h * hs * 27


def test_nan_and_infinity_stay_in_their_pair(usp):
    r = usp.rope(64, 64, 0, 10000.0)
    q = torch.ones(3, 2, 64, device="cuda")
    q[1, 0, 5], q[2, 1, 40] = float("nan"), float("inf")
    out = torch.empty_like(q)
    usp.usp_rope_rows(r, q, None, out, None, sl.ints([3, 4, 5]), 3, 2, 0, 64, 128, 0, 128, 0, sl.FP32, False)
    bad = (~torch.isfinite(out)).nonzero().tolist()
    assert bad == [[1, 0, 5], [1, 0, 37], [2, 1, 8], [2, 1, 40]]


def test_captured_and_on_another_stream(usp):
    rng = np.random.default_rng(9)
    r = usp.rope(128, 128, 0, 10000.0)
    q, pos = made(rng, (9, 4, 128), sl.BF16), sl.ints(rng.integers(0, 1000, 9))
    want, out = torch.empty_like(q), torch.empty_like(q)
    call = lambda o: usp.usp_rope_rows(r, q, None, o, None, pos, 9, 4, 0, 128, 512, 0, 512, 0, sl.BF16, False)  # noqa: E731
    call(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in range(3):
        q.copy_(made(rng, (9, 4, 128), sl.BF16))
        pos += 17
        out.zero_()
        graph.replay()
        call(want)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_tensors_that_are_not_on_the_device_are_refused(usp):
    r = usp.rope(64, 64, 0, 10000.0)
    q = torch.ones(1, 1, 64)
    with pytest.raises(ValueError):
        usp.usp_rope_rows(r, q, None, q, None, sl.ints([0]), 1, 1, 0, 64, 64, 0, 64, 0, sl.FP32, False)
