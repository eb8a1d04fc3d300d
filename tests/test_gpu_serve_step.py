"""GPU: the operators together, as they are used: requests that are answered token by token over the 8-bit cache, after a prompt that
usp_attn_fwd ran; and a training step with rotary positions."""
import numpy as np
import pytest
import torch

from oracle import usp_oracle as orc
from tests import serve_testlib as sl
from tests import usp_testlib as tl

pytestmark = pytest.mark.gpu


class Server:
    """What a serving program keeps: the cache, tables and lengths on the device, and one step's calls."""

    def __init__(self, usp, n, pages, page, hq, hk, hs, most):
        self.usp, self.n, self.hq, self.hk, self.hs, self.page, self.pages, self.most = usp, n, hq, hk, hs, page, pages, most
        u8 = dict(dtype=torch.uint8, device="cuda")
        self.codes = [torch.full((pages, hk, page, hs), 0x7f, **u8), torch.full((pages, hk, page // 16, hs, 16), 0x7f, **u8)]
        self.scales = [torch.full((pages, hk), 255, **u8) for _ in range(2)]
        self.c = usp.cache(*self.codes, *self.scales, pages, page, hk, hs)
        self.table, self.lens = torch.full((n, most), -1, dtype=torch.int32, device="cuda"), sl.ints([0] * n)
        self.free = torch.randperm(pages, device="cuda").int()
        self.after, self.taken = sl.ints([0] * n), sl.ints([0, 0])
        self.rope = usp.rope(hs, hs, usp.USP_ROPE_HALVES, 10000.0)

    def step(self, qkv, cu, total, max_q, o, lse, slots, positions, ws):
        """qkv [total][hq + 2 hk][hs], turned in place."""
        usp, w = self.usp, qkv.stride(0)
        usp.usp_cache_extend(cu, self.lens, self.n, total, self.table, self.most, self.page, self.pages, self.free, self.free.numel(), self.after,
                             slots, positions, self.taken)
        q, k, v = qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hk], qkv[:, self.hq + self.hk:]
        usp.usp_rope_rows(self.rope, q, k, q, k, positions, total, self.hq, self.hk, self.hs, w, w, w, w, sl.BF16, False)
        usp.usp_cache_append(self.c, k, v, slots, total, w, w, sl.BF16)
        usp.usp_cache_attn(self.c, q, w, cu, self.after, self.table, self.most, self.n, total, max_q, self.hq, 0.0, True, o, lse, sl.BF16, ws)
        # the next step's lists: lengths, and the free pages without those taken (moved to the front, -1 behind)
        self.lens.copy_(self.after)
        at = torch.arange(self.free.numel(), device="cuda") + self.taken[0]
        self.free.copy_(torch.where(at < self.free.numel(), self.free[at.clamp_max(self.free.numel() - 1)], -1))


def plain_step(history, qkv, cu, before, hq, hk, page, rope):
    """The same in 64 bits on the host.  history: per request, its (K, V) rows in float64 as bf16 holds them after turning."""
    outs = []
    for i in range(len(before)):
        x = qkv[cu[i]:cu[i + 1]]
        pos = np.arange(before[i], before[i] + len(x))
        turned = sl.rope(x[:, :hq + hk], pos, rope.freq[:qkv.shape[2] // 2], False, 1.0, False)[0]
        turned = torch.from_numpy(turned).bfloat16().double().numpy()
        k = np.concatenate([history[i][0], turned[:, hq:]])
        v = np.concatenate([history[i][1], x[:, hq + hk:]])
        history[i] = (k, v)
        n = len(k)
        for j in range(len(x)):
            seen = before[i] + j + 1
            row = []
            for h in range(hq):
                s = k[:seen, h // (hq // hk)] @ turned[j, h] * qkv.shape[2] ** -0.5
                p = np.exp(s - s.max())
                row.append(p @ v[:seen, h // (hq // hk)] / p.sum())
            outs.append(row)
    return np.array(outs).reshape(-1, hq, qkv.shape[2])


def test_prompts_then_tokens_one_by_one(usp):
    """Ragged prompts, then tokens: tables grow, pages fill, exponents grow.  Against attention over the unrounded K and V: what 8 bits
    cost is at most half a step of e4m3, 2^-4 of a value (where it is normal), so that O is within a few hundredths."""
    n, hq, hk, hs, page = 5, 8, 2, 64, 16
    rng = np.random.default_rng(1)
    server = Server(usp, n, 64, page, hq, hk, hs, 12)
    history, before = [(np.zeros((0, hk, hs)), np.zeros((0, hk, hs))) for _ in range(n)], np.zeros(n, dtype=int)
    for step, new in enumerate([[40, 1, 0, 16, 33], [1, 1, 7, 1, 1], [1, 1, 1, 1, 1], [1, 1, 1, 1, 1], [0, 1, 1, 3, 1]]):
        cu = np.concatenate([[0], np.cumsum(new)])
        total = int(cu[-1])
        x = rng.standard_normal((total, hq + 2 * hk, hs))
        x = torch.from_numpy(x).bfloat16()
        qkv = x.cuda()
        o, lse = torch.empty(total, hq, hs, dtype=torch.bfloat16, device="cuda"), torch.empty(hq, total, device="cuda")
        slots, positions = sl.ints([0] * total), sl.ints([0] * total)
        ws = torch.empty(usp.usp_cache_attn_workspace_bytes(server.c, hq, max(new)), dtype=torch.uint8, device="cuda")
        server.step(qkv, sl.ints(cu), total, max(new), o, lse, slots, positions, ws)
        want = plain_step(history, x.double().numpy(), cu, before, hq, hk, page, server.rope)
        before = before + new
        assert np.array_equal(server.lens.cpu().numpy(), before)
        got = sl.f64(o)
        # scores: sum of hs products q * dk * hs^-1/2 with |dk| <= 2^-4 |k|: standard deviation about 2^-5 to 2^-4; so P is off by
        # some percent, O (a mean of N(0,1) values, themselves off by up to 2^-4) by about a twentieth of its size
        assert np.linalg.norm(got - want) <= 0.07 * np.linalg.norm(want)
    assert int((server.free >= 0).sum()) == 64 - int(sum(-(-x // page) for x in before))


def test_a_captured_step_replayed(usp):
    """One token of each request per replay, nothing from the host: positions, pages and lengths move on by themselves; as eager calls do."""
    n, hq, hk, hs, page = 3, 4, 2, 128, 16
    outs = []
    x = torch.randn(40, n, hq + 2 * hk, hs, device="cuda").bfloat16()
    order = torch.randperm(24, device="cuda").int()
    for captured in (False, True):
        server = Server(usp, n, 24, page, hq, hk, hs, 8)
        server.free.copy_(order)
        qkv, o, lse = torch.empty_like(x[0]), torch.empty(n, hq, hs, dtype=torch.bfloat16, device="cuda"), torch.empty(hq, n, device="cuda")
        slots, positions, cu = sl.ints([0] * n), sl.ints([0] * n), sl.ints(range(n + 1))
        ws = torch.empty(usp.usp_cache_attn_workspace_bytes(server.c, hq, 1), dtype=torch.uint8, device="cuda")
        run = lambda: server.step(qkv, cu, n, 1, o, lse, slots, positions, ws)  # noqa: E731
        got = []
        if captured:
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):       # (torch's own operators want a first call before a capture)
                qkv.copy_(x[0])
                run()
            side.synchronize()
            server.lens.zero_()
            server.table.fill_(-1)
            server.free.copy_(order)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                run()
        for i in range(x.shape[0]):
            qkv.copy_(x[i])
            if captured:
                graph.replay()
            else:
                run()
            torch.cuda.synchronize()
            got.append((o.clone(), lse.clone(), slots.clone()))
        outs.append(got)
    for a, b in zip(*outs):
        for s, t in zip(a, b):
            assert torch.equal(s, t)
    assert outs[0][-1][2].unique().numel() == n


@pytest.mark.parametrize("U,R", [(2, 2), (1, 4), (1, 1)])
def test_training_step_with_rotary_positions(usp, U, R):
    """Q and K turned in their shards, attention, its backward, and the rotation's backward on dQ and dK: the gradients are those of the
    whole, by the oracle's attention gradient on Q and K as bf16 holds them after turning."""
    seed, bs, L, hc, hk, hs = 77, 1, 512, 4, 4 if U == 2 else 2, 64
    prob = tl.Problem(seed, bs, L, hc, hk, hs, U, R, True, True, tl.BF16, with_do=True)
    p = usp.problem(bs, L, hc, hk, hs, U, R, True)
    r = usp.rope(hs, hs, usp.USP_ROPE_PAIRS, 10000.0, magnitude=0.9)
    N = prob.N
    q, k, v, do = (prob.seq_layout_dev(x) for x in ("q", "k", "v", "do"))
    usp.usp_rope_shards(p, r, q, k, q, k, False, 0, N)
    o, dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    lse = torch.empty(N, bs, hc // U, L // R, device="cuda")
    room = max(usp.usp_attn_fwd_workspace_bytes(p, N), usp.usp_attn_bwd_workspace_bytes(p, N), 16)
    ws = torch.empty(room, dtype=torch.uint8, device="cuda")
    usp.usp_attn_fwd(p, q, k, v, o, lse, 0, N, ws)
    usp.usp_attn_bwd(p, q, k, v, o, lse, do, dq, dk, dv, 0, N, ws)
    before = dq.clone(), dk.clone()
    usp.usp_rope_shards(p, r, dq, dk, dq, dk, True, 0, N)

    pos = np.arange(L)
    turn = lambda x, back: sl.rope(x, pos, r.freq[:hs // 2], True, r.magnitude, back)[0]  # noqa: E731
    tq = torch.from_numpy(turn(prob.val["q"], False)).bfloat16().double().numpy()
    tk = torch.from_numpy(turn(prob.val["k"], False)).bfloat16().double().numpy()
    grads = orc.attention_backward(tq, tk, prob.val["v"], prob.val["do"], True)
    for got, mid, ref in ((dq, before[0], grads[0]), (dk, before[1], grads[1])):
        want = turn(ref, True)
        for rank in range(N):
            at = prob.rank_positions(rank)
            # the rotation mixes two elements that are each within the backward's 5e-2 of their value, and rounds once more
            assert np.abs(sl.f64(got)[rank] - want[:, at]).max() <= 5e-2 * 0.9 * 2 ** 0.5 + 2.0 ** -8 * np.abs(want).max()
            y, size = sl.rope(sl.f64(mid)[rank], at, r.freq[:hs // 2], True, r.magnitude, True)
            assert np.all(np.abs(sl.f64(got)[rank] - y) <= sl.rope_tolerance(y, size, sl.BF16, at, r.freq[:hs // 2]))
