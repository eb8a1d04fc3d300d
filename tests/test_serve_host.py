"""CPU: what the entry points of rotary positions and of the 8-bit cache refuse, frequencies, workspace sizes, and how the
attention over the cache shares its steps among waves (in bounds and complete, whatever the lengths and tables hold)."""
import ctypes
import os

import numpy as np
import pytest

import paper_2405_07719_amd as usp
from tests import serve_testlib as sl
from tests.host_side import compile_host_side

A = 1 << 40          # an aligned address that is never followed


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(usp.LIB_PATH):
        from paper_2405_07719_amd import build
        build.build(verbose=False)
    return usp.load()


def test_e4m3_reference_is_torchs():
    import torch
    codes = torch.arange(256, dtype=torch.uint8)
    v = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, sl.VALUES, equal_nan=True)
    x = np.concatenate([np.random.default_rng(0).uniform(-448, 448, 4000), np.random.default_rng(1).standard_normal(4000) * 2.0 ** -7,
                        (sl.VALUES[:0x7e] + sl.VALUES[1:0x7f]) / 2, [0.0, -0.0, 448.0, -448.0, np.nan]])
    got = torch.tensor(x, dtype=torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert sl.same_codes(got, sl.e4m3_codes(x.astype(np.float32)))


@pytest.mark.parametrize("hs,d", [(64, 64), (128, 128), (128, 16), (128, 112), (64, 48)])
@pytest.mark.parametrize("scaling,kind", [("none", 0), ("linear", 1), ("base", 2), ("parts", 3)])
def test_frequencies(lib, hs, d, scaling, kind):
    r = usp.rope(hs, d, usp.USP_ROPE_PAIRS, 10000.0, kind, 4.0, 1.0, 32.0, 4096, 1.25)
    ref = sl.rope_frequencies(d, 10000.0, scaling, 4.0, 1.0, 32.0, 4096)
    assert (r.rotary_dim, r.layout, r.magnitude) == (d, 1, 1.25)
    np.testing.assert_allclose(r.freq[:d // 2], ref, rtol=2e-15)
    assert not any(r.freq[d // 2:])


def refused(status, call, *args, **kw):
    with pytest.raises(usp.UspError) as e:
        call(*args, **kw)
    assert e.value.status == status, e.value


def test_rope_refusals(lib):
    for status, args in ((6, (96, 64, 0, 1e4)), (2, (128, 24, 0, 1e4)), (2, (128, 0, 0, 1e4)), (2, (64, 128, 0, 1e4)), (6, (128, 64, 2, 1e4)),
                         (6, (128, 64, 0, 0.0)), (6, (128, 64, 0, float("inf"))), (6, (128, 64, 0, float("nan"))), (6, (128, 64, 0, 1e4, 4)),
                         (6, (128, 64, 0, 1e4, 1, 0.0)), (6, (128, 64, 0, 1e4, 3, 2.0, 5.0, 5.0, 100)), (6, (128, 64, 0, 1e4, 3, 2.0, 1.0, 5.0, 0)),
                         (6, (128, 64, 0, 1e-30)), (6, (128, 64, 0, 1e4, 0, 1.0, 1.0, 2.0, 0, float("inf")))):
        refused(status, usp.rope, *args)
    r = usp.rope(128, 128, 0, 1e4)
    rows = lambda q=A, k=A + (1 << 20), qo=A + (2 << 20), ko=A + (3 << 20), pos=A + (4 << 20), n=4, hq=4, hk=2, hs=128, qs=512, ks=256, qos=512, kos=256, dt=0, rope=r: (  # noqa: E731
        usp.usp_rope_rows(rope, q, k, qo, ko, pos, n, hq, hk, hs, qs, ks, qos, kos, dt, False, 0))
    refused(2, rows, n=-1)
    refused(4, rows, dt=2)
    refused(1, rows, pos=None)
    refused(1, rows, qo=None)
    refused(1, rows, q=None, qo=None, k=None, ko=None)
    refused(2, rows, hq=0)
    refused(2, rows, qs=504)
    refused(2, rows, kos=128)
    refused(6, rows, q=A + 2)
    refused(6, rows, ko=A + 8)
    refused(6, rows, qs=516)                       # rows not on 16 bytes
    refused(6, rows, qs=(1 << 30) + 512)
    refused(6, rows, hs=96)
    refused(6, rows, qo=A + 16)                    # over its own input, but not in place
    refused(6, rows, qo=A, qos=1024)               # in place at another stride
    refused(6, rows, qo=A + (1 << 20))             # over the other input
    refused(6, rows, qo=A + (3 << 20), ko=A + (3 << 20))
    refused(6, rows, qs=1024, k=A + 1024, ks=1024, qo=A + 512, qos=1024)    # columns that meet those of k
    rows(n=0, q=None, k=None, qo=None, ko=None, pos=None)                   # nothing to do
    bad = usp.rope(128, 128, 0, 1e4)
    bad.freq[3] = float("nan")
    refused(6, rows, rope=bad)
    bad.freq[3] = 2e6
    refused(6, rows, rope=bad)
    p = usp.problem(1, 256, 4, 2, 128, 2, 2, True)
    shards = lambda q=A, k=A + (1 << 20), qo=A + (2 << 20), ko=A + (3 << 20), b=0, e=4, rope=r, p=p: usp.usp_rope_shards(p, rope, q, k, qo, ko, False, b, e, 0)  # noqa: E731
    refused(6, shards, b=3, e=2)
    refused(6, shards, e=5)
    refused(6, shards, b=-1)
    refused(1, shards, q=None)
    refused(6, shards, qo=A + 512)
    refused(6, shards, qo=A + (1 << 20))
    refused(6, shards, q=A + 4)
    refused(2, shards, p=usp.problem(1, 250, 4, 2, 128, 2, 2, True))
    refused(2, shards, rope=usp.rope(128, 128, 0, 1e4), p=usp.problem(1, 256, 4, 2, 64, 2, 2, True))     # 128 elements of 64
    shards(b=2, e=2)


def cache(pages=10, page=32, hk=2, hs=128, kc=A, vc=A + (1 << 30)):
    return usp.cache(kc, vc, A + (2 << 30), A + (3 << 30), pages, page, hk, hs)


def test_cache_refusals(lib):
    ext = lambda cu=A, before=A + 64, n=3, total=8, table=A + 128, mp=4, page=16, pages=20, free=A + 192, nf=5, after=A + 256, slots=A + 320, pos=A + 384, taken=A + 448: (  # noqa: E731
        usp.usp_cache_extend(cu, before, n, total, table, mp, page, pages, free, nf, after, slots, pos, taken, 0))
    for status, kw in ((2, dict(n=-1)), (2, dict(total=-1)), (2, dict(nf=-1)), (2, dict(mp=0)), (2, dict(pages=0)), (6, dict(page=48)), (6, dict(page=8)),
                       (6, dict(n=8193)), (6, dict(total=1 << 31)), (6, dict(pages=1 << 27)), (1, dict(taken=None)), (1, dict(cu=None)),
                       (1, dict(table=None)), (1, dict(slots=None)), (1, dict(free=None)), (6, dict(after=A + 64)), (6, dict(slots=A)),
                       (6, dict(pos=A + 320))):
        refused(status, ext, **kw)
    app = lambda c=None, k=A + (4 << 30), v=A + (5 << 30), slots=A + (6 << 30), n=4, ks=256, vs=256, dt=0: usp.usp_cache_append(c or cache(), k, v, slots, n, ks, vs, dt, 0)  # noqa: E731
    for status, kw in ((2, dict(c=cache(pages=0))), (2, dict(c=cache(hk=0))), (6, dict(c=cache(hs=96))), (6, dict(c=cache(page=24))),
                       (6, dict(c=cache(pages=1 << 26))), (1, dict(c=cache(kc=None))), (6, dict(c=cache(vc=A + 8))), (2, dict(n=-1)), (4, dict(dt=3)),
                       (1, dict(k=None)), (1, dict(slots=None)), (2, dict(ks=248)), (6, dict(vs=260)), (6, dict(k=A + 2)), (6, dict(ks=(1 << 30) + 8))):
        refused(status, app, **kw)
    app(n=0, k=None, v=None, slots=None)
    need = usp.usp_cache_attn_workspace_bytes(cache(), 8, 1)
    att = lambda c=None, q=A + (4 << 30), qs=1024, cu=A + (5 << 30), lens=A + (6 << 30), table=A + (7 << 30), mp=4, n=2, total=2, mq=1, hq=8, scale=0.0, o=A + (8 << 30), lse=A + (9 << 30), dt=0, ws=A + (10 << 30), room=need: (  # noqa: E731
        usp.usp_cache_attn(c or cache(), q, qs, cu, lens, table, mp, n, total, mq, hq, scale, True, o, lse, dt, ws, room, 0))
    for status, kw in ((2, dict(n=-1)), (2, dict(total=-1)), (2, dict(mq=-1)), (2, dict(mp=0)), (2, dict(hq=0)), (3, dict(hq=7)), (6, dict(n=8193)),
                       (6, dict(total=1 << 31)), (6, dict(total=(1 << 31) - 1, hq=64)), (4, dict(dt=2)), (6, dict(scale=-1.0)), (6, dict(scale=float("nan"))), (6, dict(scale=float("inf"))),
                       (1, dict(q=None)), (1, dict(lse=None)), (1, dict(table=None)), (2, dict(qs=1016)), (6, dict(qs=1028)), (6, dict(q=A + 8)),
                       (6, dict(o=A + (8 << 30) + 2)), (5, dict(ws=None)), (5, dict(room=need - 1)), (6, dict(ws=A + (10 << 30) + 4)),
                       (6, dict(o=A + (4 << 30))), (6, dict(c=cache(hs=256)))):
        refused(status, att, **kw)
    att(total=0, q=None, cu=None, lens=None, table=None, o=None, lse=None, ws=None, room=0)
    att(n=0, q=None, cu=None, lens=None, table=None, o=None, lse=None, ws=None, room=0)
    assert usp.usp_cache_attn_workspace_bytes(cache(), 7, 1) == 0 == usp.usp_cache_attn_workspace_bytes(cache(hs=32), 8, 1)


def test_attention_workspace_depends_on_the_rows_of_a_tile_alone(lib):
    sizes = {(hs, hq, mq): usp.usp_cache_attn_workspace_bytes(cache(hs=hs), hq, mq) for hs in (64, 128) for hq in (2, 8, 64) for mq in (0, 1, 4, 5, 9, 4096)}
    assert max(sizes.values()) <= 96 << 20
    assert sizes[128, 8, 1] == sizes[128, 8, 0] == sizes[128, 8, 4] == usp.usp_cache_attn_workspace_bytes(cache(pages=1000, page=128, hk=4), 16, 8)


PLAN = """
#include <hip/hip_runtime.h>
#include <vector>
#include "serve_internal.h"
using namespace usp;
// Every wave's share of the steps, as the kernel walks it: how often each (row, key of a tile) is walked, and what the shares leave.
extern "C" int walk(const int32_t* cu, const int32_t* lens, int n, int64_t total, int group, int hk, int max_pages, int shift, int causal, int rt,
                    int waves, int64_t* keys_walked, int32_t* chains) {
  CacheAttnArgs a = {};
  a.cu_q = cu; a.kv_len = lens; a.total_q = total; a.group = group; a.hk = hk; a.max_pages = max_pages; a.page_shift = shift;
  a.n_seqs = n; a.causal = causal;
  int64_t all = 0;
  std::vector<int64_t> before(n + 1, 0);
  for (int i = 0; i < n; ++i) before[i + 1] = all += CacheUnits<>(a, i, rt).per_head * hk;
  const int shares = all < waves ? (int)all : waves;
  int open = 0;      // a unit that began and is not at its end yet
  int seq = 0;
  for (int w = 0; w < shares; ++w) {
    int64_t pos = all * w / shares;
    const int64_t stop = all * (w + 1) / shares;
    if (pos >= stop) return 1;                      // a share without steps would break a chain
    while (seq && before[seq] > pos) --seq;
    int first = 0;
    while (pos < stop) {
      while (before[seq + 1] <= pos) ++seq;
      const CacheUnits<> u(a, seq, rt);
      const auto at = u.locate(pos - before[seq]);
      const int of = u.steps(at.tile);
      if (at.head < 0 || at.head >= hk || at.tile < 0 || at.tile >= u.tiles || at.step < 0 || at.step >= of) return 2;
      const int rows = u.rows(a, at.tile, rt);
      if (rows < 1 || rows > rt) return 3;
      const int64_t row0 = (int64_t)at.tile * rt;
      const int vis = u.seen_by((row0 + rows - 1) / group), vis_first = u.seen_by(row0 / group);
      if (vis_first > vis || vis > u.len) return 4;
      if (vis > of * (int64_t)kCacheStep) return 5;     // keys that no step would walk
      const int s1 = stop - pos < of - at.step ? at.step + (int)(stop - pos) : of;
      const int64_t from = (int64_t)at.step * kCacheStep, to = (int64_t)s1 * kCacheStep < vis ? (int64_t)s1 * kCacheStep : vis;
      if (to > from) keys_walked[seq] += (to - from) * rows;
      const bool begins = at.step == 0, ends = s1 == of;
      if (!begins) {
        if (!open || first) return 6;
        first = 1;
        if (ends) open = 0;
      } else {
        if (open) return 7;
        if (!ends) open = 1, ++*chains;
      }
      pos += s1 - at.step;
    }
  }
  return open ? 8 : 0;
}
extern "C" int page_at(const int32_t* row, int b, int vis, int shift, int64_t pages) {
  const int number = row[cache_entry(b, vis, shift)];
  return cache_counts(b, vis, number, pages) ? number : -1;
}
extern "C" int entry_at(int b, int vis, int shift) { return cache_entry(b, vis, shift); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return compile_host_side(tmp_path_factory.mktemp("plan"), PLAN)


def walked(plan, cu, lens, group, hk, max_pages, shift, causal, rt, waves, total=None):
    cu, lens = np.asarray(cu, np.int32), np.asarray(lens, np.int32)
    n, total = len(lens), int(cu[-1]) if total is None else total
    keys, chains = np.zeros(max(n, 1), np.int64), ctypes.c_int32()
    ptr = lambda x: x.ctypes.data_as(ctypes.c_void_p)  # noqa: E731
    rc = plan.walk(ptr(cu), ptr(lens), n, ctypes.c_int64(total), group, hk, max_pages, shift, causal, rt, waves, ptr(keys), ctypes.byref(chains))
    assert rc == 0, (rc, cu, lens)
    return keys[:n], chains.value


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("rt,waves", [(16, 2048), (256, 256), (16, 3)])
def test_every_key_is_walked_once(plan, causal, rt, waves):
    rng = np.random.default_rng(rt + waves + causal)
    for _ in range(60):
        n = int(rng.integers(1, 40))
        group, hk, shift = int(rng.choice([1, 2, 3, 4, 8, 32, 71])), int(rng.choice([1, 2, 8])), int(rng.integers(4, 8))
        new = rng.choice([0, 1, 1, 1, 2, 7, 33, 300], n)
        lens = np.where(rng.random(n) < 0.2, rng.integers(0, 40, n), rng.integers(0, 20000, n))
        cu = np.concatenate([[0], np.cumsum(new)])
        max_pages = int(-(-lens.max() // (1 << shift))) + 1
        keys, _ = walked(plan, cu, lens, group, hk, max_pages, shift, causal, rt, waves)
        for i in range(n):
            # a tile is walked as far as its last row sees; so per head
            want, rows = 0, int(new[i]) * group
            for r0 in range(0, rows, rt):
                r1 = min(r0 + rt, rows)
                vis = lens[i] if not causal else max(0, int(lens[i]) - int(new[i]) + (r1 - 1) // group + 1)
                want += vis * (r1 - r0)
            assert keys[i] == want * hk, (i, new[i], lens[i], group)


def test_lengths_that_lie_are_held_within_the_table(plan):
    big = 2 ** 31 - 1
    keys, _ = walked(plan, [0, 1, 2, 3, 4], [-5, big, 100, 64], 4, 2, 8, 4, 1, 16, 2048)
    assert keys.tolist() == [0, 128 * 8, 100 * 8, 64 * 8]            # no more than 8 pages of 16 tokens
    # offsets that fall, lie outside or end behind the rows
    keys, _ = walked(plan, [-7, 3, 2, 1000000], [50, 50, 50], 1, 1, 8, 4, 0, 16, 2048, total=6)
    assert keys.tolist() == [3 * 50, 0, 4 * 50]
    assert walked(plan, [0, 0], [0], 1, 1, 1, 4, 1, 16, 2048)[0].tolist() == [0]
    # the longest that there can be: counts pass 32 bits
    keys, _ = walked(plan, [0, 70000], [big], 1, 8, 2 ** 24, 7, 0, 256, 256)
    assert keys[0] == (2 ** 31 - 128) * 70000 * 8


def test_pages_that_are_none(plan):
    row = np.array([3, -1, 9, 10, 0x7fffffff, -2 ** 31], np.int32)
    ptr = row.ctypes.data_as(ctypes.c_void_p)
    pages = lambda b, vis=10 ** 6, shift=5: plan.page_at(ptr, b, vis, shift, ctypes.c_int64(10))  # noqa: E731
    assert [pages(b) for b in range(12)] == [3, 3, -1, -1, 9, 9, -1, -1, -1, -1, -1, -1]
    assert [pages(b, 17) for b in range(4)] == [3, 3, -1, -1]
    for shift in range(4, 8):          # no entry behind the last page with a key that counts is read
        for vis in (1, 15, 16, 17, 127, 128, 129, 2 ** 31 - 1):
            assert all(0 <= plan.entry_at(b, vis, shift) <= (vis - 1) >> shift for b in (0, 1, 7, 8, 9, 2 ** 27 - 1))
