"""codecomp_attend_shared, codecomp_attend_mass and codecomp_evict against the fp64 oracle (copies and numbers of rows: exactly): lengths, groups, masks, pages, types,
garbage where nothing is read, graphs, streams, and a run of them together."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from oracle import serve_oracle as srv
from paper_2604_10235_amd import binding as b
from tests import cache_util as cu_

pytestmark = pytest.mark.gpu


def dev(x, kind=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype=kind))).cuda()


def cum(x):
    return np.concatenate([[0], np.cumsum(x)]).astype(np.int32)


def scales(fp8):
    return dict(k_scale=0.03, v_scale=0.02) if fp8 else {}


class Forked:
    """Groups of requests; the table of a group's first request holds the shared rows, the others' entries for whole shared pages are numbers of no page.  `loose`: the bound on
    lengths that calls are told, under which there may be some work, or much: what is short, or little, goes to one kernel whatever its rows."""

    def __init__(self, rng, members, prefixes, news, owns, *, n_q, n_kv, d, page, fp8=False, layers=1, wrong_entries=True, width_more=0, loose=0):
        self.of = [g for g, n in enumerate(members) for _ in range(n)]
        self.members, self.prefixes, self.news, self.n_q = members, prefixes, news, n_q
        self.lens = [prefixes[g] + max(o, 0) for g, o in zip(self.of, owns)]
        self.loose = loose and max([loose] + self.lens)
        width_more = max(width_more, -(-loose // page))
        self.cache = cu_.Cache(rng, self.lens, n_kv=n_kv, d=d, page=page, fp8=fp8, layers=layers, width_more=width_more, **scales(fp8))
        self.cu_groups = cum(members)
        if wrong_entries:
            for r, g in enumerate(self.of):
                if r != self.cu_groups[g]:
                    self.cache.table[r, : prefixes[g] // page] = rng.choice([-1, self.cache.n_pages, 2**31 - 1])
        self.cu = cum(news)
        self.T = int(self.cu[-1])
        self.q = cu_.bf16(rng.standard_normal((self.T, n_q, d))).cuda()

    def batch(self, **kw):
        if self.loose and kw.get("max_kv") is None:
            kw["max_kv"] = self.loose
        return cu_.make_batch(self.cache, self.news, self.n_q, lens=self.lens, **kw)[0]

    def groups(self, max_prefix=None, max_own=None):
        own = max([n - self.prefixes[g] for n, g in zip(self.lens, self.of)] + [0])
        return b.make_groups(cu_groups_host=self.cu_groups, cu_groups=dev(self.cu_groups), prefix_lens=dev(self.prefixes),
                             max_prefix_len=(self.loose or max(self.prefixes)) if max_prefix is None else max_prefix, max_own_len=own if max_own is None else max_own)

    def want(self, layer=0, causal=True, scale=None):
        k, v = self.cache.values(layer)
        return srv.attend_shared(cu_.f64(self.q), k, v, self.cache.table, self.lens, self.cu, self.cu_groups, self.prefixes, causal=causal, scale=scale)

    def bits(self):
        """Bits of the weights of shared rows, token by token."""
        rows = [sum(n for n, h in zip(self.news, self.of) if h == g) * self.n_q // self.cache.k.shape[2] for g in range(len(self.members))]
        return [16 if rows[g] <= 64 else 8 for r, g in enumerate(self.of) for _ in range(self.news[r])]


def shared_workspace(batch, groups, pages):
    """Of exactly the bytes asked for, NaN were they read as floats, with a pattern behind them."""
    n = b.codecomp_attend_shared_workspace_bytes(batch, groups, pages)
    whole = torch.full((n + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    whole[n:] = 0xA5
    return whole[:n], whole[n:]


def check_shared(f, *, causal=True, layer=0, softmax_scale=0.0, max_kv=None, max_prefix=None, max_own=None):
    batch = f.batch(causal=causal, softmax_scale=softmax_scale, max_kv=max_kv)
    pages, groups = f.cache.pages(), f.groups(max_prefix, max_own)
    ws, guard = shared_workspace(batch, groups, pages)
    out = torch.full((f.T + 3, f.n_q, f.cache.d), 7.0, dtype=torch.bfloat16, device="cuda")          # rows behind the last token stay
    lse = torch.full((f.T + 3, f.n_q), 7.0, dtype=torch.float32, device="cuda")
    b.codecomp_attend_shared(f.q, batch, groups, pages, layer, out[: f.T], ws, lse=lse[: f.T])
    want = f.want(layer, causal, softmax_scale or None)
    fine = np.array(f.bits()) == 16
    for these, weight_bits in ((fine, 16), (~fine, 8)):
        if these.any():
            at = torch.from_numpy(these).cuda()
            cu_.assert_attended(out[: f.T][at], lse[: f.T][at], tuple(x[these] for x in want), f.cache.d, weight_bits)
    assert bool((out[f.T:] == 7.0).all()) and bool((lse[f.T:] == 7.0).all()) and bool((guard == 0xA5).all())
    again = torch.empty_like(out)
    ws.fill_(0x7F)
    b.codecomp_attend_shared(f.q, batch, groups, pages, layer, again[: f.T], ws)                       # without lse: the same bits
    assert torch.equal(again[: f.T], out[: f.T])
    return out[: f.T], lse[: f.T]


# members of the groups, shared rows, new tokens and own rows of every request, query heads, KV heads, head_dim, page, 8 bits
SHARED = [
    ([1], [1], [1], [1], 1, 1, 64, 16, False), ([2], [0], [1, 1], [5, 33], 4, 2, 128, 16, False), ([3], [64], [1, 1, 1], [0, 0, 0], 4, 2, 128, 16, False),
    ([4], [133], [1] * 4, [1, 40, 7, 129], 28, 4, 128, 64, False), ([2, 3], [700, 31], [1, 2, 1, 0, 3], [4, 2, 60, 9, 3], 14, 2, 128, 32, True),
    ([3, 0, 1, 2], [257, 90, 16, 129], [1, 4, 2, 1, 1, 9], [300, 4, 2, 90, 1, 9], 8, 2, 64, 8, False), ([2], [1030], [1, 1], [3, 600], 7, 1, 64, 1, True),
    # more than 64 rows together: blocks of 256
    ([12], [333], [1] * 12, [1, 2, 3, 60, 0, 31, 32, 33, 100, 5, 64, 1], 28, 4, 128, 64, False), ([40], [65], [1] * 40, list(range(1, 41)), 14, 2, 128, 16, True),
    ([9, 11], [1000, 129], [1] * 20, [7] * 20, 8, 1, 64, 4, False), ([17], [2100], [3] * 17, [3, 50] * 8 + [200], 8, 2, 64, 256, True),
    ([2, 2], [63, 640], [70, 5, 1, 40], [70, 5, 33, 90], 4, 4, 128, 16, False), ([3], [500], [300, 1, 129], [300, 20, 200], 7, 1, 128, 32, False),
    # both kinds
    ([2, 30, 1], [300, 200, 77], [1] * 33, [3] * 33, 8, 2, 128, 16, False), ([1, 2, 20], [130, 0, 900], [1, 8, 0] + [1] * 20, [2, 8, 1] + [5] * 20, 32, 8, 128, 32, True)]


@pytest.mark.parametrize("members, prefixes, news, owns, n_q, n_kv, d, page, fp8", SHARED, ids=range(len(SHARED)))
@pytest.mark.parametrize("loose", [0, 1100, 70000])
@pytest.mark.parametrize("causal", [True, False])
def test_shared(members, prefixes, news, owns, n_q, n_kv, d, page, fp8, causal, loose):
    rng = np.random.default_rng([sum(prefixes), sum(owns), n_q, page])
    f = Forked(rng, members, prefixes, news, [max(o, n) for o, n in zip(owns, news)] if causal else owns, n_q=n_q, n_kv=n_kv, d=d, page=page, fp8=fp8, loose=loose)
    check_shared(f, causal=causal)


@pytest.mark.parametrize("case", [4, 7, 13])
@pytest.mark.parametrize("max_prefix, max_own", [(5000, 3000), (60000, 900), (1000, 60000)])
def test_shared_with_loose_bounds(case, max_prefix, max_own):
    """Chunks that no request has rows in, and different numbers of them for the two kinds of groups."""
    members, prefixes, news, owns, n_q, n_kv, d, page, fp8 = SHARED[case]
    rng = np.random.default_rng([case, max_prefix])
    f = Forked(rng, members, prefixes, news, [max(o, n) for o, n in zip(owns, news)], n_q=n_q, n_kv=n_kv, d=d, page=page, fp8=fp8, width_more=60000 // page + 1)
    check_shared(f, max_kv=60000, max_prefix=max_prefix, max_own=max_own)


@pytest.mark.parametrize("members, news", [([3], [1, 1, 1]), ([30], [1] * 30)])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page", [8, 32])
@pytest.mark.parametrize("loose", [0, 1100, 70000])
def test_shared_pages_that_are_not_held_and_lengths_out_of_range(members, news, fp8, page, loose):
    rng = np.random.default_rng([41, members[0], page])
    n = members[0]
    f = Forked(rng, members, [700], news, [40] * n, n_q=8, n_kv=2, d=64, page=page, fp8=fp8, wrong_entries=False, loose=loose)
    f.cache.table[0, [1, 5, 6]] = [-1, f.cache.n_pages, -(2**31)]
    f.cache.table[1, (700 + page - 1) // page] = 2**31 - 1
    check_shared(f)
    # lengths are cut to what the host said
    batch, pages, groups = f.batch(), f.cache.pages(), f.groups()
    ws, guard = shared_workspace(batch, groups, pages)
    out, lse, again, lse2 = (torch.empty_like(f.q) if i % 2 == 0 else torch.empty(f.T, 8, device="cuda") for i in range(4))
    b.codecomp_attend_shared(f.q, batch, groups, pages, 0, out, ws, lse=lse)
    groups._keep[2].fill_(2**31 - 1)
    batch._keep[2].fill_(2**31 - 1)
    b.codecomp_attend_shared(f.q, batch, groups, pages, 0, again, ws, lse=lse2)
    assert bool((guard == 0xA5).all())
    if not loose:                                                       # else they are cut to more rows than there are
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    groups._keep[2].fill_(-5)
    batch._keep[2].fill_(-5)
    b.codecomp_attend_shared(f.q, batch, groups, pages, 0, again, ws, lse=lse2)
    assert bool((again == 0).all()) and bool(torch.isneginf(lse2).all())


@pytest.mark.parametrize("members, news, n_q", [([3], [1, 4, 1], 8), ([30], [1] * 30, 8), ([2], [60, 33], 4)])
@pytest.mark.parametrize("fp8, d", [(False, 128), (True, 64)])
@pytest.mark.parametrize("loose", [0, 1100, 70000])
def test_shared_garbage_in_places_that_are_not_seen(members, news, n_q, fp8, d, loose):
    """NaN in rows behind the last one of a request, in the others' copies of the page that the shared rows end in, and in pages that are nobody's."""
    rng = np.random.default_rng([42, members[0], d])
    n, prefix = members[0], 333
    f = Forked(rng, members, [prefix], news, [x + int(rng.integers(0, 70)) for x in news], n_q=n_q, n_kv=2, d=d, page=32, fp8=fp8, loose=loose)
    out, lse = check_shared(f)
    seen = np.zeros((f.cache.n_pages, 32), bool)
    for r in range(n):
        for j in range(f.lens[r]):
            if r == 0 or j >= prefix:
                p, at = orc.place(f.cache.table, r, j, 32, f.cache.n_pages)
                seen[p, at] = True
    bad = torch.from_numpy(~seen).cuda()[None, :, None, :, None]
    for x in (f.cache.k, f.cache.v):
        raw = x.view(torch.uint8) if fp8 else x.view(torch.int16)
        raw.copy_(torch.where(bad, torch.full_like(raw, 0x7F if fp8 else 0x7FC0), raw))
    again, lse2 = check_shared_bits(f)
    assert torch.equal(again, out) and torch.equal(lse2, lse)


def check_shared_bits(f, causal=True):
    batch, pages, groups = f.batch(causal=causal), f.cache.pages(), f.groups()
    ws, _ = shared_workspace(batch, groups, pages)
    out, lse = torch.empty_like(f.q), torch.empty(f.T, f.n_q, device="cuda")
    b.codecomp_attend_shared(f.q, batch, groups, pages, 0, out, ws, lse=lse)
    return out, lse


@pytest.mark.parametrize("members, news, n_q", [([3], [1, 4, 1], 8), ([30], [1] * 30, 8), ([2], [60, 33], 4), ([3], [90, 40, 1], 3)])
@pytest.mark.parametrize("fp8, d, page", [(False, 128, 32), (True, 64, 8), (False, 64, 256)])
@pytest.mark.parametrize("loose", [0, 1100, 70000])
def test_shared_infinities_and_nan_among_values_that_are_seen(members, news, n_q, fp8, d, page, loose):
    """One element of one value row: that element of every token that sees the row is infinite or NaN, everything else keeps its bits."""
    rng = np.random.default_rng([43, members[0], d])
    prefix = 205
    f = Forked(rng, members, [prefix], news, [x + 37 for x in news], n_q=n_q, n_kv=1, d=d, page=page, fp8=fp8, wrong_entries=False, loose=loose)
    clean, lse = check_shared_bits(f)
    raw = f.cache.v.view(torch.uint8) if fp8 else f.cache.v
    r = 1
    own = f.lens[r] - news[r]                                           # row of the request's first new token
    for owner, key in [(0, 0), (0, prefix - 1), (r, prefix), (r, own - 1), (r, own), (r, own + news[r] // 2), (r, f.lens[r] - 1)]:
        p, at = orc.place(f.cache.table, owner, key, page, f.cache.n_pages)
        for x in [0x7F] if fp8 else [float("nan"), float("inf"), -float("inf")]:
            keep, e = raw[0, p, 0, at].clone(), int(rng.integers(d))
            raw[0, p, 0, at, e] = x
            got, got_lse = check_shared_bits(f)
            raw[0, p, 0, at] = keep
            hit = torch.zeros_like(got, dtype=torch.bool)
            if key < prefix:
                hit[:, :, e] = True
            else:
                hit[int(f.cu[r]) + max(0, key - own): int(f.cu[r + 1]), :, e] = True
            assert not bool(torch.isfinite(got[hit]).any()), (key, x)
            assert torch.equal(got[~hit], clean[~hit]) and torch.equal(got_lse, lse), (key, x)


@pytest.mark.parametrize("members, news, n_q", [([3], [1, 4, 1], 8), ([30], [1] * 30, 8), ([3], [90, 40, 1], 3)])
@pytest.mark.parametrize("fp8, d", [(False, 128), (True, 64)])
@pytest.mark.parametrize("loose", [0, 1100, 70000])
def test_shared_nan_among_keys_that_are_seen(members, news, n_q, fp8, d, loose):
    """A NaN in one key: tokens that see it have NaN everywhere, the others keep their bits."""
    rng = np.random.default_rng([53, members[0], d])
    prefix = 205
    f = Forked(rng, members, [prefix], news, [x + 37 for x in news], n_q=n_q, n_kv=1, d=d, page=16, fp8=fp8, wrong_entries=False, loose=loose)
    clean, lse = check_shared_bits(f)
    raw = f.cache.k.view(torch.uint8) if fp8 else f.cache.k
    r, own = 1, f.lens[1] - news[1]
    for owner, key in [(0, 0), (0, prefix - 1), (r, prefix), (r, own), (r, f.lens[r] - 1)]:
        p, at = orc.place(f.cache.table, owner, key, 16, f.cache.n_pages)
        keep = raw[0, p, 0, at].clone()
        raw[0, p, 0, at, 3] = 0x7F if fp8 else float("nan")
        got, got_lse = check_shared_bits(f)
        raw[0, p, 0, at] = keep
        hit = torch.zeros(f.T, dtype=torch.bool, device="cuda")
        hit[slice(None) if key < prefix else slice(int(f.cu[r]) + max(0, key - own), int(f.cu[r + 1]))] = True
        assert bool(torch.isnan(got[hit]).all()) and bool(torch.isnan(got_lse[hit]).all()), key
        assert torch.equal(got[~hit], clean[~hit]) and torch.equal(got_lse[~hit], lse[~hit]), key


@pytest.mark.parametrize("loose", [0, 1100, 70000])
def test_shared_strides_scale_layers_and_another_stream(loose):
    rng = np.random.default_rng(44)
    f = Forked(rng, [3, 9], [100, 230], [1, 2, 1] + [1] * 9, [9] * 12, n_q=8, n_kv=2, d=64, page=16, layers=3, loose=loose)
    check_shared(f, layer=2, softmax_scale=0.3)
    out, lse = check_shared(f, layer=1)
    fused, wide = torch.zeros((f.T, 12, 64), dtype=torch.bfloat16, device="cuda"), torch.full((f.T, 9, 72), 5.0, dtype=torch.bfloat16, device="cuda")
    fused[:, :8] = f.q
    x = f.batch(q_stride_tok=12 * 64, out_stride_tok=9 * 72, out_stride_head=72)
    pages, groups = f.cache.pages(), f.groups()
    ws, _ = shared_workspace(x, groups, pages)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.codecomp_attend_shared(fused[:, :8], x, groups, pages, 1, wide[:, :8, :64], ws)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(wide[:, :8, :64], out) and bool((wide[:, 8] == 5.0).all()) and bool((wide[:, :, 64:] == 5.0).all())


@pytest.mark.parametrize("members, n_q", [([4], 8), ([30], 8), ([2, 28], 8)])
@pytest.mark.parametrize("loose", [0, 1100, 70000])
def test_shared_captured_calls_follow_lengths_and_tables(members, n_q, loose):
    rng = np.random.default_rng([45, members[0]])
    n = sum(members)
    f = Forked(rng, members, [300 + 17 * g for g in range(len(members))], [1] * n, [30] * n, n_q=n_q, n_kv=2, d=128, page=16, wrong_entries=False, loose=loose)
    batch, pages, groups = f.batch(), f.cache.pages(), f.groups(max_own=60)
    ws, _ = shared_workspace(batch, groups, pages)
    out, lse = torch.empty_like(f.q), torch.empty(f.T, n_q, device="cuda")
    b.codecomp_attend_shared(f.q, batch, groups, pages, 0, out, ws, lse=lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.codecomp_attend_shared(f.q, batch, groups, pages, 0, out, ws, lse=lse)
    full = list(f.prefixes)
    for turn in range(4):
        f.prefixes = [max(0, p - 31 * turn) for p in full]
        f.lens = [f.prefixes[g] + 1 + (7 * r + 11 * turn) % 30 for r, g in enumerate(f.of)]
        groups._keep[2].copy_(dev(f.prefixes))
        batch._keep[2].copy_(dev(f.lens))
        f.q.copy_(cu_.bf16(rng.standard_normal(f.q.shape)))
        out.fill_(3.0)
        graph.replay()
        got, got_lse = out.clone(), lse.clone()
        b.codecomp_attend_shared(f.q, batch, groups, pages, 0, out, ws, lse=lse)
        assert torch.equal(out, got) and torch.equal(lse, got_lse)
        cu_.assert_attended(got, got_lse, f.want(), 128, min(f.bits()))


def test_shared_without_tokens_and_many_groups():
    rng = np.random.default_rng(46)
    f = Forked(rng, [2], [10], [0, 0], [5, 6], n_q=4, n_kv=2, d=64, page=16)
    assert b.codecomp_attend_shared_workspace_bytes(f.batch(), f.groups(), f.cache.pages()) == 0
    b.codecomp_attend_shared(f.q, f.batch(), f.groups(), f.cache.pages(), 0, torch.empty_like(f.q), None)
    members = [int(x) for x in rng.integers(0, 3, 300)]
    n = sum(members)
    f = Forked(rng, members, [int(x) for x in rng.integers(0, 40, 300)], [int(x) for x in rng.integers(0, 3, n)], [int(x) for x in rng.integers(3, 20, n)], n_q=4, n_kv=2, d=64, page=16)
    check_shared(f)


@pytest.mark.parametrize("page, d", [(16, 64), (1, 128)])
@pytest.mark.parametrize("n_groups, most", [(90, 3), (40, 5), (700, 2)])
def test_shared_many_groups_and_prompts(n_groups, most, page, d):
    """More groups and requests than a wave has lanes, and than a workgroup has threads, some of them empty or without tokens; rows that fill blocks, and that do not."""
    rng = np.random.default_rng([52, n_groups, d])
    members = [int(x) for x in rng.integers(0, most, n_groups)]
    n = sum(members)
    news = [int(x) for x in rng.choice([0, 1, 1, 2, 9, 40], n)]
    news[n // 2] = 300
    f = Forked(rng, members, [int(x) for x in rng.integers(0, 150, n_groups)], news, [x + int(rng.integers(0, 70)) for x in news], n_q=4, n_kv=2, d=d, page=page, loose=70000 // (1 + n_groups // 100))
    check_shared(f)


def test_shared_very_many_steps_over_short_caches():
    """Enough of them that sharing pays where nothing is long; and a prompt beside many of them, for whose rows most workgroups would be empty."""
    rng = np.random.default_rng(54)
    for members, more in ((([260] * 2), []), ([300], [1, 600])):
        n = sum(members) + len(more)
        news = [1] * sum(members) + more
        f = Forked(rng, members + [1] * len(more), [200] * (len(members) + len(more)), news, [x + int(rng.integers(0, 60)) for x in news], n_q=16, n_kv=4, d=64, page=16, width_more=60)
        check_shared(f, max_kv=1000, max_prefix=400 if not more else 200, max_own=100 if not more else 620)


# requests that have their groups' tables, and no new tokens; groups of 33 to 64 rows under a loose bound (weights of 16 bits in the kernel for many rows); own rows that are joined
# in one workgroup although there are many of them
@pytest.mark.parametrize("members, prefixes, news, own, n_q, n_kv, d, page, bounds", [
    ([3, 30], [140, 333], [0, 1, 2] + [0] + [1] * 29, 9, 8, 2, 64, 16, {}),
    ([9], [700], [1] * 9, 40, 28, 4, 128, 32, dict(max_kv=70000, max_prefix=60000, max_own=300)),
    ([16, 10, 3], [65, 700, 90], [4] * 16 + [4] * 10 + [4] * 3, 60, 8, 8, 64, 8, dict(max_kv=70000, max_prefix=60000, max_own=9000)),
    ([60], [300], [1] * 60, 1500, 16, 4, 64, 64, {}), ([60], [300], [2] * 60, 700, 32, 4, 128, 16, dict(max_kv=9000, max_own=3000)),
    # own rows in the kernel for many rows: of single tokens and prompts beside one another, causal within a block and behind its end, shared rows that end inside a tile
    ([9, 2, 1], [205, 90, 0], [1, 70, 0, 3, 1, 33, 1, 9, 1, 1, 2, 150], 300, 8, 2, 64, 16, {}), ([5, 4], [1000, 63], [300, 1, 129, 2, 40, 1, 1, 1, 90], 400, 14, 2, 128, 1, {}),
    ([30], [129], [1, 9] * 15, 200, 16, 4, 128, 128, dict(max_kv=5000, max_prefix=5000, max_own=4000)), ([2, 1], [320, 64], [65, 64, 300], 1, 4, 4, 64, 64, {}),
    # prompts with many rows of their own: in chunks, the causal end in the last ones or before them
    ([2, 2], [150, 63], [300, 1, 70, 5], 5000, 4, 2, 64, 16, {}), ([3], [1000], [260, 40, 1], 9000, 7, 1, 128, 64, {}), ([1, 1], [0, 5], [900, 700], 3000, 2, 1, 128, 8, dict(max_kv=40000, max_own=30000))])
@pytest.mark.parametrize("loose", [0, 1100, 70000])
@pytest.mark.parametrize("causal", [True, False])
def test_shared_kinds_of_groups(members, prefixes, news, own, n_q, n_kv, d, page, bounds, causal, loose):
    rng = np.random.default_rng([47, own, page])
    owns = [max(n, int(x)) for n, x in zip(news, rng.integers(0, own, sum(members)))]
    if loose:
        bounds = {"max_own": min(bounds["max_own"], loose)} if "max_own" in bounds else {}
    more = (bounds.get("max_kv", 0)) // page
    check_shared(Forked(rng, members, prefixes, news, owns, n_q=n_q, n_kv=n_kv, d=d, page=page, width_more=more, loose=loose), causal=causal, **bounds)


@pytest.mark.parametrize("loose", [0, 1100, 70000])
def test_shared_pool_with_strides_of_its_own(loose):
    rng = np.random.default_rng(48)
    f = Forked(rng, [3, 30], [140, 333], [1, 3, 2] + [1] * 30, [7] * 33, n_q=8, n_kv=2, d=64, page=16, layers=2, loose=loose)
    dense, lse = check_shared(f, layer=1)
    f.cache.k, f.cache.v = (t.permute(1, 3, 0, 2, 4).contiguous().permute(2, 0, 3, 1, 4) for t in (f.cache.k, f.cache.v))
    again, lse2 = check_shared(f, layer=1)
    assert torch.equal(again, dense) and torch.equal(lse, lse2)


@pytest.mark.parametrize("members", [[3], [30], [2, 28]])
@pytest.mark.parametrize("loose", [0, 1100, 70000])
def test_shared_two_graphs_and_two_streams(members, loose):
    """Graphs replayed one after the other on one workspace; calls at the same time on workspaces of their own."""
    rng = np.random.default_rng([49, members[0]])
    n = sum(members)
    fs = [Forked(rng, members, [500 + 33 * g for g in range(len(members))], [1] * n, [70] * n, n_q=8, n_kv=2, d=64, page=16, loose=loose) for _ in range(2)]
    want = [check_shared(f) for f in fs]
    calls = [(f.batch(), f.cache.pages(), f.groups()) for f in fs]
    shared = shared_workspace(calls[0][0], calls[0][2], calls[0][1])[0]
    alone = [shared_workspace(x, g, p)[0] for x, p, g in calls]
    outs, lses, graphs = [torch.empty_like(f.q) for f in fs], [torch.empty(f.T, 8, device="cuda") for f in fs], [torch.cuda.CUDAGraph() for _ in fs]
    torch.cuda.synchronize()
    for i, (x, p, g) in enumerate(calls):
        with torch.cuda.graph(graphs[i]):
            b.codecomp_attend_shared(fs[i].q, x, g, p, 0, outs[i], shared, lse=lses[i])
    for turn in range(6):
        outs[turn % 2].fill_(9.0)
        graphs[turn % 2].replay()
        assert torch.equal(outs[turn % 2], want[turn % 2][0]) and torch.equal(lses[turn % 2], want[turn % 2][1])
    streams = [torch.cuda.Stream() for _ in fs]
    torch.cuda.synchronize()
    for turn in range(20):
        for i, (x, p, g) in enumerate(calls):
            with torch.cuda.stream(streams[i]):
                outs[i].fill_(9.0)
                b.codecomp_attend_shared(fs[i].q, x, g, p, 0, outs[i], alone[i], lse=lses[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], want[i][0]) and torch.equal(lses[i], want[i][1])


def far_away(cache):
    """The same rows where offsets are beyond 2^32 bytes and elements: in the last pages of a pool of 2^33 elements, and in its second layer."""
    n = cache.n_pages
    _, _, h, page, d = cache.k.shape
    more = 2**32 // (h * page * d) + 1
    big = [torch.empty((2, more + n, h, page, d), dtype=cache.k.dtype, device="cuda") for _ in range(2)]
    for to, x in zip(big, (cache.k, cache.v)):
        to[1, more:] = x[0]
    cache.k, cache.v = big
    cache.table = np.where(cache.table >= 0, cache.table + more, -1).astype(np.int32)
    cache.n_pages += more


@pytest.mark.parametrize("members", [[3], [30]])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("loose", [0, 1100, 70000])
def test_shared_offsets_beyond_32_bits(members, fp8, loose):
    rng = np.random.default_rng([50, members[0]])
    n = members[0]
    f = Forked(rng, members, [300], [1] * n, [20] * n, n_q=8, n_kv=2, d=64, page=16, fp8=fp8, wrong_entries=False, loose=loose)
    near, near_lse = check_shared(f)
    far_away(f.cache)
    batch, pages, groups = f.batch(), f.cache.pages(), f.groups()
    out, lse = torch.empty_like(f.q), torch.empty(f.T, 8, device="cuda")
    b.codecomp_attend_shared(f.q, batch, groups, pages, 1, out, shared_workspace(batch, groups, pages)[0], lse=lse)
    assert torch.equal(out, near) and torch.equal(lse, near_lse)


# ---------------------------------------------------------------- sums of attention weights

def mass_setup(rng, lens, news, n_q, *, n_kv, d, page, fp8=False, layers=1, first=None, width=None, causal=True, softmax_scale=0.0, max_kv=None, sharp=1.0, width_more=0):
    c = cu_.Cache(rng, lens, n_kv=n_kv, d=d, page=page, fp8=fp8, layers=layers, width_more=width_more, **scales(fp8))
    batch, cu = cu_.make_batch(c, news, n_q, causal=causal, softmax_scale=softmax_scale, max_kv=max_kv)
    q = cu_.bf16(rng.standard_normal((int(cu[-1]), n_q, d)) * sharp).cuda()
    width = max(list(lens) + [1]) + 3 if width is None else width
    sums = torch.from_numpy(rng.random((layers, len(lens), n_kv, width), dtype=np.float32)).cuda()
    return c, batch, cu, q, sums


def mass_tolerance(want, added, reach, decay, old, rows):
    """A weight is off by its logit's error (d products and sums of fp32 of half a step each, and those of the logit and the log-sum-exp, which are
    scaled and subtracted) and that of exp2, 2^-21; the sum of `rows` positive weights by at most `rows` half steps (fewer, in fact); then the sum's share, its product and
    its addition to what stood there."""
    half = 2.0 ** -24
    return added * (2 * (half * reach + 2.0 ** -21) + half * (rows + 4)) + 2 * half * (np.abs(want) + np.abs(decay * old)) + 2.0 ** -140


def mass_workspace(batch, pages, mass):
    n = b.codecomp_attend_mass_workspace_bytes(batch, pages, mass)
    whole = torch.full((n + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    whole[n:] = 0xA5
    return whole[:n] if n else None, whole[n:]


def check_mass(rng, lens, news, n_q, *, layer=0, decay=1.0, first=None, causal=True, softmax_scale=0.0, lose=(), spoil=None, **kw):
    c, batch, cu, q, sums = mass_setup(rng, lens, news, n_q, causal=causal, softmax_scale=softmax_scale, **kw)
    if spoil is not None:
        spoil(c)
        batch._keep[3].copy_(c.dev_table())
    pages, m = c.pages(), b.make_mass(sums)
    k, v = c.values(layer)
    _, lse, _, _ = orc.attend(cu_.f64(q), k, v, c.table, lens, cu, max_kv_len=batch.max_kv_len, causal=causal, scale=softmax_scale or None)
    lse = lse.astype(np.float32)
    for t, h in lose:
        lse[t, h] = -np.inf
    before = sums.cpu().numpy().copy()
    ws, guard = mass_workspace(batch, pages, m)
    f = None if first is None else dev(first)
    b.codecomp_attend_mass(q, torch.from_numpy(lse).cuda(), batch, pages, layer, m, ws, first=f, decay=decay)
    got = sums.cpu().numpy()
    want, added, reach = srv.attend_mass(cu_.f64(q), lse, k, c.table, lens, cu, before[layer], first=first, decay=decay, causal=causal, scale=softmax_scale or None)
    rows = max(news) * n_q // c.k.shape[2]
    tol = mass_tolerance(want, added, reach, decay, before[layer], rows)
    off = np.abs(got[layer] - want)
    assert np.all(off <= tol), (float((off / tol).max()), np.unravel_index(np.argmax(off / tol), off.shape))
    touched = np.zeros(before.shape, bool)
    for r, n in enumerate(lens):
        if news[r] > 0:
            touched[layer, r, :, (0 if first is None else max(0, first[r])):n] = True
    assert np.array_equal(got[~touched], before[~touched]) and bool((guard == 0xA5).all())
    # the same bits again
    sums.copy_(torch.from_numpy(before))
    if ws is not None:
        ws.fill_(0x7F)
    b.codecomp_attend_mass(q, torch.from_numpy(lse).cuda(), batch, pages, layer, m, ws, first=f, decay=decay)
    assert np.array_equal(sums.cpu().numpy(), got)
    return c, batch, q, sums, got, added


MASS = [
    ([1], [1], 1, 1, 64, 16, False), ([0, 1, 2, 31, 32, 33, 63, 64, 65, 700], [1] * 10, 4, 2, 128, 16, False), ([257, 129, 1030], [1, 1, 1], 28, 4, 128, 64, False),
    ([257, 129, 1030], [1, 1, 1], 14, 2, 128, 32, True), ([90, 500, 17, 300], [2, 8, 1, 0], 16, 2, 64, 1, False), ([90, 500, 17, 300], [2, 4, 1, 3], 32, 8, 128, 128, True),
    ([40, 16, 5], [64, 16, 5], 1, 1, 128, 8, False), ([2000], [9], 7, 1, 128, 256, False), ([3001], [16], 4, 1, 64, 16, True),
    # more than 64 rows
    ([65], [65], 1, 1, 64, 16, False), ([300], [300], 7, 1, 128, 16, False), ([700, 130], [100, 130], 8, 2, 128, 64, True), ([700, 64, 20, 900], [70, 64, 20, 1], 14, 2, 64, 1, False),
    ([50, 10, 333], [90, 90, 333], 4, 4, 128, 32, False), ([1100], [33], 28, 4, 128, 128, False), ([500, 90], [200, 90], 4, 2, 64, 8, True), ([600], [600], 6, 1, 64, 64, False),
    ([0, 129, 128, 127], [80, 80, 80, 80], 6, 3, 64, 8, True), ([520], [1500], 2, 2, 128, 16, True)]


@pytest.mark.parametrize("lens, news, n_q, n_kv, d, page, fp8", MASS, ids=range(len(MASS)))
@pytest.mark.parametrize("causal", [True, False])
def test_mass(lens, news, n_q, n_kv, d, page, fp8, causal):
    rng = np.random.default_rng([sum(lens), n_q, page, 3])
    check_mass(rng, lens, news, n_q, n_kv=n_kv, d=d, page=page, fp8=fp8, causal=causal)


@pytest.mark.parametrize("max_kv", [900, 70000])
@pytest.mark.parametrize("news", [[16, 17, 64, 65, 1, 0], [16, 17, 64, 33, 1, 0], [16, 15, 1, 65, 0, 1]])
@pytest.mark.parametrize("d, page, fp8", [(128, 16, False), (64, 4, True)])
def test_mass_of_rows_around_the_numbers_that_decide(max_kv, news, d, page, fp8):
    """One query head: rows are tokens.  With a loose bound on lengths there may be much work for either kernel."""
    rng = np.random.default_rng([74, sum(news), d])
    check_mass(rng, [100, 600, 64, 900, 513, 77], news, 2, n_kv=2, d=d, page=page, fp8=fp8, first=[5, 0, 0, 512, 1, 0], decay=0.9, max_kv=max_kv, width=max_kv, width_more=70000 // page)


@pytest.mark.parametrize("lens, news, n_q, d", [([300, 77, 900], [1, 1, 3], 4, 128), ([300, 77, 900], [90, 40, 1], 4, 64), ([300, 77, 900], [2, 77, 100], 14, 128)])
@pytest.mark.parametrize("first", [[0, 77, 130], [299, 0, 511], [300, 1000, -7], [31, 32, 256]])
@pytest.mark.parametrize("decay", [0.0, 0.75])
def test_mass_behind_protected_rows_and_fading(lens, news, n_q, d, first, decay):
    rng = np.random.default_rng([51, n_q, first[0]])
    check_mass(rng, lens, news, n_q, n_kv=2, d=d, page=16, first=first, decay=decay)


@pytest.mark.parametrize("news", [[1, 2], [80, 1], [100, 200]])
@pytest.mark.parametrize("fp8", [False, True])
def test_mass_layers_scale_pages_that_are_not_held_and_rows_that_see_nothing(news, fp8):
    rng = np.random.default_rng([52, news[0]])

    def spoil(c):
        c.table[0, [1, 5]] = [-1, c.n_pages]
        c.table[1, 3] = 2**31 - 1

    check_mass(rng, [300, 210], news, 4, n_kv=2, d=64, page=16, fp8=fp8, layers=3, layer=1, softmax_scale=0.21, lose=[(0, 1), (0, 0), (news[0], 3)], spoil=spoil)


@pytest.mark.parametrize("news", [[1, 1], [90, 150]])
def test_mass_sums_are_those_of_attention(news):
    """A call's weights of one token and head add up to one: all sums of a head to tokens, whatever the lengths."""
    rng = np.random.default_rng([53, news[0]])
    c, batch, cu, q, sums = mass_setup(rng, [777, 400], news, 14, n_kv=2, d=128, page=32)
    pages, m = c.pages(), b.make_mass(sums)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    b.codecomp_attend(q, batch, pages, 0, out, cu_.workspace(batch, pages), lse=lse)
    sums.zero_()
    b.codecomp_attend_mass(q, lse, batch, pages, 0, m, mass_workspace(batch, pages, m)[0])
    total = sums.double().sum(-1)[0].cpu().numpy()
    assert np.allclose(total, np.array(news, float)[:, None], rtol=2.0 ** -15, atol=0)


@pytest.mark.parametrize("news, n_q", [([1, 4], 4), ([70, 90], 4), ([1, 90], 4)])
@pytest.mark.parametrize("fp8, d, page", [(False, 128, 16), (True, 64, 8)])
def test_mass_garbage_where_nothing_is_seen_and_where_it_is(news, n_q, fp8, d, page):
    """NaN keys behind the last rows and in protected rows change nothing; in a row that is seen they make its sum NaN and no other."""
    rng = np.random.default_rng([54, news[0], d])
    lens, first = [300, 207], [20, 0]
    c, batch, q, sums, got, _ = check_mass(rng, lens, news, n_q, n_kv=2, d=d, page=page, fp8=fp8, first=first)
    lse = torch.zeros(q.shape[:2], device="cuda")
    pages, m = c.pages(), b.make_mass(sums)
    ws, _ = mass_workspace(batch, pages, m)
    call = lambda: (sums.fill_(0.5), b.codecomp_attend_mass(q, lse, batch, pages, 0, m, ws, first=dev(first)), sums.clone())[2]  # noqa: E731
    clean = call()
    raw = c.k.view(torch.uint8) if fp8 else c.k
    used = np.zeros((c.n_pages, page), bool)
    for r in range(2):
        for j in range(first[r], lens[r]):
            used[orc.place(c.table, r, j, page, c.n_pages)] = True
    bad = torch.from_numpy(~used).cuda()[None, :, None, :, None]
    raw.copy_(torch.where(bad, torch.full_like(raw, 0x7F if fp8 else float("nan")), raw))
    assert torch.equal(call(), clean)
    for r, j in [(0, 20), (0, 299), (1, 100)]:
        p, at = orc.place(c.table, r, j, page, c.n_pages)
        raw[0, p, 1, at, 5] = 0x7F if fp8 else float("nan")
    x = call()
    hit = torch.zeros_like(x, dtype=torch.bool)
    for r, j in [(0, 20), (0, 299), (1, 100)]:
        hit[0, r, 1, j] = True
    assert bool(torch.isnan(x[hit]).all()) and torch.equal(x[~hit], clean[~hit])
    sums.fill_(float("nan"))                       # what is not read: sums of new rows, and any with a decay of zero
    b.codecomp_attend_mass(q, lse, batch, pages, 0, m, ws, first=dev(first), decay=0.0)
    assert not bool(torch.isnan(sums[0, 0, 0, 20:300]).any()) and bool(torch.isnan(sums[0, 0, 0, :20]).all())


@pytest.mark.parametrize("news", [[1, 3, 1], [90, 40, 70]])
def test_mass_captured_strided_and_on_another_stream(news):
    rng = np.random.default_rng([55, news[0]])
    c, batch, cu, q, _ = mass_setup(rng, [400, 300, 200], news, 8, n_kv=2, d=64, page=16)
    wide = torch.zeros((3, 2, 2, 512), device="cuda")                    # [requests][heads][layers][rows] in memory
    sums = wide.permute(2, 0, 1, 3)[:, :, :, 7:450]
    pages, first, dense = c.pages(), dev([3, 0, 100]), torch.zeros((1, 3, 2, 443), device="cuda")
    pages2, m, dm = b.make_pages(torch.cat([c.k, c.k]), torch.cat([c.v, c.v])), b.make_mass(sums), b.make_mass(dense)
    ws, _ = mass_workspace(batch, pages, dm)
    lse = torch.from_numpy(rng.standard_normal(q.shape[:2]).astype(np.float32)).cuda() + 5.0
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        b.codecomp_attend_mass(q, lse, batch, pages2, 1, m, ws, first=first, decay=0.5)
    for turn in range(4):
        batch._keep[2].copy_(dev([400 - 37 * turn, 300 - turn, 200]))
        first.fill_(5 * turn)
        q.copy_(cu_.bf16(rng.standard_normal(q.shape)))
        graph.replay()
        b.codecomp_attend_mass(q, lse, batch, pages, 0, dm, ws, first=first, decay=0.5)
        assert torch.equal(sums[1], dense[0])
    assert bool((wide[:, :, 0] == 0).all()) and bool((wide[..., :7] == 0).all()) and bool((wide[..., 450:] == 0).all())


@pytest.mark.parametrize("lens, news, n_q, n_kv, d, page, fp8, first", [
    ([3000, 5, 0, 1500, 64, 700], [1, 1, 1, 0, 5, 2], 8, 2, 128, 16, False, [130, 0, 5, 0, 64, -3]), ([3000, 5, 0, 1500, 64, 700], [1, 1, 1, 0, 5, 2], 8, 2, 64, 4, True, [1, 4, 0, 9, 0, 513]),
    ([3000, 5, 0, 1500, 64, 700], [1, 1, 1, 0, 5, 2], 12, 2, 64, 64, True, None), ([2100, 40, 777], [3, 2, 4], 14, 2, 128, 1, False, [2099, 41, 12]),
    ([23, 0, 41, 7] * 75, [1, 1, 2, 1] * 75, 8, 8, 128, 16, False, None), ([23, 0, 41, 7] * 75, [1, 1, 0, 3] * 75, 8, 8, 64, 8, False, [3, 1, 32, 7] * 75),
    ([9000, 4001], [1, 2], 8, 8, 128, 32, True, [0, 257])])
def test_mass_of_few_rows_in_equal_shares(lens, news, n_q, n_kv, d, page, fp8, first):
    """A bound on lengths under which there may be many keys: strips of all requests and heads in a row, several of them for a workgroup, or few."""
    rng = np.random.default_rng([56, len(lens), n_q, page])
    check_mass(rng, lens, news, n_q, n_kv=n_kv, d=d, page=page, fp8=fp8, first=first, decay=0.5, max_kv=70000, width=70000, width_more=70000 // page + 1)


def test_mass_of_a_few_among_very_many_requests():
    """More requests and heads than a launch has workgroups; those with a token as they would be alone."""
    rng = np.random.default_rng(62)
    H, n, who = 1024, 20000, [0, 7000, 19999]
    k = torch.from_numpy(rng.standard_normal((1, 4, H, 16, 64), dtype=np.float32)).bfloat16().cuda()
    q, lse = cu_.bf16(rng.standard_normal((3, H, 64))).cuda(), torch.full((3, H), 3.0, device="cuda")
    pages, sums = b.make_pages(k, k), torch.full((1, n, H, 16), 0.25, device="cuda")
    lens, table, news = np.full(n, 5), np.zeros((n, 1)), np.zeros(n, int)
    lens[who], table[who, 0], news[who] = [16, 1, 9], [3, 1, 2], 1
    make = lambda news, lens, table: b.make_batch(n_q_heads=H, cu_q_host=cum(news), cu_q=dev(cum(news)), kv_lens=dev(lens), table=dev(table), max_kv_len=16)  # noqa: E731
    b.codecomp_attend_mass(q, lse, make(news, lens, table), pages, 0, b.make_mass(sums), None, decay=0.5)
    alone = torch.full((1, 3, H, 16), 0.25, device="cuda")
    b.codecomp_attend_mass(q, lse, make(news[who], lens[who], table[who]), pages, 0, b.make_mass(alone), None, decay=0.5)
    assert torch.equal(sums[:, who], alone) and not bool((alone[0, 0] == 0.25).any())
    sums[:, who] = 0.25
    assert bool((sums == 0.25).all())


@pytest.mark.parametrize("d, fp8", [(64, True), (128, False)])
def test_mass_of_many_short_prompts(d, fp8):
    """More blocks of keys than workgroups: several for each, of requests and heads one after the other, some without any, and a few rows here and there."""
    rng = np.random.default_rng([57, d])
    lens, news = [int(x) for x in rng.integers(34, 80, 220)], [33, 34, 33, 0, 33, 1, 33, 36, 33, 33] * 22
    check_mass(rng, lens, news, 4, n_kv=2, d=d, page=8, fp8=fp8, first=[0, 5, 0, 0, 0, 0, 90, 0, 33, 1] * 22)


@pytest.mark.parametrize("news", [[1, 3], [40, 60]])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_mass_queries_and_sums_of_weights_that_are_no_numbers(news, bad):
    """A token and head whose log-sum-exp is NaN, or whose query has an infinity or NaN: sums of the rows that it sees are no numbers, others keep their bits."""
    rng = np.random.default_rng([58, news[0]])
    c, batch, cu, q, sums = mass_setup(rng, [333, 260], news, 8, n_kv=2, d=64, page=16)
    pages, m, lse = c.pages(), b.make_mass(sums), torch.full((sum(news), 8), 2.0, device="cuda")
    ws, _ = mass_workspace(batch, pages, m)

    def call():
        sums.fill_(0.5)
        b.codecomp_attend_mass(q, lse, batch, pages, 0, m, ws)
        return sums.clone()

    clean = call()
    t, h = news[0], 5                                                  # the second request's first token, of the second KV head
    sees = 260 - news[1] + 1
    hit = torch.zeros_like(clean, dtype=torch.bool)
    hit[0, 1, 1, :sees] = True
    keep = q[t, h, 3].clone()
    q[t, h, 3] = bad
    x = call()
    q[t, h, 3] = keep
    assert torch.equal(x[~hit], clean[~hit])
    if bad != bad:
        assert bool(torch.isnan(x[hit]).all())
    else:                                                              # the key's sign says which infinity the logit is: a weight of infinity or of zero
        assert bool(torch.isinf(x[hit]).any()) and not bool(torch.isnan(x[hit]).any())
    lse[t, h] = float("nan")
    x = call()
    assert bool(torch.isnan(x[hit]).all()) and torch.equal(x[~hit], clean[~hit])
    lse[t, h] = float("inf")                                          # no weight
    x = call()
    lse[t, h] = -float("inf")
    assert torch.equal(call(), x)


@pytest.mark.parametrize("news", [[1, 3, 1], [90, 40, 70]])
def test_mass_strides_of_queries_and_pool(news):
    rng = np.random.default_rng([59, news[0]])
    c, batch, cu, q, sums = mass_setup(rng, [400, 300, 200], news, 8, n_kv=2, d=64, page=16, layers=2)
    pages, m, lse = c.pages(), b.make_mass(sums), torch.full((sum(news), 8), 2.0, device="cuda")
    ws, _ = mass_workspace(batch, pages, m)
    before = sums.clone()
    b.codecomp_attend_mass(q, lse, batch, pages, 1, m, ws, decay=0.5)
    want = sums.clone()
    wide = torch.zeros((9, sum(news), 72), dtype=torch.bfloat16, device="cuda")
    wide[:8, :, :64] = q.transpose(0, 1)
    x, _ = cu_.make_batch(c, news, 8, q_stride_tok=72, q_stride_head=72 * sum(news))
    c.k, c.v = (t.permute(1, 3, 0, 2, 4).contiguous().permute(2, 0, 3, 1, 4) for t in (c.k, c.v))
    sums.copy_(before)
    b.codecomp_attend_mass(wide.transpose(0, 1)[:, :8, :64], lse, x, c.pages(), 1, m, ws, decay=0.5)
    assert torch.equal(sums, want)


@pytest.mark.parametrize("news", [[1, 3], [90, 40]])
@pytest.mark.parametrize("fp8", [False, True])
def test_mass_offsets_beyond_32_bits(news, fp8):
    rng = np.random.default_rng([60, news[0]])
    c, batch, cu, q, sums = mass_setup(rng, [400, 300], news, 8, n_kv=2, d=64, page=16, fp8=fp8)
    lse = torch.full((sum(news), 8), 2.0, device="cuda")
    m = b.make_mass(sums)
    ws, _ = mass_workspace(batch, c.pages(), m)
    before = sums.clone()
    b.codecomp_attend_mass(q, lse, batch, c.pages(), 0, m, ws, decay=0.5)
    far_away(c)
    batch = cu_.make_batch(c, news, 8)[0]
    at = torch.empty(2**32 + 2**31 + 2000, device="cuda").as_strided((2, 2, 2, 403), (2**32, 2**31, 1000, 1))
    at[1] = before[0]
    b.codecomp_attend_mass(q, lse, batch, c.pages(), 1, b.make_mass(at), ws, decay=0.5)
    assert torch.equal(at[1], sums[0])


def test_mass_two_graphs_and_two_streams():
    rng = np.random.default_rng(61)
    news = [90, 2, 70]
    xs = [mass_setup(rng, [700, 300, 500], news, 8, n_kv=2, d=64, page=16) for _ in range(2)]
    lse = torch.full((sum(news), 8), 4.0, device="cuda")
    ms, pages, graphs, want = [b.make_mass(x[4]) for x in xs], [x[0].pages() for x in xs], [torch.cuda.CUDAGraph() for _ in xs], []
    shared = mass_workspace(xs[0][1], pages[0], ms[0])[0]
    alone = [mass_workspace(x[1], p, m)[0] for x, p, m in zip(xs, pages, ms)]
    call = lambda i, ws: b.codecomp_attend_mass(xs[i][3], lse, xs[i][1], pages[i], 0, ms[i], ws, decay=0.0)  # noqa: E731
    for i in range(2):
        call(i, shared)
        want.append(xs[i][4].clone())
    torch.cuda.synchronize()
    for i in range(2):
        with torch.cuda.graph(graphs[i]):
            call(i, shared)
    for turn in range(6):
        xs[turn % 2][4].copy_(want[1 - turn % 2])
        xs[turn % 2][4][:, :, :, 700:] = want[turn % 2][:, :, :, 700:]
        for r, n in enumerate([700, 300, 500]):
            xs[turn % 2][4][:, r, :, n:] = want[turn % 2][:, r, :, n:]
        graphs[turn % 2].replay()
        assert torch.equal(xs[turn % 2][4], want[turn % 2])
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for turn in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                call(i, alone[i])
    torch.cuda.synchronize()
    assert all(torch.equal(xs[i][4], want[i]) for i in range(2))


# ---------------------------------------------------------------- eviction

def evict_setup(rng, lens, budgets, *, n_kv=2, d=64, page=16, fp8=False, layers=2, width=None, values="tail"):
    c = cu_.Cache(rng, lens, n_kv=n_kv, d=d, page=page, fp8=fp8, layers=layers)
    shape = (layers, len(lens), n_kv, (max(lens) + 5) if width is None else width)
    x = np.exp(2 * rng.standard_normal(shape)).astype(np.float32)
    if values == "ties":
        x = rng.integers(0, 4, shape).astype(np.float32)
    elif values == "signs":
        x = rng.choice(np.array([0.0, -0.0, 1e-45, -1e-45, np.inf, -np.inf, np.nan, -1.0, 1.0, 3e38, -3e38], np.float32), shape)
        x.view(np.uint32)[np.isnan(x)] ^= rng.integers(0, 2, int(np.isnan(x).sum())).astype(np.uint32) << 31        # NaN of both signs
    elif values == "zeros":
        x[...] = 0
    elif values == "near":
        x = (1.0 + rng.integers(0, 300, shape) * 2.0 ** -23).astype(np.float32)
    return c, x


def check_evict(rng, lens, budgets, *, recent, max_budget, first=None, elsewhere=False, spoil=None, max_kv=None, **kw):
    c, x = evict_setup(rng, lens, budgets, **kw)
    if spoil is not None:
        spoil(c)
    L, n, H, width = x.shape
    k0, v0 = (t.view(torch.uint8).cpu().numpy().copy() for t in (c.k, c.v))
    sums = torch.from_numpy(x).cuda()
    to = torch.full_like(sums, 9.0) if elsewhere else None
    kept, new_lens = torch.full((L, n, H, max_budget), 77, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    e = b.make_eviction(kv_lens=dev(lens), table=c.dev_table(), budgets=dev(budgets), max_kv_len=max(lens) if max_kv is None else max_kv, max_budget=max_budget, recent=recent,
                        first=None if first is None else dev(first))
    b.codecomp_evict(b.make_mass(sums), e, c.pages(), kept, new_lens, kept_mass=None if to is None else b.make_mass(to))
    want, want_lens = srv.evict(x, lens, budgets, recent=recent, max_budget=max_budget, first=first)
    assert np.array_equal(new_lens.cpu().numpy(), want_lens)
    assert np.array_equal(kept.cpu().numpy(), want)
    wk, wv, ws = k0.copy(), v0.copy(), (np.full_like(x, 9.0) if elsewhere else x.copy())
    for r in range(n):
        f = 0 if first is None else min(max(first[r], 0), lens[r])
        for l in range(L):
            for h in range(H):
                for i, j in enumerate(want[l, r, h]):
                    if j < 0:
                        continue
                    ws[l, r, h, f + i] = x[l, r, h, j]
                    a, t = orc.place(c.table, r, int(j), c.page, c.n_pages), orc.place(c.table, r, f + i, c.page, c.n_pages)
                    if t is not None and j != f + i:
                        wk[l, t[0], h, t[1]] = k0[l, a[0], h, a[1]] if a else 0
                        wv[l, t[0], h, t[1]] = v0[l, a[0], h, a[1]] if a else 0
    assert np.array_equal(c.k.view(torch.uint8).cpu().numpy(), wk) and np.array_equal(c.v.view(torch.uint8).cpu().numpy(), wv)
    got = (to if elsewhere else sums).cpu().numpy()
    assert np.array_equal(got.view(np.uint32), ws.view(np.uint32))
    if elsewhere:
        assert np.array_equal(sums.cpu().numpy().view(np.uint32), x.view(np.uint32))


EVICT = [
    ([1], [1], 0, 1, None), ([2, 1, 0], [1, 1, 1], 0, 1, None), ([2, 1, 0], [1, 1, 1], 1, 1, None), ([100, 40, 300], [30, 40, 41], 7, 50, None),
    ([257, 256, 255, 513], [256, 256, 256, 1], 0, 256, None), ([600, 90], [64, 64], 64, 64, None), ([600, 90], [-5, 1000], 3, 64, None),
    ([700, 300, 80], [100, 200, 10], 10, 200, [300, 301, 77]), ([700, 300, 80], [100, 200, 10], 0, 500, [700, 5000, -3]), ([1500], [1499], 1, 1499, [16]),
    ([5000, 17], [1025, 16], 100, 1030, [33, 0])]


@pytest.mark.parametrize("lens, budgets, recent, max_budget, first", EVICT, ids=range(len(EVICT)))
@pytest.mark.parametrize("elsewhere", [False, True])
def test_evict(lens, budgets, recent, max_budget, first, elsewhere):
    rng = np.random.default_rng([sum(lens), recent])
    check_evict(rng, lens, budgets, recent=recent, max_budget=max_budget, first=first, elsewhere=elsewhere)


@pytest.mark.parametrize("values", ["ties", "signs", "zeros", "near"])
@pytest.mark.parametrize("fp8, d, page, n_kv", [(False, 128, 16, 2), (True, 64, 1, 3), (True, 128, 64, 1), (False, 64, 256, 4)])
def test_evict_equal_and_special_sums(values, fp8, d, page, n_kv):
    rng = np.random.default_rng([61, d, page])
    check_evict(rng, [400, 290, 1030], [100, 7, 700], recent=5, max_budget=700, first=[0, 20, 3], values=values, fp8=fp8, d=d, page=page, n_kv=n_kv, layers=2)


def test_evict_pages_that_are_not_held():
    def spoil(c):
        c.table[0, [0, 3, 9]] = [-1, c.n_pages, 2**31 - 1]
    check_evict(np.random.default_rng(62), [300, 200], [120, 100], recent=10, max_budget=120, spoil=spoil)


@pytest.mark.parametrize("n", [1, 2, 15])
def test_evict_of_few_and_many_problems(n):
    """Rows in one stretch and in more, short requests and long ones, in one kernel and in two."""
    for layers, rows, budget in ((1, 333, 100), (20, 333, 100), (1, 150, 100), (1, 1300, 1100), (1, 9000, 300)):
        check_evict(np.random.default_rng([63, n, layers, rows]), [rows] * n, [budget] * n, recent=10, max_budget=budget, first=[7] * n, n_kv=2, d=128, layers=layers)


@pytest.mark.parametrize("n, rows, budget", [(102, 190, 60), (102, 1000, 60), (102, 1100, 60), (102, 4500, 60), (3, 2048, 70), (3, 2048, 700), (3, 2049, 1500), (3, 4097, 80), (3, 8193, 80), (3, 16385, 4000)])
@pytest.mark.parametrize("d, fp8", [(64, True), (128, False), (64, False)])
def test_evict_around_the_sizes_that_decide(n, rows, budget, d, fp8):
    """Requests that are as long as the bound, one that is not, and one that is empty."""
    rng = np.random.default_rng([71, n, rows, d])
    lens = [0, rows] + [int(x) for x in rng.integers(1, 90, n - 2)]
    check_evict(rng, lens, [budget] * n, recent=3, max_budget=budget, first=[5] * n, n_kv=4, d=d, page=16, fp8=fp8, layers=1, values="ties")


def test_evict_lengths_out_of_range_and_again():
    """Lengths are cut to what the host said; a second call has nothing to do."""
    rng = np.random.default_rng(64)
    c, x = evict_setup(rng, [200, 150], None)
    sums, table, budgets = torch.from_numpy(x).cuda(), c.dev_table(), dev([64, 64])
    kept, lens = torch.empty((2, 2, 2, 64), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    e = b.make_eviction(kv_lens=dev([2**31 - 1, -4]), table=table, budgets=budgets, max_kv_len=200, max_budget=64, recent=4)
    b.codecomp_evict(b.make_mass(sums), e, c.pages(), kept, lens)
    want, _ = srv.evict(x, [200, 0], [64, 64], recent=4, max_budget=64)
    assert lens.tolist() == [64, 0] and np.array_equal(kept.cpu().numpy(), want)
    k, s = c.k.clone(), sums.clone()
    again, lens2 = torch.empty_like(kept), torch.empty_like(lens)
    e = b.make_eviction(kv_lens=lens, table=table, budgets=budgets, max_kv_len=200, max_budget=64, recent=4)
    b.codecomp_evict(b.make_mass(sums), e, c.pages(), again, lens2)
    assert torch.equal(lens2, lens) and torch.equal(c.k, k) and torch.equal(sums, s)
    assert np.array_equal(again[:, 0].cpu().numpy(), np.broadcast_to(np.arange(64, dtype=np.int32), (2, 2, 64))) and bool((again[:, 1] == -1).all())


def test_evict_of_a_long_request_on_another_stream_and_captured():
    rng = np.random.default_rng(65)
    lens, budget = [70001], 5000
    k = torch.from_numpy(rng.standard_normal((1, 70001 // 256 + 1, 1, 256, 64), dtype=np.float32)).bfloat16().cuda()
    table = torch.from_numpy(rng.permutation(k.shape[1]).astype(np.int32))[None].cuda()
    x = np.exp(rng.standard_normal((1, 1, 1, 70001))).astype(np.float32)
    sums, to = torch.from_numpy(x).cuda(), torch.zeros(1, 1, 1, 70001, device="cuda")
    kept, new_lens = torch.empty((1, 1, 1, budget), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    kv_lens = dev(lens)
    e = b.make_eviction(kv_lens=kv_lens, table=table, budgets=dev([budget]), max_kv_len=70001, max_budget=budget, recent=100, first=dev([1000]))
    work_k, work_v = k.clone(), k.clone()
    pages, m, tm = b.make_pages(work_k, work_v), b.make_mass(sums), b.make_mass(to)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        b.codecomp_evict(m, e, pages, kept, new_lens, kept_mass=tm)
    for n in (70001, 40000, 6000, 5999):
        kv_lens.fill_(n)
        work_k.copy_(k)
        work_v.copy_(k)
        graph.replay()
        want, want_lens = srv.evict(x, [n], [budget], recent=100, max_budget=budget, first=[1000])
        assert new_lens.tolist() == want_lens.tolist() and np.array_equal(kept.cpu().numpy(), want)
        at = torch.from_numpy(want[0, 0, 0][want[0, 0, 0] >= 0]).long().cuda()
        rows = lambda p, i: p[0, table[0, i // 256].long(), 0, i % 256]  # noqa: E731
        target = 1000 + torch.arange(len(at), device="cuda")
        assert torch.equal(rows(work_k, target), rows(k, at)) and torch.equal(work_v, work_k)
        assert torch.equal(to[0, 0, 0, target], sums[0, 0, 0, at])


@pytest.mark.parametrize("d, fp8, page, n_kv", [(128, False, 16, 2), (64, True, 8, 4), (64, False, 1, 2), (128, True, 64, 8)])
@pytest.mark.parametrize("elsewhere", [False, True])
def test_evict_of_very_many_problems(d, fp8, page, n_kv, elsewhere):
    """Numbers and rows in one kernel: a workgroup for each of 1024 problems and more; one request has more rows than a workgroup holds."""
    rng = np.random.default_rng([66, d, page])
    n = 1024 // (2 * n_kv) + 1
    lens = [int(x) for x in rng.integers(0, 60, n)]
    lens[n // 2], lens[3], lens[4] = 5200, 2, 0
    first = [int(x) for x in rng.integers(-2, 20, n)]
    budgets = [int(x) for x in rng.integers(0, 40, n)]
    budgets[n // 2] = 900
    for values in ("ties", "tail"):
        check_evict(rng, lens, budgets, recent=5, max_budget=900, first=first, n_kv=n_kv, d=d, page=page, fp8=fp8, layers=2, elsewhere=elsewhere, values=values)


def test_evict_largest_and_smallest_numbers():
    """Budgets, numbers of protected rows and lengths at the ends of their type."""
    low, high = -(2**31), 2**31 - 1
    for problems in (1, 520):
        rng = np.random.default_rng([67, problems])
        n = 4 * problems
        check_evict(rng, [90, 33, 90, 90] * problems, [high, low, low, high] * problems, recent=3, max_budget=30, first=[low, 5, high, 80] * problems, n_kv=1, d=64, layers=1 if problems > 1 else 3)


@pytest.mark.parametrize("fp8", [False, True])                          # rows of a cache line, and of half a line, whose other half is another workgroup's
def test_evict_strides_of_pool_and_sums(fp8):
    rng = np.random.default_rng(68)
    c, x = evict_setup(rng, [200, 150], None, layers=2, fp8=fp8)
    table, budgets, lens = c.dev_table(), dev([64, 30]), dev([200, 150])
    kept, new_lens = torch.empty((2, 2, 2, 64), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    e = b.make_eviction(kv_lens=lens, table=table, budgets=budgets, max_kv_len=200, max_budget=64, recent=4)
    k, v = (t.permute(1, 3, 0, 2, 4).contiguous().permute(2, 0, 3, 1, 4) for t in (c.k, c.v))
    wide = torch.zeros((2, 2, 2, 300), device="cuda")                    # [requests][heads][layers][rows] in memory
    sums = wide.permute(2, 0, 1, 3)[..., 7: 7 + x.shape[3]]
    sums.copy_(torch.from_numpy(x))
    to = torch.zeros((2, 2, 2, x.shape[3] + 9), device="cuda").permute(1, 0, 2, 3)[..., : x.shape[3]]
    dense, dense_kept, dense_lens = torch.from_numpy(x).cuda(), torch.empty_like(kept), torch.empty_like(new_lens)
    b.codecomp_evict(b.make_mass(sums), e, b.make_pages(k, v), kept, new_lens, kept_mass=b.make_mass(to))
    assert torch.equal(sums, dense)
    b.codecomp_evict(b.make_mass(dense), e, c.pages(), dense_kept, dense_lens)
    assert torch.equal(kept, dense_kept) and torch.equal(new_lens, dense_lens)
    assert torch.equal(k.view(torch.uint8), c.k.view(torch.uint8)) and torch.equal(v.view(torch.uint8), c.v.view(torch.uint8))
    for r, n in enumerate(dense_lens.tolist()):
        assert torch.equal(to[:, r, :, :n], dense[:, r, :, :n])
    b.codecomp_evict(b.make_mass(sums), e, c.pages(), kept, new_lens)    # in place, strided
    assert torch.equal(kept, dense_kept) and torch.equal(sums, dense)
    assert bool((wide[..., :7] == 0).all()) and bool((wide[..., 7 + x.shape[3]:] == 0).all())


@pytest.mark.parametrize("fp8, d", [(True, 64), (True, 128), (False, 64)])
def test_evict_of_many_heads_side_by_side(fp8, d):
    """Rows of all heads of a token one behind the other: lines of memory that several workgroups write to, each its own part, on whatever die."""
    rng = np.random.default_rng([72, d])
    c, x = evict_setup(rng, [300] * 9, None, layers=6, n_kv=8, fp8=fp8, d=d)
    table, budgets, lens, first = c.dev_table(), dev([100] * 9), dev([300] * 9), dev([3] * 9)
    make = lambda bound: b.make_eviction(kv_lens=lens, table=table, budgets=budgets, max_kv_len=bound, max_budget=100, recent=4, first=first)  # noqa: E731
    dense = torch.from_numpy(x).cuda()
    kept, new_lens = torch.empty((6, 9, 8, 100), dtype=torch.int32, device="cuda"), torch.empty(9, dtype=torch.int32, device="cuda")
    mixed = [t.permute(1, 3, 0, 2, 4).contiguous().permute(2, 0, 3, 1, 4) for t in (c.k, c.v)]
    b.codecomp_evict(b.make_mass(dense), make(300), b.make_pages(*mixed), kept, new_lens)
    again = torch.from_numpy(x).cuda()
    b.codecomp_evict(b.make_mass(again), make(300), c.pages(), torch.empty_like(kept), new_lens)
    for t, want in zip(mixed, (c.k, c.v)):
        assert torch.equal(t.view(torch.uint8), want.view(torch.uint8))
    assert torch.equal(dense, again) and np.array_equal(kept.cpu().numpy(), srv.evict(x, [300] * 9, [100] * 9, recent=4, max_budget=100, first=[3] * 9)[0])


@pytest.mark.parametrize("n, budget", [(2, 500), (2, 40), (300, 100)])
def test_evict_where_values_are_the_keys(n, budget):
    rng = np.random.default_rng([73, n])
    c, x = evict_setup(rng, [700] * n, None, layers=1)
    sums, other = torch.from_numpy(x).cuda(), torch.from_numpy(x).cuda()
    kept, lens = torch.empty((1, n, 2, budget), dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    e = b.make_eviction(kv_lens=dev([700] * n), table=c.dev_table(), budgets=dev([budget] * n), max_kv_len=700, max_budget=budget, recent=4)
    one = c.k.clone()
    b.codecomp_evict(b.make_mass(sums), e, b.make_pages(one, one), kept, lens)
    b.codecomp_evict(b.make_mass(other), e, c.pages(), kept, lens)
    assert torch.equal(one, c.k) and torch.equal(sums, other)


@pytest.mark.parametrize("fp8", [False, True])
def test_evict_offsets_beyond_32_bits(fp8):
    rng = np.random.default_rng([69, fp8])
    for n in (2, 300):                                                  # two kernels, one
        c, x = evict_setup(rng, [90] * n, None, fp8=fp8, layers=1)
        far_away(c)
        wide = torch.empty(2**32 + 2**31 + 1000 * n, device="cuda")
        sums = wide.as_strided((2, n, 2, x.shape[3]), (2**32, 200, 2**31, 1))
        sums[1] = torch.from_numpy(x[0]).cuda()
        sums[0] = 0
        kept, lens = torch.empty((2, n, 2, 40), dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
        e = b.make_eviction(kv_lens=dev([90] * n), table=c.dev_table(), budgets=dev([40] * n), max_kv_len=90, max_budget=40, recent=4)
        more = c.k.shape[1] - 6 * n - 3
        was = c.k[1, more:].clone()
        b.codecomp_evict(b.make_mass(sums), e, c.pages(), kept, lens)
        want, _ = srv.evict(np.stack([np.zeros_like(x[0]), x[0]]), [90] * n, [40] * n, recent=4, max_budget=40)
        assert np.array_equal(kept.cpu().numpy(), want)
        table = torch.from_numpy(c.table).cuda().long()
        for r in range(0, n, 7):
            for h in range(2):
                j = kept[1, r, h].long()
                i = torch.arange(40, device="cuda")
                rows = lambda pool, at: pool[table[r, at // 16], h, at % 16]  # noqa: E731
                assert torch.equal(rows(c.k[1], i), was[table[r, j // 16] - more, h, j % 16])
                assert torch.equal(sums[1, r, h, :40].cpu(), torch.from_numpy(x[0, r, h])[j.cpu()])
        del wide, sums, c
        torch.cuda.empty_cache()


def test_evict_twice_at_once():
    """Two calls at the same time, on caches of their own; and two graphs."""
    rng = np.random.default_rng(70)
    xs = []
    for _ in range(2):
        c, x = evict_setup(rng, [500, 300], None, layers=2)
        xs.append((c, x, torch.from_numpy(x).cuda(), c.k.clone(), c.v.clone(), torch.empty((2, 2, 2, 80), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda"),
                   b.make_eviction(kv_lens=dev([500, 300]), table=c.dev_table(), budgets=dev([80, 60]), max_kv_len=500, max_budget=80, recent=4)))
    call = lambda x: b.codecomp_evict(b.make_mass(x[2]), x[7], x[0].pages(), x[5], x[6])  # noqa: E731
    reset = lambda x: (x[2].copy_(torch.from_numpy(x[1])), x[0].k.copy_(x[3]), x[0].v.copy_(x[4]), x[5].fill_(-7))  # noqa: E731
    want, graphs, streams = [], [torch.cuda.CUDAGraph() for _ in xs], [torch.cuda.Stream() for _ in xs]
    for x in xs:
        call(x)
        want.append([t.clone() for t in (x[2], x[0].k, x[0].v, x[5], x[6])])
        assert np.array_equal(x[5].cpu().numpy(), srv.evict(x[1], [500, 300], [80, 60], recent=4, max_budget=80)[0])
    same = lambda i: all(torch.equal(t, w) for t, w in zip((xs[i][2], xs[i][0].k, xs[i][0].v, xs[i][5], xs[i][6]), want[i]))  # noqa: E731
    torch.cuda.synchronize()
    for g, x in zip(graphs, xs):
        with torch.cuda.graph(g):
            call(x)
    for turn in range(4):
        reset(xs[turn % 2])
        graphs[turn % 2].replay()
        assert same(turn % 2)
    for x in xs:
        reset(x)
    torch.cuda.synchronize()
    for s, x in zip(streams, xs):
        with torch.cuda.stream(s):
            call(x)
    torch.cuda.synchronize()
    assert same(0) and same(1)


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("n, count, wide", [(3, 1, 0), (12, 2, 0), (12, 2, 4000)])
def test_forked_requests_grow_and_are_evicted(fp8, n, count, wide):
    """A prompt's rows are shared; every request appends tokens, attends over shared and own rows, sums up weights on its own rows, and loses the lightest of them every few
    steps.  Attention and sums are checked against fp64 at every step, what is kept against the sums that there are."""
    rng = np.random.default_rng([71, n, count])
    L, Hq, Hkv, d, page, prefix, budget, recent = 2, 8, 2, 64, 16, 150, 10, 2 * count
    c = cu_.Cache(rng, [prefix] + [32] * n, n_kv=Hkv, d=d, page=page, fp8=fp8, layers=L, spare=2 * n, **scales(fp8))
    pages = c.pages()
    full = prefix // page
    free = [p for p in range(c.n_pages) if p not in set(c.table[0].tolist())]
    table = np.full((n, full + 3 + wide), -1, np.int32)                 # `wide`: bounds on lengths with which there may be much work
    for r in range(n):
        table[r, :full] = c.table[0, :full]
        table[r, full: full + 3] = free[3 * r: 3 * r + 3]
    table[0, full] = c.table[0, full]
    b.codecomp_pages_copy(pages, dev([[c.table[0, full], table[r, full]] for r in range(1, n)]))
    dt, lens, first, budgets = dev(table), dev([prefix] * n), dev([prefix] * n), dev([budget] * n)
    sums = torch.full((L, n, Hkv, table.shape[1] * page), float("nan"), device="cuda")          # never cleared
    mass = b.make_mass(sums)
    kept, new_lens = torch.empty((L, n, Hkv, budget), dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    groups = b.make_groups(cu_groups_host=[0, n], cu_groups=dev([0, n]), prefix_lens=dev([prefix]), max_prefix_len=table.shape[1] * page if wide else prefix, max_own_len=3 * page - prefix % page)
    cu = cum([count] * n)
    batch = b.make_batch(n_q_heads=Hq, cu_q_host=cu, cu_q=dev(cu), kv_lens=lens, table=dt, max_kv_len=table.shape[1] * page)
    eviction = b.make_eviction(kv_lens=lens, table=dt, budgets=budgets, max_kv_len=table.shape[1] * page, max_budget=budget, recent=recent, first=first)
    ws = torch.empty(b.codecomp_attend_shared_workspace_bytes(batch, groups, pages), dtype=torch.uint8, device="cuda")
    mws = torch.empty(max(256, b.codecomp_attend_mass_workspace_bytes(batch, pages, mass)), dtype=torch.uint8, device="cuda")
    rotary = b.make_rotary(d)
    at = prefix
    for step in range(9):
        lens += count
        host_lens = lens.tolist()
        for layer in range(L):
            q = cu_.bf16(rng.standard_normal((n * count, Hq, d))).cuda()
            k, v = (cu_.bf16(rng.standard_normal((n * count, Hkv, d)) * (5 if fp8 else 1)).cuda() for _ in range(2))
            b.codecomp_append(q, k, v, dev(np.tile(np.arange(at, at + count), n)), rotary, batch, pages, layer, q)
            out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
            b.codecomp_attend_shared(q, batch, groups, pages, layer, out, ws, lse=lse)
            kk, vv = c.values(layer)
            cu_.assert_attended(out, lse, srv.attend_shared(cu_.f64(q), kk, vv, table, host_lens, cu, [0, n], [prefix]), d, 16 if n * count * Hq // Hkv <= 64 else 8)
            before = sums[layer].cpu().numpy().copy()
            b.codecomp_attend_mass(q, lse, batch, pages, layer, mass, mws, first=first, decay=0.9)
            want, added, reach = srv.attend_mass(cu_.f64(q), lse.cpu().numpy(), kk, table, host_lens, cu, before, first=[prefix] * n, decay=0.9)
            got = sums[layer].cpu().numpy()
            there = np.zeros(got.shape, bool)
            for r in range(n):
                there[r, :, prefix: host_lens[r]] = True
            old = np.where(np.isnan(before), 0.0, before)
            assert np.all(np.abs(got - want)[there] <= mass_tolerance(want, added, reach, 0.9, old, count * Hq // Hkv)[there])
        at += count
        if step % 3 == 2:
            x = sums.cpu().numpy().copy()
            k0 = c.k.view(torch.uint8).cpu().numpy().copy()
            b.codecomp_evict(mass, eviction, pages, kept, new_lens)
            want, want_lens = srv.evict(x, host_lens, [budget] * n, recent=recent, max_budget=budget, first=[prefix] * n)
            assert np.array_equal(kept.cpu().numpy(), want) and np.array_equal(new_lens.cpu().numpy(), want_lens)
            k1 = c.k.view(torch.uint8).cpu().numpy()
            for r in range(n):
                for i, j in enumerate(want[1, r, 0]):
                    if j >= 0:
                        a, t = orc.place(table, r, int(j), page, c.n_pages), orc.place(table, r, prefix + i, page, c.n_pages)
                        assert np.array_equal(k1[1, t[0], 0, t[1]], k0[1, a[0], 0, a[1]])
            shared = c.table[0, :full]
            assert np.array_equal(k1[:, shared], k0[:, shared])
            lens.copy_(new_lens)


def test_readme_examples_run_one_after_another():
    """The examples of the README as they stand: compression, service from what was kept, and answers that share it."""
    import pathlib
    import re
    text = (pathlib.Path(__file__).resolve().parent.parent / "README.md").read_text()
    blocks = re.findall(r"(?:^    .*\n|^\n(?=    ))+", text[text.index("    import numpy as np, torch"):], re.M)
    assert len(blocks) == 3
    ns = {}
    for i, block in enumerate(blocks):
        exec(compile(re.sub(r"^    ", "", block, flags=re.M), f"README.md block {i}", "exec"), ns)
    torch.cuda.synchronize()
    n, kept, sums, rows = ns["n"], ns["kept"], ns["sums"], ns["kept_rows"]
    assert ns["lens"].tolist() == [kept + 128 + 400 - 300] * n                                    # 300 rows of its own each, 128 of them, 100 more
    assert bool((rows[..., -16:].cpu() == torch.arange(kept + 284, kept + 300)).all()) and bool((rows.diff(dim=-1) > 0).all()) and int(rows.min()) >= kept
    own = sums[..., kept: kept + 228]
    assert bool(torch.isfinite(own).all()) and bool((own > 0).all()) and bool(torch.isfinite(ns["out"].float()).all())
    # a token gives its rows of one head a weight of less than one in all: no more than a number of them that fades comes together
    assert float(own.sum(-1).max()) < 1 / (1 - 0.98)
