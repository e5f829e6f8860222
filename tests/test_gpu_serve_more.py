"""Operators for shared and evicted caches, what their calls have beside them: how exact the weights of a request are whatever is in its group and batch, groups of few
rows and of many in one batch, sums behind evicted rows."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from oracle import serve_oracle as srv
from paper_2604_10235_amd import binding as b
from tests import cache_util as cu_
from tests.test_gpu_serve import Forked, cum, dev, evict_setup, mass_setup, mass_tolerance, shared_workspace

pytestmark = pytest.mark.gpu


def check_weights(f, causal, max_prefix=None, max_own=None):
    """Tokens of requests of up to 64 rows against the tolerance of weights of 16 bits, the others' of 8; all rows, shared and own."""
    batch, pages, groups = f.batch(causal=causal), f.cache.pages(), f.groups(max_prefix, max_own)
    ws, guard = shared_workspace(batch, groups, pages)
    out, lse = torch.full_like(f.q, 7.0), torch.full((f.T, f.n_q), 7.0, device="cuda")
    b.codecomp_attend_shared(f.q, batch, groups, pages, 0, out, ws, lse=lse)
    want = f.want(0, causal)
    short = np.array([n * f.n_q // f.cache.k.shape[2] <= 64 for n in f.news for _ in range(n)])
    for these, bits in ((short, 16), (~short, 8)):
        if these.any():
            at = torch.from_numpy(these).cuda()
            cu_.assert_attended(out[at], lse[at], tuple(x[these] for x in want), f.cache.d, bits)
    assert bool((guard == 0xA5).all())
    return short


# groups of more than 64 rows in all, of single tokens and of some, alone and beside prompts, which begin and end inside of blocks of 256 rows; several groups, some of one request,
# of none, or of prompts alone
@pytest.mark.parametrize("members, prefixes, news, n_q, n_kv", [
    ([30], [700], [1] * 30, 8, 2), ([70], [333], [1, 2, 0] * 23 + [4], 28, 4), ([11], [900], [16] * 11, 8, 2), ([9], [600], [1, 90, 1, 1, 17, 16, 0, 300, 2], 8, 2),
    ([5, 0, 40, 2], [500, 9, 640, 130], [100, 1, 70, 1, 1] + [1] * 40 + [80, 120], 14, 2), ([3], [1030], [64, 65, 64], 2, 2),
    ([600], [90], [1] * 300 + [100, 0] + [1] * 298, 4, 2)])
@pytest.mark.parametrize("fp8, d, page", [(False, 128, 16), (True, 128, 8), (False, 64, 4), (True, 64, 64)])
@pytest.mark.parametrize("causal, loose", [(True, 0), (True, 70000), (False, 70000)])
def test_weights_of_short_requests_in_large_groups(members, prefixes, news, n_q, n_kv, fp8, d, page, causal, loose):
    rng = np.random.default_rng([81, sum(news), d, page])
    f = Forked(rng, members, prefixes, news, [n + int(rng.integers(0, 90)) for n in news], n_q=n_q, n_kv=n_kv, d=d, page=page, fp8=fp8, loose=loose)
    assert check_weights(f, causal).any()


# no shared rows, by a bound that lets there be many: all weights are those of own rows
@pytest.mark.parametrize("members, news, own", [([30], [1] * 30, 400), ([12], [1, 16, 2, 300, 1, 9, 0, 1, 40, 16, 17, 3], 700), ([2, 9], [70, 1] + [8] * 9, 1500)])
@pytest.mark.parametrize("fp8, d, page", [(False, 128, 16), (True, 64, 8), (False, 64, 128)])
@pytest.mark.parametrize("causal, loose, max_own", [(True, 70000, None), (True, 70000, 20000), (False, 9000, None)])
def test_weights_of_own_rows_in_large_groups(members, news, own, fp8, d, page, causal, loose, max_own):
    rng = np.random.default_rng([82, sum(news), d, page])
    f = Forked(rng, members, [0] * len(members), news, [n + int(rng.integers(0, own)) for n in news], n_q=8, n_kv=2, d=d, page=page, fp8=fp8, loose=loose)
    assert check_weights(f, causal, max_own=max_own and min(max_own, loose)).any()


# groups of few rows and of many in all orders, with different numbers of chunks (by loose bounds), some without requests or tokens; more tokens than a workgroup has threads, and more groups
@pytest.mark.parametrize("members, prefixes, news, own, n_q, n_kv", [
    ([30, 1], [700, 700], [1] * 31, 90, 8, 2), ([1, 30], [2000, 300], [1] * 31, 9, 8, 2), ([1, 0, 2, 40, 1, 1], [333, 4, 90, 700, 64, 1], [1, 2, 0] + [2] * 40 + [0, 3], 40, 14, 2),
    ([2, 1, 1], [600, 900, 130], [300, 260, 1, 290], 600, 4, 2), ([1] * 300 + [100], [70] * 301, [int(x) for x in np.arange(300) % 3] + [1] * 100, 20, 8, 2),
    ([100] + [2] * 300, [200] + [50] * 300, [2] * 100 + [1] * 600, 1100, 8, 2)])
@pytest.mark.parametrize("fp8, d, page", [(False, 128, 16), (True, 64, 8)])
@pytest.mark.parametrize("causal, loose", [(True, 0), (True, 3000), (False, 30000)])
def test_groups_of_both_kinds_side_by_side(members, prefixes, news, own, n_q, n_kv, fp8, d, page, causal, loose):
    rng = np.random.default_rng([83, sum(news), d, page])
    f = Forked(rng, members, prefixes, news, [n + int(rng.integers(0, own)) for n in news], n_q=n_q, n_kv=n_kv, d=d, page=page, fp8=fp8, loose=loose)
    check_weights(f, causal)


def test_groups_of_both_kinds_of_very_many_tokens():
    """All values of a group are one number, a power of two of its own: so is every output, but for the weights' rounding (half a step of 8 bits) and the output's."""
    members, news, G, d, page, prefix, own = [1, 3, 1, 0, 2], [150000, 1, 1, 1, 90001, 2, 3], 2, 64, 16, 48, 9
    of, n = [g for g, m in enumerate(members) for _ in range(m)], len(news)
    gen = torch.Generator(device="cuda").manual_seed(3)
    k = torch.randn((1, 4 * n, 1, page, d), generator=gen, device="cuda").bfloat16()
    v = torch.empty_like(k)
    for r in range(n):
        v[:, 4 * r: 4 * r + 4] = 2.0 ** (2 * of[r] - 4)
    table, cu, cg = torch.arange(4 * n, device="cuda").int().view(n, 4), np.concatenate([[0], np.cumsum(news)]).astype(np.int32), np.concatenate([[0], np.cumsum(members)]).astype(np.int32)
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
    wide = torch.zeros((n, 64), dtype=torch.int32, device="cuda")
    wide[:, :4] = table
    pages = b.make_pages(k, v)
    batch = b.make_batch(n_q_heads=G, cu_q_host=cu, cu_q=i32(cu), kv_lens=i32([prefix + own] * n), table=wide, max_kv_len=1024, causal=False)
    groups = b.make_groups(cu_groups_host=cg, cu_groups=i32(cg), prefix_lens=i32([prefix] * len(members)), max_prefix_len=1000, max_own_len=20)
    ws, guard = shared_workspace(batch, groups, pages)
    q = torch.randn((int(cu[-1]), G, d), generator=gen, device="cuda").bfloat16()
    out = torch.empty_like(q)
    b.codecomp_attend_shared(q, batch, groups, pages, 0, out, ws)
    want = torch.repeat_interleave(torch.tensor([2.0 ** (2 * g - 4) for g in of], device="cuda"), i32(news))[:, None, None]
    assert bool(((out.float() - want).abs() <= (2.0 ** -8 + 2.0 ** -8) * want * (1 + 2.0 ** -7)).all()) and bool((guard == 0xA5).all())


# ---------------------------------------------------------------- sums of weights behind evicted rows

@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("news", [[1, 3], [40, 30]])
@pytest.mark.parametrize("fp8", [False, True])
def test_sums_of_rows_appended_where_evicted_ones_stood(causal, news, fp8):
    """Causal: whatever stands in the sums of the new rows, they start from nothing.  Else their sums are cleared, or they go on from what stood there."""
    rng = np.random.default_rng([84, news[0]])
    lens, n_q, n_kv, d, page, budget = [300, 170], 8, 2, 64, 16, 60
    c, x = evict_setup(rng, lens, None, n_kv=n_kv, d=d, page=page, fp8=fp8, layers=1)
    table, sums, pages = c.dev_table(), torch.from_numpy(x).cuda(), c.pages()
    kept, new_lens = torch.empty((1, 2, n_kv, budget), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    m = b.make_mass(sums)
    b.codecomp_evict(m, b.make_eviction(kv_lens=dev(lens), table=table, budgets=dev([budget] * 2), max_kv_len=300, max_budget=budget, recent=8), pages, kept, new_lens)
    assert new_lens.tolist() == [budget] * 2
    cu, now = cum(news), [budget + n for n in news]
    batch = b.make_batch(n_q_heads=n_q, cu_q_host=cu, cu_q=dev(cu), kv_lens=dev(now), table=table, max_kv_len=300, causal=causal)
    q = cu_.bf16(rng.standard_normal((int(cu[-1]), n_q, d))).cuda()
    k, v = (cu_.bf16(rng.standard_normal((int(cu[-1]), n_kv, d)) * (5 if fp8 else 1)).cuda() for _ in range(2))
    b.codecomp_append(q, k, v, dev(np.arange(int(cu[-1]))), b.make_rotary(d), batch, pages, 0, q)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    b.codecomp_attend(q, batch, pages, 0, out, cu_.workspace(batch, pages), lse=lse)
    ws = torch.empty(max(256, b.codecomp_attend_mass_workspace_bytes(batch, pages, m)), dtype=torch.uint8, device="cuda")
    kk, _ = c.values(0)
    for new_sums in ([float("nan")] if causal else [0.0, None]):
        if new_sums is not None:
            sums[..., budget:] = new_sums
        else:
            sums.copy_(torch.from_numpy(x))
        before = sums[0].cpu().numpy().copy()
        b.codecomp_attend_mass(q, lse, batch, pages, 0, m, ws, decay=0.75)
        got = sums[0].cpu().numpy()
        want, added, reach = srv.attend_mass(cu_.f64(q), lse.cpu().numpy(), kk, c.table, now, cu, before, decay=0.75, causal=causal)
        for r in range(2):
            there = np.s_[r, :, :now[r]]
            old = np.where(np.isnan(before), 0.0, before)
            assert np.all(np.abs(got - want)[there] <= mass_tolerance(want, added, reach, 0.75, old, news[r] * n_q // n_kv)[there])
            if new_sums == 0.0 or causal:                          # nothing but the weights of this call
                fresh = np.s_[r, :, budget:now[r]]
                assert np.all(np.abs(got - added)[fresh] <= mass_tolerance(added, added, reach, 0.0, 0.0, news[r] * n_q // n_kv)[fresh])


@pytest.mark.parametrize("news", [[1, 3], [40, 60]])
@pytest.mark.parametrize("where", ["query", "key"])
def test_sums_of_infinite_logits(news, where):
    """Plus infinity makes a sum infinite, minus infinity adds nothing; the sign is that of the other factor."""
    rng = np.random.default_rng([85, news[0]])
    c, batch, cu, q, sums = mass_setup(rng, [333, 260], news, 8, n_kv=2, d=64, page=16)
    pages, m, lse = c.pages(), b.make_mass(sums), torch.full((sum(news), 8), 2.0, device="cuda")
    ws = torch.empty(max(256, b.codecomp_attend_mass_workspace_bytes(batch, pages, m)), dtype=torch.uint8, device="cuda")

    def call():
        sums.fill_(0.5)
        b.codecomp_attend_mass(q, lse, batch, pages, 0, m, ws)
        return sums.clone()

    clean = call()
    t, h = news[0], 5                                                  # the second request's first token, of the second KV head
    if where == "query":
        q[t, h, 3] = float("inf")
        x = call()
        sees = 260 - news[1] + 1
        p = [orc.place(c.table, 1, j, 16, c.n_pages) for j in range(sees)]
        factor = torch.stack([c.k[0, a, 1, i, 3] for a, i in p]).float()
        assert bool((torch.isposinf(x[0, 1, 1, :sees]) == (factor > 0)).all()) and bool(torch.isfinite(x[0, 1, 1, :sees][factor < 0]).all())
        # what the token adds nothing to is what the other tokens and heads make of it
        q[t, h, 3] = 0.0
        lse[t, h] = -float("inf")
        without = call()
        assert torch.equal(x[0, 1, 1, :sees][factor < 0], without[0, 1, 1, :sees][factor < 0])
        x[0, 1, 1, :sees] = clean[0, 1, 1, :sees]
        assert torch.equal(x, clean)
    else:
        a, i = orc.place(c.table, 1, 17, 16, c.n_pages)
        c.k[0, a, 1, i, 3] = -float("inf")
        x = call()
        factor = q[news[0]:, 4:, 3].float()
        assert bool((factor != 0).all()) and bool(torch.isposinf(x[0, 1, 1, 17])) == bool((factor < 0).any())
        x[0, 1, 1, 17] = clean[0, 1, 1, 17]
        assert torch.equal(x, clean)
