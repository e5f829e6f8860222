"""codecomp_attend_shared: how exact the weights of a request are, whatever stands beside it in its group and in the batch."""
import numpy as np
import pytest
import torch

from tests import cache_util as cu_
from tests.test_gpu_serve import Forked, shared_workspace

pytestmark = pytest.mark.gpu


def check_weights(f, causal, max_prefix=None, max_own=None):
    """Tokens of requests of up to 64 rows against the tolerance of weights of 16 bits, the others' of 8; all rows, shared and own."""
    from paper_2604_10235_amd import binding as b
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
    from paper_2604_10235_amd import binding as b
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
