"""codecomp_attend against the fp64 oracle: lengths, masks, pages, types, garbage where nothing is read, graphs, streams, and a run of the
whole path from compression to steps of one token."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from paper_2604_10235_amd import binding as b
from tests import cache_util as cu_

pytestmark = pytest.mark.gpu


def check(rng, cache, news, n_q, *, causal=True, lens=None, weight_bits=8, sharp=1.0, max_kv=None, softmax_scale=0.0, layer=0):
    batch, cu = cu_.make_batch(cache, news, n_q, lens=lens, max_kv=max_kv, causal=causal, softmax_scale=softmax_scale)
    T = int(cu[-1])
    q = cu_.bf16(rng.standard_normal((T, n_q, cache.d)) * sharp).cuda()
    pages = cache.pages()
    out = torch.full((T + 3, n_q, cache.d), 7.0, dtype=torch.bfloat16, device="cuda")          # rows behind the last token stay
    lse = torch.full((T + 3, n_q), 7.0, dtype=torch.float32, device="cuda")
    ws = cu_.workspace(batch, pages)
    b.codecomp_attend(q, batch, pages, layer, out[:T], ws, lse=lse[:T])
    k, v = cache.values(layer)
    want = orc.attend(cu_.f64(q), k, v, cache.table, cache.lens if lens is None else lens, cu, max_kv_len=batch.max_kv_len, causal=causal,
                      scale=softmax_scale or None)
    cu_.assert_attended(out[:T], lse[:T], want, cache.d, weight_bits)
    assert bool((out[T:] == 7.0).all()) and bool((lse[T:] == 7.0).all())
    again = torch.empty_like(out)
    b.codecomp_attend(q, batch, pages, layer, again[:T], ws)                                     # without lse: the same bits
    assert torch.equal(again[:T], out[:T])
    return q, batch, out[:T], lse[:T], want


# requests of up to 64 rows (new tokens x query heads per KV head): 16-bit weights
@pytest.mark.parametrize("lens, news, n_q, n_kv, d, page, fp8", [
    ([1], [1], 1, 1, 64, 16, False), ([0, 1, 2, 31, 32, 33, 63, 64, 65, 700], [1] * 10, 4, 2, 128, 16, False),
    ([257, 129, 1030], [1, 1, 1], 28, 4, 128, 64, False), ([257, 129, 1030], [1, 1, 1], 14, 2, 128, 32, True),
    ([90, 500, 17, 300], [2, 8, 1, 0], 16, 2, 64, 1, False), ([90, 500, 17, 300], [2, 4, 1, 3], 32, 8, 128, 128, True),
    ([40, 16, 5], [64, 16, 5], 1, 1, 128, 8, False), ([2000, 5000], [1, 9], 7, 1, 128, 256, False), ([3001], [16], 4, 1, 64, 16, True)])
@pytest.mark.parametrize("causal", [True, False])
def test_few_rows(lens, news, n_q, n_kv, d, page, fp8, causal):
    rng = np.random.default_rng([sum(lens), n_q, page])
    c = cu_.Cache(rng, lens, n_kv=n_kv, d=d, page=page, fp8=fp8, k_scale=0.03 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
    check(rng, c, news, n_q, causal=causal, weight_bits=16)


@pytest.mark.parametrize("lens, news, n_q, n_kv, d, page, fp8", [
    ([65], [65], 1, 1, 64, 16, False), ([300], [300], 7, 1, 128, 16, False), ([1000, 130], [100, 130], 8, 2, 128, 64, True),
    ([700, 64, 20, 1500], [70, 64, 20, 1], 14, 2, 64, 1, False), ([50, 10, 333], [90, 90, 333], 4, 4, 128, 32, False),
    ([2049], [33], 28, 4, 128, 128, False), ([500, 90], [200, 90], 7, 1, 128, 8, False), ([500, 90], [200, 90], 4, 2, 128, 2, True), ([900], [257], 2, 1, 128, 256, True), ([0, 129, 128, 127], [80, 80, 80, 80], 6, 3, 64, 8, True)])
@pytest.mark.parametrize("causal", [True, False])
def test_many_rows(lens, news, n_q, n_kv, d, page, fp8, causal):
    rng = np.random.default_rng([sum(lens), n_q, page, 1])
    c = cu_.Cache(rng, lens, n_kv=n_kv, d=d, page=page, fp8=fp8, k_scale=0.03 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
    check(rng, c, news, n_q, causal=causal)


# How the work is shared out: blocks of rows cut by several workgroups, shared by none, more blocks than threads that count them, more
# requests than such threads, requests without tokens among them, short requests beside long ones and along with them.
@pytest.mark.parametrize("lens, news, n_q, n_kv, d, page", [
    ([9000], [70], 1, 1, 64, 64), ([5000, 100], [300, 90], 7, 1, 128, 16), ([700] * 3, [700, 650, 600], 2, 2, 64, 4), ([500] * 4, [500, 1, 70, 300], 4, 1, 128, 16),
    ([2100, 2100], [2100, 1], 2, 1, 64, 32), ([300, 900] * 12, [1, 80] * 12, 4, 2, 64, 16), ([3000] + [2600] * 40, [90] + [1] * 40, 8, 8, 64, 128),
    ([40] * 700, [0, 1, 0, 33, 2, 0, 0] * 100, 4, 2, 64, 8), ([200] * 520, [9] * 519 + [200], 2, 1, 64, 16)])
def test_shares(lens, news, n_q, n_kv, d, page):
    rng = np.random.default_rng([sum(lens), n_q, page, 2])
    c = cu_.Cache(rng, lens, n_kv=n_kv, d=d, page=page)
    check(rng, c, news, n_q)


@pytest.mark.parametrize("n", [600, 3000])
@pytest.mark.parametrize("fp8", [False, True])
def test_many_requests_and_few_tokens(n, fp8):
    """Runs of requests without tokens, between ones with few and with many, over two heads."""
    rng = np.random.default_rng([29, n])
    news = [90 if r % 290 == 7 else 1 if r % 3 == 0 and r % 500 < 200 else 0 for r in range(n)]
    lens = [int(x) for x in rng.integers(0, 40, n)]
    lens[7], lens[297] = 400, 131
    c = cu_.Cache(rng, lens, n_kv=2, d=64, page=16, fp8=fp8, width_more=40, k_scale=0.03 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
    check(rng, c, news, 4)                                        # short lengths: blocks that are not shared
    check(rng, c, news, 4, max_kv=1000)
    check(rng, c, [1 if x == 1 or r == 7 else 0 for r, x in enumerate(news)], 4, weight_bits=16)


# Requests of few rows whose bound on lengths makes the batch a large one: keys of all of them cut into equal parts, which end inside requests, hold
# several, or are less than 128 keys; requests without keys or tokens, more of them than a workgroup has threads, pages that are not held.
@pytest.mark.parametrize("lens, news, n_q, n_kv, d, fp8", [
    ([1300, 140, 16], [1, 1, 1], 8, 2, 128, False), ([1300, 140, 16], [4, 1, 3], 8, 1, 128, False), ([40000, 3, 0, 517, 30000], [1, 1, 1, 0, 1], 4, 2, 64, False),
    ([40000, 3, 0, 517, 30000], [2, 2, 2, 0, 4], 14, 2, 128, True), ([0, 0, 0], [1, 2, 1], 4, 2, 64, True), ([65000, 900], [1, 1], 7, 1, 128, False),
    ([5, 300, 0, 129] * 160, [1, 0, 1, 1] * 160, 2, 1, 64, True)])
@pytest.mark.parametrize("causal", [True, False])
def test_equal_parts(lens, news, n_q, n_kv, d, fp8, causal):
    rng = np.random.default_rng([26, len(lens), d])
    c = cu_.Cache(rng, lens, n_kv=n_kv, d=d, page=256, fp8=fp8, width_more=6000, k_scale=0.03 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
    c.table[0, 2:4] = [-1, c.n_pages]
    check(rng, c, news, n_q, causal=causal, weight_bits=16, max_kv=1 << 20)


# 33 .. 64 rows, alone and beside single tokens, where the bound on lengths makes the batch a small one and a large one.
@pytest.mark.parametrize("news", [[9, 0, 16], [9, 1, 16], [1, 2, 5], [13, 1, 3]])
@pytest.mark.parametrize("fp8", [False, True])
def test_middle_sized_chunks_of_long_caches(news, fp8):
    rng = np.random.default_rng([24, news[0]])
    c = cu_.Cache(rng, [1300, 140, 16], n_kv=2, d=128, page=256, fp8=fp8, width_more=300, k_scale=0.03 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
    for max_kv in (1300, 70000):
        check(rng, c, news, 8, max_kv=max_kv)
        check(rng, c, news, 8, max_kv=max_kv, causal=False)


# Up to 64 rows have weights of 16 bits whatever kernel they take.
@pytest.mark.parametrize("news, n_q, d", [([9, 1, 16], 8, 128), ([13, 1, 3], 8, 64), ([64, 2, 16], 2, 64), ([9, 2, 9], 14, 128)])
@pytest.mark.parametrize("fp8, max_kv", [(False, 100000), (True, 700000)])
@pytest.mark.parametrize("page", [2048, 8])
def test_middle_sized_chunks_have_fine_weights(news, n_q, d, fp8, max_kv, page):
    rng = np.random.default_rng([27, news[0], n_q, page])
    c = cu_.Cache(rng, [1300, 140, 16], n_kv=2, d=d, page=page, fp8=fp8, width_more=max_kv // page, k_scale=0.03 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
    check(rng, c, news, n_q, max_kv=max_kv, weight_bits=16)
    check(rng, c, news, n_q, max_kv=max_kv, weight_bits=16, causal=False)


@pytest.mark.parametrize("news", [[9, 16], [1, 16]])
def test_middle_sized_chunks_of_very_long_8_bit_caches(news):
    rng = np.random.default_rng([25, news[0]])
    c = cu_.Cache(rng, [1300, 140], n_kv=2, d=64, page=4096, fp8=True, width_more=200, k_scale=0.03, v_scale=0.02)
    check(rng, c, news, 8, max_kv=700000)


def test_many_tokens_of_one_prompt():
    """More blocks of rows than a workgroup has threads: 66000 tokens of two heads, which see few keys each."""
    rng = np.random.default_rng(21)
    c = cu_.Cache(rng, [130], n_kv=2, d=64, page=16)
    check(rng, c, [66000], 4, causal=False)
    check(rng, c, [66000], 4)                  # all but the last 130 see nothing


@pytest.mark.parametrize("news", [[1, 2, 1], [100, 40, 1]])
def test_logits_of_hundreds(news):
    """Maxima that keep growing along the keys, and rows that see one key only."""
    rng = np.random.default_rng(12)
    c = cu_.Cache(rng, [900, 300, 1], n_kv=2, d=128, page=16)
    for r in range(2):          # keys that grow with their place
        for j in range(c.lens[r]):
            p, at = orc.place(c.table, r, j, 16, c.n_pages)
            c.k[0, p, :, at] *= 0.02 * j
    check(rng, c, news, 8, sharp=4.0)
    check(rng, c, news, 8, sharp=-4.0, softmax_scale=0.5)


@pytest.mark.parametrize("news", [[1, 1, 1, 1], [3, 8, 1, 2], [200, 70, 65, 1]])
@pytest.mark.parametrize("fp8", [False, True])
def test_pages_that_are_not_held(news, fp8):
    rng = np.random.default_rng(13)
    c = cu_.Cache(rng, [330, 100, 70, 40], n_kv=2, d=64, page=16, fp8=fp8, k_scale=0.03, v_scale=0.02)
    c.table[0, 3], c.table[0, 20], c.table[1, 0] = -1, c.n_pages, -2**31
    c.table[2, :], c.table[3, :] = -1, 2**31 - 1          # nothing held: zeros, and a log-sum-exp of minus infinity
    _, _, out, lse, _ = check(rng, c, news, 4)
    T = sum(news[:2])
    assert bool((out[T:] == 0).all()) and bool(torch.isneginf(lse[T:]).all())


@pytest.mark.parametrize("news, n_q", [([1, 1], 8), ([6, 3], 8), ([150, 90], 2), ([40, 300], 8)])
@pytest.mark.parametrize("d, fp8", [(128, False), (64, True), (64, False), (128, True)])
def test_garbage_in_places_that_are_not_seen(news, n_q, d, fp8):
    """NaN and infinities behind the end, in pages of nobody, and in new tokens that earlier ones do not see."""
    rng = np.random.default_rng([14, d])
    lens = [333, 310]
    c = cu_.Cache(rng, lens, n_kv=2, d=d, page=16, fp8=fp8, k_scale=0.03 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
    batch, cu = cu_.make_batch(c, news, n_q)
    q = cu_.bf16(rng.standard_normal((sum(news), n_q, d))).cuda()
    ws = cu_.workspace(batch, c.pages())
    clean, lse = torch.empty_like(q), torch.empty(sum(news), n_q, device="cuda")
    b.codecomp_attend(q, batch, c.pages(), 0, clean, ws, lse=lse)
    nobody = np.setdiff1d(np.arange(c.n_pages), c.table)
    spoil = [float("nan")] if fp8 else [float("nan"), float("inf"), -float("inf"), 3e38]
    set_ = lambda t, p, at, x: t.view(torch.uint8)[0, p, :, at].fill_(0x7F) if fp8 else t[0, p, :, at].fill_(x)  # noqa: E731
    for x in spoil:
        for p in nobody:
            for at in range(16):
                set_(c.k, int(p), at, x), set_(c.v, int(p), at, x)
        for r, n in enumerate(lens):
            for at in range(n % 16, 16):
                set_(c.k, int(c.table[r, n // 16]), at, x), set_(c.v, int(c.table[r, n // 16]), at, x)
        got, got_lse = torch.empty_like(q), torch.empty_like(lse)
        b.codecomp_attend(q, batch, c.pages(), 0, got, ws, lse=got_lse)
        assert torch.equal(got, clean) and torch.equal(got_lse, lse), x
        # the last new token of each request: only it may see it
        keep = c.k.clone(), c.v.clone()
        for r, n in enumerate(lens):
            p, at = orc.place(c.table, r, n - 1, 16, c.n_pages)
            set_(c.k, p, at, x), set_(c.v, p, at, x)
        b.codecomp_attend(q, batch, c.pages(), 0, got, ws, lse=got_lse)
        c.k.copy_(keep[0]), c.v.copy_(keep[1])
        last = np.zeros(sum(news), bool)
        last[cu[1:] - 1] = True
        seen, unseen = torch.from_numpy(last).cuda(), torch.from_numpy(~last).cuda()
        # (the tile's sums are the same numbers in the same order: the same bits)
        assert torch.equal(got[unseen], clean[unseen]) and torch.equal(got_lse[unseen], lse[unseen]), x
        if x != x:
            assert bool(torch.isnan(got[seen]).all())
    # values alone, in the middle of a chunk: tokens from there on have it, no earlier one
    if news[0] > 2:
        keep, at_token = c.v.clone(), news[0] // 2
        p, at = orc.place(c.table, 0, lens[0] - news[0] + at_token, 16, c.n_pages)
        set_(c.v, p, at, spoil[-1] if fp8 else float("inf"))
        b.codecomp_attend(q, batch, c.pages(), 0, got, ws)
        c.v.copy_(keep)
        assert torch.equal(got[:at_token], clean[:at_token]) and not bool(torch.isfinite(got[at_token: news[0]]).any())


@pytest.mark.parametrize("news, n_q", [([1, 1], 8), ([6, 3], 8), ([9, 14], 8), ([3, 14], 8)])
@pytest.mark.parametrize("d, fp8", [(128, False), (64, True), (64, False)])
def test_garbage_where_lengths_may_be_long(monkeypatch, news, n_q, d, fp8):
    """The same with a bound on lengths that selects equal parts, and fine weights in the many-row kernel."""
    cache, batch = cu_.Cache, cu_.make_batch
    monkeypatch.setattr(cu_, "Cache", lambda rng, lens, **kw: cache(rng, lens, width_more=1 << 16, **kw))
    monkeypatch.setattr(cu_, "make_batch", lambda c, news, n_q: batch(c, news, n_q, max_kv=1 << 20))
    test_garbage_in_places_that_are_not_seen(news, n_q, d, fp8)


@pytest.mark.parametrize("news", [[1, 2], [100, 40]])
def test_scales_at_the_ends_of_fp32(news):
    """Logits that all vanish: every key weighs the same, hidden ones still nothing."""
    rng = np.random.default_rng(22)
    c = cu_.Cache(rng, [200, 77], n_kv=2, d=64, page=16, fp8=True, k_scale=1e-30)
    check(rng, c, news, 4, softmax_scale=1e-30)


@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("news", [[1, 2], [100, 40]])
def test_logits_near_the_ends_of_fp32(news, sign):
    """Logits of +-2^117: all keys weigh the same, and no row counts as one that sees nothing.  The mean of n values is off by half a step and by the
    rounding of n fp32 sums and of a quotient."""
    rng = np.random.default_rng(23)
    c = cu_.Cache(rng, [2000, 777], n_kv=2, d=64, page=16)
    c.k[:] = 0.0
    c.k[..., 5] = sign * 2.0**60
    batch, cu = cu_.make_batch(c, news, 4, causal=False)
    q = torch.zeros(int(cu[-1]), 4, 64, dtype=torch.bfloat16, device="cuda")
    q[..., 5] = 2.0**60
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    b.codecomp_attend(q, batch, c.pages(), 0, out, cu_.workspace(batch, c.pages()), lse=lse)
    assert bool((lse / (sign * 2.0**117) - 1).abs().max() < 2.0**-20)          # 2^120 / sqrt(64); ln 2000 is nothing beside it
    v = c.values()[1]
    for r, n in enumerate(c.lens):
        rows = np.stack([v[c.table[r, j // 16], :, j % 16] for j in range(n)])                       # [keys, KV heads, d]
        mean, spread = rows.mean(0).repeat(2, 0), np.abs(rows).mean(0).repeat(2, 0)
        got = cu_.f64(out[cu[r]: cu[r + 1]])
        assert np.all(np.abs(got - mean) <= 2.0**-8 * np.abs(mean) + 1.01 * (n + 4) * 2.0**-24 * spread)


def test_a_batch_without_tokens():
    c = cu_.Cache(np.random.default_rng(23), [40, 3], n_kv=2, d=64, page=16)
    batch, _ = cu_.make_batch(c, [0, 0], 4)
    q, k = (torch.empty((0, h, 64), dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    pos = torch.empty(0, dtype=torch.int32, device="cuda")
    before = c.k.clone()
    b.codecomp_append(q, k, k, pos, b.make_rotary(64), batch, c.pages(), 0, q)
    b.codecomp_attend(q, batch, c.pages(), 0, q, None, lse=torch.empty((0, 4), device="cuda"))
    b.codecomp_rotate(q, pos, b.make_rotary(64), q)
    b.codecomp_pages_copy(c.pages(), torch.empty((0, 2), dtype=torch.int32, device="cuda"))
    assert torch.equal(c.k, before)


def test_strides_scale_and_layers():
    rng = np.random.default_rng(15)
    for news in ([1, 3], [120, 5]):
        c = cu_.Cache(rng, [200, 77], n_kv=2, d=128, page=32, layers=3)
        c.k, c.v = (t.permute(1, 0, 3, 2, 4).contiguous().permute(1, 0, 3, 2, 4) for t in (c.k, c.v))         # token-major pages, layers inside
        assert not c.k.is_contiguous()
        T = sum(news)
        batch, cu = cu_.make_batch(c, news, 6, q_stride_tok=10 * 128, out_stride_tok=136, out_stride_head=136 * T, softmax_scale=0.2)
        q = cu_.bf16(rng.standard_normal((T, 10, 128))).cuda()[:, :6]
        out = torch.full((6, T, 136), 5.0, dtype=torch.bfloat16, device="cuda")
        b.codecomp_attend(q, batch, c.pages(), 2, out.transpose(0, 1)[..., :128], cu_.workspace(batch, c.pages()))
        k, v = c.values(2)
        want = orc.attend(cu_.f64(q), k, v, c.table, c.lens, cu, max_kv_len=200, scale=0.2)
        cu_.assert_attended(out.transpose(0, 1)[..., :128], None, want, 128)
        assert bool((out[..., 128:] == 5.0).all())


def test_pool_beyond_32_bit_offsets():
    """Pages whose elements lie beyond 2^31, in both types."""
    rng = np.random.default_rng(16)
    for fp8, pages in ((False, 70000), (True, 140000)):
        c = cu_.Cache(rng, [300, 90], n_kv=2, d=128, page=128, fp8=fp8, k_scale=0.03 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
        small, small_v, table = c.k, c.v, c.table.copy()
        far = lambda t: torch.empty((1, pages, *t.shape[2:]), dtype=t.dtype, device="cuda")  # noqa: E731
        c.k, c.v = far(small), far(small_v)
        at = pages - 1 - 7 * np.arange(c.n_pages)
        bits = lambda t: t.view(torch.uint8) if fp8 else t  # noqa: E731
        bits(c.k)[:, torch.from_numpy(at).cuda()], bits(c.v)[:, torch.from_numpy(at).cuda()] = bits(small), bits(small_v)
        held = table >= 0
        c.table[held] = at[table[held]]
        k, v = cu_.f64(small[0]) * c.k_scale, cu_.f64(small_v[0]) * c.v_scale
        for news in ([1, 1], [80, 70]):
            batch, cu = cu_.make_batch(c, news, 4)
            q = cu_.bf16(rng.standard_normal((sum(news), 4, 128))).cuda()
            pool = b.make_pages(c.k, c.v, k_scale=c.k_scale, v_scale=c.v_scale)
            new = cu_.bf16(rng.standard_normal((sum(news), 2, 128))).cuda()
            out = torch.empty_like(q)
            b.codecomp_attend(q, batch, pool, 0, out, cu_.workspace(batch, pool))
            cu_.assert_attended(out, None, orc.attend(cu_.f64(q), k, v, table, c.lens, cu, max_kv_len=300), 128)
            if not fp8:
                keep = c.k.clone(), c.v.clone()
                b.codecomp_append(None, new, new, None, None, batch, pool, 0, None)
                p, row = orc.place(c.table, 1, 89, 128, pages)
                assert torch.equal(c.k[0, p, :, row], new[-1])
                b.codecomp_pages_copy(pool, torch.tensor([[p, pages // 2]], dtype=torch.int32, device="cuda"))
                assert torch.equal(c.k[0, pages // 2], c.k[0, p])
                c.k.copy_(keep[0]), c.v.copy_(keep[1])
                del keep
        del c, small, small_v


def test_parts_are_joined_by_their_log_sum_exp():
    """A cache attended to in two halves, joined with the halves' lse, is the whole; and the call is the same on a stream of its own."""
    rng = np.random.default_rng(17)
    c = cu_.Cache(rng, [512], n_kv=2, d=64, page=32)
    q = cu_.bf16(rng.standard_normal((3, 4, 64))).cuda()
    parts = []
    for rows in (slice(0, 16), slice(0, 5), slice(5, 16)):
        half = cu_.Cache(rng, [32 * (rows.stop - rows.start)], n_kv=2, d=64, page=32)
        half.k, half.v, half.table, half.n_pages = c.k, c.v, np.ascontiguousarray(c.table[:, rows]), c.n_pages
        batch, _ = cu_.make_batch(half, [3], 4, causal=False)
        out, lse = torch.empty_like(q), torch.empty(3, 4, device="cuda")
        ws = cu_.workspace(batch, half.pages())
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            b.codecomp_attend(q, batch, half.pages(), 0, out, ws, lse=lse)
        torch.cuda.current_stream().wait_stream(s)
        parts.append((out.double(), lse.double()))
    (whole, lse), (a, la), (z, lz) = parts
    top = torch.logaddexp(la, lz)
    joined = a * torch.exp(la - top)[..., None] + z * torch.exp(lz - top)[..., None]
    assert torch.allclose(top, lse, atol=2e-6, rtol=0)
    bound = cu_.HALF_BF16 * (whole.abs() + a.abs() + z.abs()) + 1e-4
    assert bool(((joined - whole).abs() <= bound).all())


@pytest.mark.parametrize("news", [[1, 1, 1], [4, 1, 0], [9, 1, 2], [70, 1, 1]])
def test_captured_calls_of_large_batches(news):
    """As below, for what a large bound on lengths selects: equal parts of all keys, chunks in the many-row kernel, and steps beside them."""
    rng = np.random.default_rng([28, news[0]])
    top = [3000, 500, 200]
    c = cu_.Cache(rng, top, n_kv=2, d=128, page=64, width_more=17000)
    batch, cu = cu_.make_batch(c, news, 8, max_kv=1 << 20)
    lens, table, pages = batch._keep[2], batch._keep[3], c.pages()
    q = cu_.bf16(rng.standard_normal((sum(news), 8, 128))).cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    ws = cu_.workspace(batch, pages)
    run = lambda: b.codecomp_attend(q, batch, pages, 0, out, ws, lse=lse)  # noqa: E731
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for i in range(4):
        now = [max(n, int(x)) for n, x in zip(news, rng.integers(0, top))]
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        c.table[c.table >= 0] = rng.permutation(c.n_pages).astype(np.int32)[: int((c.table >= 0).sum())]
        table.copy_(torch.from_numpy(c.table))
        q.copy_(cu_.bf16(rng.standard_normal(q.shape)))
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        run()
        assert torch.equal(out, got) and torch.equal(lse, got_lse)
        want = orc.attend(cu_.f64(q), *c.values(), c.table, now, cu, max_kv_len=1 << 20)
        cu_.assert_attended(got, got_lse, want, 128)


@pytest.mark.parametrize("news", [[1, 1, 1], [40, 1, 30]])
def test_captured_calls_follow_lengths_and_tables(news):
    """A step (append and attend) in a graph; lengths, tables, tokens and positions change between replays; two graphs with workspaces of their
    own run in turn, with eager calls between them."""
    rng = np.random.default_rng(18)
    top = [400, 150, 90]
    T = sum(news)
    c = cu_.Cache(rng, top, n_kv=2, d=128, page=16)
    batch, cu = cu_.make_batch(c, news, 8, max_kv=400)
    lens, table = batch._keep[2], batch._keep[3]
    pages, rot = c.pages(), b.make_rotary(128)
    q, k, v = (cu_.bf16(rng.standard_normal((T, n, 128))).cuda() for n in (8, 2, 2))
    pos = torch.zeros(T, dtype=torch.int32, device="cuda")
    turned, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(T, 8, device="cuda")

    def step(ws, out=out, lse=lse):
        b.codecomp_append(q, k, v, pos, rot, batch, pages, 0, turned)
        b.codecomp_attend(turned, batch, pages, 0, out, ws, lse=lse)

    graphs = []
    for _ in range(2):
        ws = cu_.workspace(batch, pages)
        step(ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(ws)
        graphs.append((g, ws))
    eager_ws = cu_.workspace(batch, pages)
    for i in range(6):
        lens.copy_(torch.tensor([max(n, int(x)) for n, x in zip(news, rng.integers(1, top))], dtype=torch.int32))
        order = rng.permutation(c.n_pages).astype(np.int32)
        c.table[c.table >= 0] = order[: int((c.table >= 0).sum())]
        table.copy_(torch.from_numpy(c.table))
        q.copy_(cu_.bf16(rng.standard_normal(q.shape)))
        k.copy_(cu_.bf16(rng.standard_normal(k.shape)))
        pos.copy_(torch.from_numpy(rng.integers(0, 100000, T).astype(np.int32)))
        out.zero_()
        graphs[i % 2][0].replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        step(eager_ws)
        assert torch.equal(out, got) and torch.equal(lse, got_lse)
        kk, vv = c.values()
        want = orc.attend(cu_.f64(turned), kk, vv, c.table, lens.cpu().numpy(), cu, max_kv_len=400)
        cu_.assert_attended(got, got_lse, want, 128)


@pytest.mark.parametrize("fp8", [False, True])
def test_from_compression_to_single_steps(fp8):
    """Two chunks are compressed, their compact rows go one behind the other into the pages of one request, the query's tokens are
    appended at their own positions and attended, the request forks, and both go on by single tokens; then its cache is compacted once more."""
    rng = np.random.default_rng(19)
    L, Hq, Hkv, d, W, page = 2, 4, 2, 64, 16, 16
    lens, budgets = np.array([300, 200]), np.array([60, 45])
    cu, cb = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (lens, budgets))
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    dcu, dcb = dev(cu), dev(cb)
    kv = lambda n: (torch.randn(L, Hkv, n, d) * (30 if fp8 else 1)).to(torch.float8_e4m3fn if fp8 else torch.bfloat16).cuda()  # noqa: E731
    torch.manual_seed(4)
    k, v = kv(500), kv(500)
    q_obs = torch.randn(L, 2, Hq, W, d).bfloat16().cuda()
    params = b.make_params(n_layers=L, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, window=W, pool_kernel=5, prior_weight=1.0, cu_seqlens_host=cu,
                           cu_budgets_host=cb, cu_seqlens_dev=dcu.data_ptr(), cu_budgets_dev=dcb.data_ptr(), kv_dtype=b.KV_FP8_E4M3 if fp8 else b.KV_BF16,
                           softmax_scale=0.01 if fp8 else 0.0)
    prior = torch.zeros(500, device="cuda")
    scores, idx = torch.empty(L, Hkv, 500, device="cuda"), torch.empty(L, Hkv, 105, dtype=torch.int32, device="cuda")
    ko, vo = torch.empty_like(kv(105)), torch.empty_like(kv(105))
    ws = torch.empty(b.codecomp_workspace_bytes(params), dtype=torch.uint8, device="cuda")
    b.codecomp_compress(q_obs, k, v, prior, params, scores, idx, ko, vo, ws)
    scale = 0.03 if fp8 else 1.0
    shape = (L, 40, Hkv, page, d)
    pk, pv = (torch.zeros(shape, dtype=torch.uint8 if fp8 else torch.bfloat16, device="cuda").view(k.dtype) for _ in range(2))
    pages = b.make_pages(pk, pv, k_scale=scale, v_scale=scale)
    order = rng.permutation(40).astype(np.int32)
    table = np.stack([order[:12], order[:12]])                       # request 1 is still nobody's: it will be the fork
    both = dev(np.stack([table[0], table[0]]))
    b.codecomp_pages_store(ko, vo, None, params, pages, both, dev(np.array([0, budgets[0]], np.int32)))
    have = torch.cat([ko, vo], 0).float().double().cpu().numpy() * scale
    mine = [[[list(have[l, h]), list(have[L + l, h])] for h in range(Hkv)] for l in range(L)]
    rot, freq = b.make_rotary(d), orc.frequencies(d)
    at, n = int(lens.max()), 105                                      # positions of the query: behind the longest chunk
    caches = [mine]

    def tokens(count, seqs, n, tab):
        """`count` new tokens of each request at positions at .. : appended, attended, and the same in fp64."""
        T = count * seqs
        cuq = (np.arange(seqs + 1) * count).astype(np.int32)
        x = b.make_batch(n_q_heads=Hq, cu_q_host=cuq, cu_q=dev(cuq), kv_lens=torch.full((seqs,), n + count, dtype=torch.int32, device="cuda"), table=dev(tab[:seqs]),
                         max_kv_len=12 * page)
        pos = np.tile(np.arange(at, at + count), seqs).astype(np.int32)
        work = cu_.workspace(x, pages)
        for l in range(L):
            q, kn, vn = (torch.randn(T, h, d).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
            out, turned = torch.empty_like(q), torch.empty_like(q)
            b.codecomp_append(q, kn, vn, dev(pos), rot, x, pages, l, turned)
            b.codecomp_attend(turned, x, pages, l, out, work)
            exact = orc.rotate(cu_.f64(kn), pos, freq)
            stored = cu_.f64(pk), cu_.f64(pv)
            for r in range(seqs):
                for i in range(count):
                    p, row = orc.place(tab, r, n + i, page, 40)
                    for h in range(Hkv):
                        got_k, got_v = stored[0][l, p, h, row] * scale, stored[1][l, p, h, row] * scale
                        step = 2.0 ** -4 if fp8 else 2.0 ** -8
                        assert np.all(np.abs(got_k - exact[r * count + i, h]) <= step * np.abs(exact[r * count + i, h]) + 2.0 ** -10 * scale + 1e-5)
                        caches[r][l][h][0].append(got_k)
                        caches[r][l][h][1].append(got_v)
            for r in range(seqs):
                kk = np.stack([np.stack(caches[r][l][h][0]) for h in range(Hkv)])[None]
                vv = np.stack([np.stack(caches[r][l][h][1]) for h in range(Hkv)])[None]
                part = slice(r * count, (r + 1) * count)
                want = orc.attend(cu_.f64(turned)[part], kk, vv, np.zeros((1, 1), np.int32), [n + count], [0, count], max_kv_len=n + count)
                cu_.assert_attended(out[part], None, want, d)

    tokens(35, 1, n, table)
    n, at = n + 35, at + 35
    full = n // page                                                  # whole pages are shared, the last one is copied
    table[1, full:] = order[12: 24 - full]
    b.codecomp_pages_copy(pages, dev(np.array([[table[0, full], table[1, full]]], np.int32)))
    caches.append([[[list(a) for a in caches[0][l][h]] for h in range(Hkv)] for l in range(L)])
    for _ in range(3):
        tokens(1, 2, n, table)
        n, at = n + 1, at + 1
    # compacted: every second row of the first request into new pages
    kept = np.tile(np.arange(0, n, 2, dtype=np.int32), (L, Hkv, 1))
    m = kept.shape[2]
    again = b.make_params(n_layers=L, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, window=1, pool_kernel=1, prior_weight=0.0,
                          cu_seqlens_host=np.array([0, n]), cu_budgets_host=np.array([0, m]), cu_seqlens_dev=dev(np.array([0, n], np.int32)).data_ptr(),
                          cu_budgets_dev=0, kv_dtype=params.kv_dtype)
    keep_dev = dev(np.array([0, n], np.int32)), dev(np.array([0, m], np.int32))
    again.cu_seqlens_dev, again.cu_budgets_dev = keep_dev[0].data_ptr(), keep_dev[1].data_ptr()
    new_table = np.array([[order[30 + i] for i in range(10)] + [-1, -1]], np.int32)
    b.codecomp_pages_compact(pages, dev(table[:1]), None, dev(kept), again, pages, dev(new_table))
    caches[:] = [[[[a[::2] for a in caches[0][l][h]] for h in range(Hkv)] for l in range(L)]]
    tokens(1, 1, m, new_table)


# Values of rows that all new tokens see, in the tile where some rows are not seen by all, and before it; chunks, equal parts, both kernels, small pages.
@pytest.mark.parametrize("news, n_q", [([1, 1], 8), ([6, 3], 8), ([9, 14], 8), ([150, 90], 1), ([40, 300], 8)])
@pytest.mark.parametrize("d, fp8", [(128, False), (64, True), (64, False), (128, True)])
@pytest.mark.parametrize("page, max_kv", [(16, 400), (8, 400), (256, 1 << 20)])
def test_infinities_and_nan_among_values_that_are_seen(news, n_q, d, fp8, page, max_kv):
    """One element of one value row: that element of every token that sees the row is infinite or NaN, everything else keeps its bits."""
    rng = np.random.default_rng([31, d, page, news[0]])
    lens = [333, 310]
    c = cu_.Cache(rng, lens, n_kv=1, d=d, page=page, fp8=fp8, width_more=max_kv // page + 1, k_scale=0.03 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
    batch, cu = cu_.make_batch(c, news, n_q, max_kv=max_kv)
    q = cu_.bf16(rng.standard_normal((sum(news), n_q, d))).cuda()
    ws = cu_.workspace(batch, c.pages())
    clean, lse, got, got_lse = torch.empty_like(q), torch.empty(sum(news), n_q, device="cuda"), torch.empty_like(q), torch.empty(sum(news), n_q, device="cuda")
    b.codecomp_attend(q, batch, c.pages(), 0, clean, ws, lse=lse)
    raw = c.v.view(torch.uint8) if fp8 else c.v
    own = lens[0] - news[0]                                             # row of the first new token: the last that all see
    for key in sorted({0, own - 1, own, (own + 1) // 32 * 32, (own + 1) // 64 * 64, (own + 1) // 64 * 64 - 1, own + news[0] // 2, lens[0] - 1}):
        p, at = orc.place(c.table, 0, key, page, c.n_pages)
        for x in [0x7F, 0xFF] if fp8 else [float("nan"), float("inf"), -float("inf")]:
            keep, e = raw[0, p, 0, at].clone(), int(rng.integers(d))
            raw[0, p, 0, at, e] = x
            b.codecomp_attend(q, batch, c.pages(), 0, got, ws, lse=got_lse)
            raw[0, p, 0, at] = keep
            sees = max(0, key - own)                                    # tokens of request 0 from there on
            hit = torch.zeros_like(got, dtype=torch.bool)
            hit[sees: news[0], :, e] = True
            assert not bool(torch.isfinite(got[hit]).any()), (key, x)
            assert torch.equal(got[~hit], clean[~hit]) and torch.equal(got_lse, lse), (key, x)


@pytest.mark.parametrize("news", [1, 90])
@pytest.mark.parametrize("max_kv", [200, 5000])
def test_infinite_values_of_weight_zero(news, max_kv):
    """Keys that give a logit of minus infinity weigh nothing, and nothing times an infinite value is NaN."""
    rng = np.random.default_rng(32)
    c = cu_.Cache(rng, [152], n_kv=1, d=64, page=8, width_more=max_kv // 8)
    batch, _ = cu_.make_batch(c, [news], 2, max_kv=max_kv, causal=False)
    q = cu_.bf16(rng.standard_normal((news, 2, 64))).cuda()
    q[..., 3] = 1.0
    for j in range(32, 64):                       # all keys that a wave has
        p, at = orc.place(c.table, 0, j, 8, c.n_pages)
        c.k[0, p, 0, at, 3] = -float("inf")
    out, ws = torch.empty_like(q), cu_.workspace(batch, c.pages())
    b.codecomp_attend(q, batch, c.pages(), 0, out, ws)
    assert bool(torch.isfinite(out).all())
    p, at = orc.place(c.table, 0, 40, 8, c.n_pages)
    c.v[0, p, 0, at, 7] = float("inf")
    b.codecomp_attend(q, batch, c.pages(), 0, out, ws)
    assert bool(torch.isnan(out[..., 7]).all()) and bool(torch.isfinite(out[..., :7]).all())


def guarded(monkeypatch):
    """Workspaces of exactly the bytes asked for, with a pattern behind them; returns what checks the pattern."""
    made = []
    def workspace(batch, pages):
        n = b.codecomp_attend_workspace_bytes(batch, pages)
        whole = torch.full((n + (1 << 16),), 0xFF, dtype=torch.uint8, device="cuda")
        whole[n:] = 0xA5
        made.append((whole, n))
        return whole[:n]
    monkeypatch.setattr(cu_, "workspace", workspace)
    def intact():
        assert made and all(bool((w[n:] == 0xA5).all()) for w, n in made)
        return [n for _, n in made]
    return intact


# Both kernels in one call, each with a workspace: equal parts of many steps beside a chunk, chunks of keys beside one (up to 32 rows, and 33 to 64), from 8 bits
# equal parts as well.
@pytest.mark.parametrize("short, count, long, n_q, n_kv, d, fp8, max_kv", [
    (1, 300, 90, 8, 4, 64, False, 5000), (2, 260, 40, 16, 4, 128, False, 3000), (1, 12, 90, 4, 2, 64, True, 4096), (5, 12, 90, 16, 2, 128, True, 4096),
    (9, 12, 70, 8, 2, 64, True, 4096), (1, 12, 90, 4, 2, 128, True, 1 << 20)])
@pytest.mark.parametrize("causal", [True, False])
def test_both_kernels_share_a_workspace(monkeypatch, short, count, long, n_q, n_kv, d, fp8, max_kv, causal):
    intact = guarded(monkeypatch)
    rng = np.random.default_rng([35, count, d])
    news = [short] * count
    news[count // 2], news[3] = long, 0
    lens = [int(x) for x in rng.integers(0, 60, count)]
    lens[0], lens[count // 2], lens[-1] = min(max_kv, 2700), min(max_kv, 1900), 1100
    c = cu_.Cache(rng, lens, n_kv=n_kv, d=d, page=64, fp8=fp8, width_more=max_kv // 64 - 40, k_scale=0.03 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
    check(rng, c, news, n_q, causal=causal, max_kv=max_kv)
    both, = intact()
    alone, _ = cu_.make_batch(c, [long if r == count // 2 else 0 for r in range(count)], n_q, max_kv=max_kv)
    assert both > b.codecomp_attend_workspace_bytes(alone, c.pages()) > 0


@pytest.mark.parametrize("lens, news, n_q, n_kv, d, fp8, max_kv", [
    ([3000, 90], [1, 2], 4, 2, 64, False, 3000), ([3000, 900, 7], [9, 1, 3], 4, 1, 128, True, 3000), ([3000, 90, 0], [1, 1, 1], 8, 2, 128, False, 1 << 20),
    ([3000, 800], [300, 90], 2, 2, 128, False, 3000), ([3000, 800], [700, 1], 4, 2, 64, True, 3000), ([1300, 140], [9, 16], 8, 2, 64, False, 100000)])
def test_workspaces_are_not_written_beyond(monkeypatch, lens, news, n_q, n_kv, d, fp8, max_kv):
    intact = guarded(monkeypatch)
    rng = np.random.default_rng([36, d, news[0]])
    c = cu_.Cache(rng, lens, n_kv=n_kv, d=d, page=256, fp8=fp8, width_more=max_kv // 256, k_scale=0.03 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
    check(rng, c, news, n_q, max_kv=max_kv)
    assert intact()[0] > 0


# Beside a long chunk as well a request of up to 64 rows has weights of 16 bits: it goes along with the chunk or takes the other kernel, over caches that are short
# and long by the host's bound, in pages of more and of less than 16 rows.
@pytest.mark.parametrize("news, n_q, n_kv, d", [([1, 90, 2, 8], 8, 2, 128), ([16, 1, 70, 9], 8, 2, 64), ([64, 65, 1, 33], 1, 1, 64), ([1, 300, 9, 4], 14, 2, 128)])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page, max_kv", [(16, 1300), (8, 1300), (256, 1 << 20)])
def test_weights_of_short_requests_beside_long_ones(news, n_q, n_kv, d, fp8, page, max_kv):
    rng = np.random.default_rng([37, d, page, news[0]])
    lens = [1300, 700, 290, 900]
    c = cu_.Cache(rng, lens, n_kv=n_kv, d=d, page=page, fp8=fp8, width_more=max_kv // page, k_scale=0.03 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
    for causal in (True, False):
        _, _, out, lse, want = check(rng, c, news, n_q, causal=causal, max_kv=max_kv)
        cu = np.concatenate([[0], np.cumsum(news)])
        short = [r for r, n in enumerate(news) if n * n_q // n_kv <= 64]
        assert 0 < len(short) < len(news)
        for r in short:
            part = slice(int(cu[r]), int(cu[r + 1]))
            cu_.assert_attended(out[part], lse[part], tuple(x[part] for x in want), d, 16)
