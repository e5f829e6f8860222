"""Rotary positions, appends and moves of rows on a paged cache against the fp64 oracle (copies: bit for bit)."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from paper_2604_10235_amd import binding as b
from tests import cache_util as cu_

pytestmark = pytest.mark.gpu

POSITIONS = [0, 1, -1, 7, 4095, 123457, 2**31 - 1, -(2**31), 1048583, 33]


def rotary_tolerance(want, x, positions, freq, magnitude):
    """Half a bf16 step; of the pair's length, what fp32 adds: sine and cosine to 2^-22 (angle 2^-24 of pi / 4 at most, polynomial, its
    roundings), two products and a sum of half a step each; and the frequency held to 2^-53 relative, twice (turns, and a turn's 64 bits)."""
    pair = np.sqrt(2.0) * np.abs(x).max(axis=-1, keepdims=True) * magnitude
    angle = np.abs(np.asarray(positions, dtype=np.float64))[:, None, None] * freq.max() * 2.0 ** -51
    return cu_.HALF_BF16 * np.abs(want) + pair * (2.0 ** -21 + angle)


@pytest.mark.parametrize("T, H, d, dim, inter, inverse, scaling, magnitude", [
    (1, 1, 64, 64, False, False, "plain", 1.0), (10, 3, 128, 128, False, False, "plain", 1.0), (10, 5, 128, 64, True, False, "linear", 1.0),
    (9, 8, 64, 16, False, True, "base", 1.0), (10, 36, 128, 32, True, True, "wavelength", 1.0), (10, 7, 128, 112, False, False, "ramp", 1.1386),
    (10, 2, 64, 48, True, False, "plain", 1.0), (1000, 9, 128, 128, False, True, "plain", 0.5), (333, 40, 64, 64, True, False, "ramp", 1.0)])
def test_rotate(T, H, d, dim, inter, inverse, scaling, magnitude):
    rng = np.random.default_rng([T, H, dim])
    x = cu_.bf16(rng.standard_normal((T, H, d)))
    pos = np.array((POSITIONS * 100)[:T], np.int32)
    kw = dict(factor=4.0, context=8192.0, low=1.0, high=32.0)
    rot = b.make_rotary(dim, scaling=b.ROTARY_SCALINGS[scaling], interleaved=inter, inverse=inverse, magnitude=magnitude, **kw)
    freq = orc.frequencies(dim, 10000.0, scaling, **kw)
    out = torch.full((T, H, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    b.codecomp_rotate(x.cuda(), torch.from_numpy(pos).cuda(), rot, out)
    xf = cu_.f64(x)
    want = orc.rotate(xf, pos, freq, interleaved=inter, inverse=inverse, magnitude=magnitude)
    off = np.abs(cu_.f64(out) - want)
    tol = rotary_tolerance(want, xf, pos, freq, magnitude)
    assert np.all(off <= tol), float((off / tol).max())
    assert np.array_equal(cu_.f64(out)[..., dim:], xf[..., dim:])        # not rotated: copied


def test_rotate_views_in_place_and_other_stream():
    """Query and key heads of a fused projection, rotated in place on a stream of their own: the value heads behind them stay."""
    rng = np.random.default_rng(5)
    fused = cu_.bf16(rng.standard_normal((37, 12, 128))).cuda()
    before, pos = fused.clone(), torch.arange(37, dtype=torch.int32, device="cuda") * 1000
    rot = b.make_rotary(128)
    want = torch.empty((37, 8, 128), dtype=torch.bfloat16, device="cuda")
    b.codecomp_rotate(fused[:, :8], pos, rot, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.codecomp_rotate(fused[:, :8], pos, rot, fused[:, :8])
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(fused[:, :8], want) and torch.equal(fused[:, 8:], before[:, 8:])
    assert not torch.equal(want, before[:, :8])


def test_inverse_is_the_gradient():
    """<R x, y> = <x, R' y>, against autograd of the formula in 64 bits, and against differences."""
    rng = np.random.default_rng(6)
    x, y = (cu_.bf16(rng.standard_normal((5, 3, 64))) for _ in range(2))
    pos, freq = np.array([0, 3, -17, 1000, 65537], np.int32), orc.frequencies(32)
    rot = b.make_rotary(32, interleaved=True, inverse=True, magnitude=1.25)
    g = torch.empty((5, 3, 64), dtype=torch.bfloat16, device="cuda")
    b.codecomp_rotate(y.cuda(), torch.from_numpy(pos).cuda(), rot, g)
    f = lambda v: float((orc.rotate(v, pos, freq, interleaved=True, magnitude=1.25) * cu_.f64(y)).sum())  # noqa: E731
    want = np.zeros((5, 3, 64))
    base = np.zeros((5, 3, 64))
    for i in np.ndindex(5, 3, 64):               # the map is linear: one difference is the derivative
        base[i] = 1.0
        want[i] = f(base)
        base[i] = 0.0
    tol = rotary_tolerance(want, cu_.f64(y), pos, freq, 1.25)
    assert np.all(np.abs(cu_.f64(g) - want) <= tol)
    leaf = torch.tensor(cu_.f64(x), requires_grad=True)
    a = torch.from_numpy(pos).double()[:, None] * torch.from_numpy(freq)
    p = leaf[..., :32].unflatten(-1, (16, 2))
    c, s = a.cos()[:, None], a.sin()[:, None]
    r = 1.25 * torch.stack([p[..., 0] * c - p[..., 1] * s, p[..., 0] * s + p[..., 1] * c], -1).flatten(-2)
    (torch.cat([r, leaf[..., 32:]], -1) * torch.tensor(cu_.f64(y))).sum().backward()
    assert np.all(np.abs(cu_.f64(g) - leaf.grad.numpy()) <= tol)


@pytest.mark.parametrize("news, lens, n_q, n_kv, d, dim, inter, fp8, page", [
    ([1], [1], 4, 4, 64, 64, False, False, 16), ([1, 1, 1], [5, 16, 33], 28, 4, 128, 128, False, False, 16),
    ([3, 0, 9, 1], [70, 12, 9, 64], 8, 2, 128, 64, True, True, 64), ([17, 40], [17, 131], 14, 2, 128, 128, False, True, 8),
    ([5, 6], [40, 41], 3, 1, 64, 32, False, True, 1), ([0, 0, 4, 0], [9, 9, 9, 9], 2, 2, 64, 0, False, False, 32)])
def test_append(news, lens, n_q, n_kv, d, dim, inter, fp8, page):
    rng = np.random.default_rng([len(news), d, page])
    c = cu_.Cache(rng, lens, n_kv=n_kv, d=d, page=page, fp8=fp8, layers=2, k_scale=0.02 if fp8 else 1.0, v_scale=0.0125 if fp8 else 1.0)
    T = sum(news)
    fused = cu_.bf16(rng.standard_normal((T, n_q + 2 * n_kv, d))).cuda()
    q, k, v = fused[:, :n_q], fused[:, n_q: n_q + n_kv], fused[:, n_q + n_kv:]
    pos = rng.integers(0, 200000, T).astype(np.int32)
    wide = (n_q + 2 * n_kv) * d
    batch, cu = cu_.make_batch(c, news, n_q, q_stride_tok=wide, new_stride_tok=wide)
    rot = b.make_rotary(dim, interleaved=inter) if dim else None
    freq = orc.frequencies(dim) if dim else np.zeros(0)
    old = c.k.clone(), c.v.clone()
    out = torch.full((T, n_q, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    b.codecomp_append(q, k, v, torch.from_numpy(pos).cuda(), rot, batch, c.pages(), 1, out)
    qf, kf, vf = cu_.f64(q), cu_.f64(k), cu_.f64(v)
    turn = (lambda x: orc.rotate(x, pos, freq, interleaved=inter)) if dim else (lambda x: x)
    tol = lambda w, x: rotary_tolerance(w, x, pos, freq, 1.0) if dim else cu_.HALF_BF16 * np.abs(w)  # noqa: E731
    assert np.all(np.abs(cu_.f64(out) - turn(qf)) <= tol(turn(qf), qf))
    touched = np.zeros((c.n_pages, page), bool)
    for name, pool, was, x, scale in (("k", c.k, old[0], turn(kf), c.k_scale), ("v", c.v, old[1], vf, c.v_scale)):
        got = cu_.f64(pool)
        for r, (n, length) in enumerate(zip(news, lens)):
            for i in range(n):
                p, at = orc.place(c.table, r, length - n + i, page, c.n_pages)
                touched[p, at] = True
                want = x[cu[r] + i] / scale
                if fp8:         # half a step of E4M3 relative (2^-4), or of its subnormals (2^-10); the fp32 before it, as above
                    want = np.clip(want, -448, 448)
                    lim = 2.0 ** -4 * np.abs(want) + 2.0 ** -10 + 1e-5 * np.abs(kf).max() / scale
                else:
                    lim = tol(x, kf)[cu[r] + i] if name == "k" else 0.0
                assert np.all(np.abs(got[1, p, :, at] - want) <= lim), (name, r, i)
        same = torch.from_numpy(~touched).cuda()
        as_int = lambda t: t.view(torch.uint8) if fp8 else t.view(torch.int16)  # noqa: E731
        assert torch.equal(as_int(pool)[0], as_int(was)[0])                                     # the other layer
        assert torch.equal(as_int(pool)[1].transpose(1, 2)[same], as_int(was)[1].transpose(1, 2)[same])


def test_append_drops_what_has_no_place():
    """Rows before the cache, pages that are not held or outside the pool: nothing is written; query heads come out all the same."""
    rng = np.random.default_rng(8)
    c = cu_.Cache(rng, [40, 40, 8, 40], n_kv=2, d=64, page=16)
    c.table[0, 1], c.table[1, 2] = -1, c.n_pages
    news = [20, 9, 12, 2]
    batch, cu = cu_.make_batch(c, news, 2, lens=[40, 40, 8, 1000])          # the third has fewer rows than new tokens, the last is cut to max_kv_len
    T = sum(news)
    k, v, q = (cu_.bf16(rng.standard_normal((T, 2, 64))).cuda() for _ in range(3))
    old, out = c.k.clone(), torch.empty_like(q)
    b.codecomp_append(q, k, v, None, None, batch, c.pages(), 0, out)
    assert torch.equal(out, q)
    want_k, want_v, seen = old.clone(), c.v.clone(), 0
    for r, n in enumerate(news):
        for i in range(n):
            at = orc.place(c.table, r, [40, 40, 8, 40][r] - n + i, 16, c.n_pages)
            if at is not None:
                want_k[0, at[0], :, at[1]] = k[cu[r] + i]
                want_v[0, at[0], :, at[1]] = v[cu[r] + i]
                seen += 1
    assert 0 < seen < T and torch.equal(c.k, want_k) and torch.equal(c.v, want_v)


def test_append_without_queries_in_place_and_8_bit_limits():
    rng = np.random.default_rng(9)
    c = cu_.Cache(rng, [8], n_kv=1, d=64, page=8, fp8=True)
    batch, _ = cu_.make_batch(c, [8], 3)
    k = torch.zeros((8, 1, 64), dtype=torch.bfloat16)
    k[0, 0, :10] = torch.tensor([448.0, 449.0, 464.0, 480.0, 1e30, float("inf"), -float("inf"), float("nan"), -600.0, 2.0 ** -10])
    b.codecomp_append(None, k.cuda(), k.cuda(), None, None, batch, c.pages(), 0, None)
    got = cu_.f64(c.k)[0, c.table[0, 0], 0, 0, :10]
    assert np.array_equal(got, [448, 448, 448, 448, 448, 448, -448, np.nan, -448, 0.0], equal_nan=True)      # 2^-10 is half of the smallest code: ties to even
    q = cu_.bf16(rng.standard_normal((8, 3, 64))).cuda()
    pos, rot = torch.arange(8, dtype=torch.int32, device="cuda"), b.make_rotary(64)
    out = torch.empty_like(q)
    b.codecomp_append(q, k.cuda(), k.cuda(), pos, rot, batch, c.pages(), 0, out)
    b.codecomp_append(q, k.cuda(), k.cuda(), pos, rot, batch, c.pages(), 0, q)
    assert torch.equal(out, q)


def rows_setup(rng, *, fp8, d, page, layers=2, n_kv=3, dense_pad=0):
    lens, budgets = [70, 1, 33], [20, 1, 33]
    cu, cb = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (lens, budgets))
    dev = torch.from_numpy(cu).cuda(), torch.from_numpy(cb).cuda()
    strides = {}
    if dense_pad:       # rows further apart than they are long
        strides = dict(kv_stride_tok=d + 16, kv_stride_head=(d + 16) * 104, kv_stride_layer=(d + 16) * 104 * n_kv,
                       out_stride_tok=d + 32, out_stride_head=(d + 32) * 54, out_stride_layer=(d + 32) * 54 * n_kv)
    params = b.make_params(n_layers=layers, n_q_heads=2 * n_kv, n_kv_heads=n_kv, head_dim=d, window=1, pool_kernel=1, prior_weight=0.0, cu_seqlens_host=cu,
                           cu_budgets_host=cb, cu_seqlens_dev=dev[0].data_ptr(), cu_budgets_dev=dev[1].data_ptr(),
                           kv_dtype=b.KV_FP8_E4M3 if fp8 else b.KV_BF16, **strides)
    params._dev = dev
    def dense(total, wide):
        x = torch.from_numpy(rng.integers(0, 256, (layers, n_kv, total, wide * (1 if fp8 else 2)), dtype=np.uint8)).cuda()
        return (x if fp8 else x.view(torch.bfloat16))[..., :d]
    idx = np.stack([np.concatenate([np.sort(rng.choice(n, m, replace=False)) for n, m in zip(lens, budgets)]) for _ in range(layers * n_kv)])
    idx = idx.reshape(layers, n_kv, -1).astype(np.int32)
    pad = dense_pad
    return lens, budgets, cu, cb, params, dense(104, d + (16 if pad else 0)), dense(54, d + (32 if pad else 0)), idx


def raw(t):
    return (t if t.dtype == torch.uint8 else t.contiguous().view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t.contiguous().view(torch.int16)).cpu().numpy()


@pytest.mark.parametrize("fp8, d, page, pad", [(False, 128, 16, 0), (True, 128, 8, 1), (False, 64, 1, 1), (True, 64, 64, 0)])
def test_rows_move_between_dense_and_pages(fp8, d, page, pad):
    rng = np.random.default_rng([d, page])
    lens, budgets, cu, cb, params, dense, compact, idx = rows_setup(rng, fp8=fp8, d=d, page=page, dense_pad=pad)
    first = np.array([3, 0, 21], np.int32)
    c = cu_.Cache(rng, [n + f for n, f in zip(lens, first)], n_kv=3, d=d, page=page, fp8=fp8, layers=2)
    c.table[0, 1] = -1                                   # a page that is not held
    tab, dev_first, dev_idx = c.dev_table(), torch.from_numpy(first).cuda(), torch.from_numpy(idx).cuda()
    bad = idx.copy()
    bad[0, 0, 0], bad[1, 2, -1] = -5, 1000               # cut into the request
    for use in (None, dev_idx, torch.from_numpy(bad).cuda()):
        src = compact if use is None else dense
        at = None if use is None else np.clip(use.cpu().numpy(), 0, np.repeat(np.array(lens) - 1, budgets)[None, None, :])
        c.k.copy_(c._fill(rng, c.k.shape, 1.0))
        c.v.copy_(c._fill(rng, c.k.shape, 1.0))
        want_k, want_v, s = raw(c.k).copy(), raw(c.v).copy(), raw(src)
        other = torch.flip(src, (0,)) if not pad else src        # V differs from K where strides allow
        b.codecomp_pages_store(src, other, use, params, c.pages(), tab, dev_first)
        o = raw(other)
        for r in range(3):
            for i in range(budgets[r]):
                p = orc.place(c.table, r, int(first[r]) + i, page, c.n_pages)
                if p is None:
                    continue
                for l in range(2):
                    for h in range(3):
                        row = cb[r] + i if use is None else cu[r] + at[l, h, cb[r] + i]
                        want_k[l, p[0], h, p[1]], want_v[l, p[0], h, p[1]] = s[l, h, row], o[l, h, row]
        assert np.array_equal(raw(c.k), want_k) and np.array_equal(raw(c.v), want_v)
        # and back
        into = [torch.zeros_like(dense if use is None else compact) for _ in range(2)]
        if pad:
            into = [torch.empty_strided(t.shape, (dense if use is None else compact).stride(), dtype=t.dtype, device="cuda") for t in into]
        b.codecomp_pages_load(c.pages(), tab, dev_first, use, params, *into)
        for got, pool in zip(into, (raw(c.k), raw(c.v))):
            g = raw(got)
            for r in range(3):
                for i in range(lens[r] if use is None else budgets[r]):
                    for l in range(2):
                        for h in range(3):
                            j = i if use is None else at[l, h, cb[r] + i]
                            p = orc.place(c.table, r, int(first[r]) + j, page, c.n_pages)
                            want = pool[l, p[0], h, p[1]] if p is not None else np.zeros_like(g[0, 0, 0])
                            assert np.array_equal(g[l, h, (cu if use is None else cb)[r] + i], want)


@pytest.mark.parametrize("fp8, d, page, page_to", [(False, 128, 16, 32), (True, 64, 4, 4)])
def test_compaction_equals_load_gather_store(fp8, d, page, page_to):
    rng = np.random.default_rng([d, page, 3])
    lens, budgets, cu, cb, params, dense, compact, idx = rows_setup(rng, fp8=fp8, d=d, page=page)
    c = cu_.Cache(rng, lens, n_kv=3, d=d, page=page, fp8=fp8, layers=2)
    to = cu_.Cache(rng, [n + 5 for n in budgets], n_kv=3, d=d, page=page_to, fp8=fp8, layers=2)
    ref = cu_.Cache(np.random.default_rng(0), [n + 5 for n in budgets], n_kv=3, d=d, page=page_to, fp8=fp8, layers=2)
    ref.k, ref.v, ref.table = to.k.clone(), to.v.clone(), to.table
    first, dev_idx = torch.tensor([5, 0, 2], dtype=torch.int32).cuda(), torch.from_numpy(idx).cuda()
    b.codecomp_pages_compact(c.pages(), c.dev_table(), None, dev_idx, params, to.pages(), to.dev_table(), first)
    k, v, ko, vo = torch.empty_like(dense), torch.empty_like(dense), torch.empty_like(compact), torch.empty_like(compact)
    b.codecomp_pages_load(c.pages(), c.dev_table(), None, None, params, k, v)
    b.codecomp_gather(k, v, dev_idx, params, ko, vo)
    b.codecomp_pages_store(ko, vo, None, params, ref.pages(), ref.dev_table(), first)
    assert np.array_equal(raw(to.k), raw(ref.k)) and np.array_equal(raw(to.v), raw(ref.v))
    # within one pool, into pages that were nobody's
    more = cu_.Cache(rng, lens, n_kv=3, d=d, page=page, fp8=fp8, layers=2, spare=60)
    spare = np.setdiff1d(np.arange(more.n_pages), more.table)
    table = np.full((3, 40), -1, np.int32)
    n = 0
    for r in range(3):
        need = -(-budgets[r] // page)
        table[r, :need] = spare[n: n + need]
        n += need
    b.codecomp_pages_compact(more.pages(), more.dev_table(), None, dev_idx, params, more.pages(), torch.from_numpy(table).cuda())
    b.codecomp_pages_load(more.pages(), more.dev_table(), None, dev_idx, params, ko, vo)
    for r in range(3):
        for i in range(budgets[r]):
            p = orc.place(table, r, i, page, more.n_pages)
            assert np.array_equal(raw(more.k)[:, p[0], :, p[1]], raw(ko)[:, :, cb[r] + i]) and np.array_equal(raw(more.v)[:, p[0], :, p[1]], raw(vo)[:, :, cb[r] + i])


@pytest.mark.parametrize("fp8, d, page, n_kv, layers", [(False, 128, 16, 4, 3), (True, 64, 1, 1, 2), (True, 128, 256, 3, 1), (False, 64, 32, 2, 2)])
def test_pages_copy(fp8, d, page, n_kv, layers):
    rng = np.random.default_rng([d, page, n_kv])
    c = cu_.Cache(rng, [page * 12], n_kv=n_kv, d=d, page=page, fp8=fp8, layers=layers)
    pairs = np.array([[0, 5], [0, 6], [3, 7], [2, 2], [-1, 8], [9, c.n_pages], [c.n_pages + 4, 10], [4, -2]], np.int32)
    want_k, want_v = raw(c.k).copy(), raw(c.v).copy()
    for a, z in ((0, 5), (0, 6), (3, 7)):
        want_k[:, z], want_v[:, z] = want_k[:, a], want_v[:, a]
    b.codecomp_pages_copy(c.pages(), torch.from_numpy(pairs).cuda())
    assert np.array_equal(raw(c.k), want_k) and np.array_equal(raw(c.v), want_v)


@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_of_far_positions_and_any_frequency(interleaved):
    """Against angles reduced with 1 / (2 pi) in whole numbers of 1500 bits (pi by Machin's formula): the error does not grow with the position or the
    frequency, and the inverse is the rotation at minus the position."""
    bits = 1500
    def arctan_of_one_over(x):
        term = total = (1 << bits + 64) // x
        k, sign = 3, -1
        while term:
            term //= x * x
            total, sign, k = total + sign * (term // k), -sign, k + 2
        return total
    pi = (16 * arctan_of_one_over(5) - 4 * arctan_of_one_over(239)) >> 64
    per_radian = (1 << 2 * bits) // (2 * pi)                              # 2^1500 / (2 pi)
    freqs = [1.0, 12345.678, 1e6 + 0.1, 2.0 ** 52 + 1, 2.0 ** 53 + 2, 1e15, 1e22, 1e100, 1e300, 1.7e308, 5e-324, 2.0 ** -70, 3e-11, 1e-5, 0.7, 0.0, -0.3, -98765.4, -1e40,
             3.0, 6.283185307179586, 100.0, 2.0 ** 63 + 2048, 1e-3, 1e-8, 2.0 ** 64, 1e19, 2.0 ** 117, 31.4159, 1e9, 7e4, 1e-19]
    pos = np.array(POSITIONS + [2**31 - 2, -(2**31) + 1, 987654321], np.int32)
    rng = np.random.default_rng(33)
    x = cu_.bf16(rng.standard_normal((len(pos), 3, 64)))
    rot = b.make_rotary(64, interleaved=interleaved)
    rot.freq[:32] = freqs
    out = torch.empty_like(x, device="cuda")
    b.codecomp_rotate(x.cuda(), torch.from_numpy(pos).cuda(), rot, out)
    angle = np.zeros((len(pos), 32))
    for i, p in enumerate(pos):
        for j, f in enumerate(freqs):
            num, den = float(f).as_integer_ratio()
            turns = (num * int(p) * per_radian // den) & ((1 << bits) - 1)
            angle[i, j] = 2 * np.pi * ((turns >> (bits - 64)) / 2.0 ** 64)
    xf = cu_.f64(x)
    x0, x1 = (xf[..., 0::2], xf[..., 1::2]) if interleaved else (xf[..., :32], xf[..., 32:])
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    y0, y1 = x0 * c - x1 * s, x0 * s + x1 * c
    want = np.stack([y0, y1], -1).reshape(xf.shape) if interleaved else np.concatenate([y0, y1], -1)
    off, tol = np.abs(cu_.f64(out) - want), rotary_tolerance(want, xf, pos * 0, np.zeros(1), 1.0)
    assert np.all(off <= tol), (float((off / tol).max()), np.unravel_index(np.argmax(off / tol), off.shape))
    # the transpose, exactly: also for the smallest frequencies
    near = pos[pos > -(2**31)]
    back, turned = torch.empty_like(out[: len(near)]), torch.empty_like(out[: len(near)])
    b.codecomp_rotate(x[: len(near)].cuda(), torch.from_numpy(-near).cuda(), rot, turned)
    rot.inverse = 1
    b.codecomp_rotate(x[: len(near)].cuda(), torch.from_numpy(near).cuda(), rot, back)
    assert torch.equal(back, turned)


# Calls long enough for four heads a thread (more than 3 * 2^16 units of 16 elements), whose last group is not full; append: groups of query, key and value heads.
@pytest.mark.parametrize("T, H, d, dim, inter, inverse, scaling, magnitude", [
    (1401, 18, 128, 128, False, False, "plain", 1.0), (1401, 18, 128, 64, True, True, "wavelength", 1.0), (10007, 5, 64, 64, True, False, "ramp", 1.1386),
    (7111, 7, 64, 32, False, True, "base", 0.5), (24600, 1, 128, 96, False, False, "linear", 1.0)])
def test_rotate_of_long_calls(T, H, d, dim, inter, inverse, scaling, magnitude):
    assert T * H * (d // 16) > 3 << 16
    rng = np.random.default_rng([T, H, dim])
    fused = cu_.bf16(rng.standard_normal((T, H + 2, d))).cuda()                 # strided: two more heads behind those that are rotated
    x, pos = fused[:, :H], rng.integers(-(2**31), 2**31, T).astype(np.int32)
    kw = dict(factor=4.0, context=8192.0, low=1.0, high=32.0)
    rot = b.make_rotary(dim, scaling=b.ROTARY_SCALINGS[scaling], interleaved=inter, inverse=inverse, magnitude=magnitude, **kw)
    freq = orc.frequencies(dim, 10000.0, scaling, **kw)
    out, dev_pos = torch.full((T + 1, H, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.from_numpy(pos).cuda()
    b.codecomp_rotate(x, dev_pos, rot, out[:T])
    xf, got = cu_.f64(x), cu_.f64(out[:T])
    want = orc.rotate(xf, pos, freq, interleaved=inter, inverse=inverse, magnitude=magnitude)
    off, tol = np.abs(got - want), rotary_tolerance(want, xf, pos, freq, magnitude)
    assert np.all(off <= tol), float((off / tol).max())
    assert np.array_equal(got[..., dim:], xf[..., dim:]) and bool((out[T] == 7.0).all())
    few = torch.empty((50, H, d), dtype=torch.bfloat16, device="cuda")              # a short call of the same tokens: the same bits
    b.codecomp_rotate(x[-50:], dev_pos[-50:], rot, few)
    assert torch.equal(few, out[T - 50: T])
    behind = fused[:, H:].clone()
    b.codecomp_rotate(x, dev_pos, rot, x)                                           # in place
    assert torch.equal(x, out[:T]) and torch.equal(fused[:, H:], behind)


LONG_APPENDS = [
    ([701, 0, 33, 650], [901, 5, 33, 650], 14, 2, 128, 128, False, False, 16), ([701, 0, 33, 650], [901, 5, 40, 650], 14, 2, 128, 64, True, True, 64),
    ([5001, 4990], [5001, 6000], 3, 1, 64, 64, False, True, 8), ([1, 5003, 2, 5001], [9, 5010, 2, 5001], 3, 1, 64, 32, True, False, 1),
    ([1300, 1301], [1300, 1400], 5, 5, 128, 0, False, False, 32)]


@pytest.mark.parametrize("news, lens, n_q, n_kv, d, dim, inter, fp8, page", LONG_APPENDS)
def test_append_of_long_chunks(news, lens, n_q, n_kv, d, dim, inter, fp8, page):
    assert sum(news) * (n_q + 2 * n_kv) * (d // 16) > 3 << 16 and (n_q + 2 * n_kv) % 4 != 0
    test_append(news, lens, n_q, n_kv, d, dim, inter, fp8, page)


@pytest.mark.parametrize("fp8", [False, True])
def test_append_of_long_chunks_in_place_and_without_queries(fp8):
    """Queries rotated in place, or none given: the pages get the same bits as from the call that writes elsewhere, and as from short calls."""
    rng = np.random.default_rng(34)
    news, n_q, n_kv, d = [4100, 4301], 6, 3, 64
    scales = dict(k_scale=0.02, v_scale=0.0125) if fp8 else {}
    c = cu_.Cache(rng, [4200, 4301], n_kv=n_kv, d=d, page=32, fp8=fp8, **scales)
    T, rot, pages = sum(news), b.make_rotary(d), c.pages()
    fused = cu_.bf16(rng.standard_normal((T, n_q + 2 * n_kv, d))).cuda()
    wide = (n_q + 2 * n_kv) * d
    q, k, v = fused[:, :n_q], fused[:, n_q: n_q + n_kv], fused[:, n_q + n_kv:]
    pos = torch.from_numpy(rng.integers(0, 10**6, T).astype(np.int32)).cuda()
    apart, cu = cu_.make_batch(c, news, n_q, q_stride_tok=wide, new_stride_tok=wide)
    inside, _ = cu_.make_batch(c, news, n_q, q_stride_tok=wide, new_stride_tok=wide, out_stride_tok=wide)
    was = raw(c.k).copy(), raw(c.v).copy()
    out = torch.empty((T, n_q, d), dtype=torch.bfloat16, device="cuda")
    b.codecomp_append(q, k, v, pos, rot, apart, pages, 0, out)
    want = raw(c.k).copy(), raw(c.v).copy()
    def again(run):
        for t, x in ((c.k, was[0]), (c.v, was[1])):
            (t.view(torch.uint8) if fp8 else t.view(torch.int16)).copy_(torch.from_numpy(x))
        run()
        assert np.array_equal(raw(c.k), want[0]) and np.array_equal(raw(c.v), want[1])
    behind = fused[:, n_q:].clone()
    keep = q.clone()
    again(lambda: b.codecomp_append(q, k, v, pos, rot, inside, pages, 0, q))
    assert torch.equal(q, out) and torch.equal(fused[:, n_q:], behind)
    q.copy_(keep)
    assert T * 2 * n_kv * (d // 16) > 3 << 16
    again(lambda: b.codecomp_append(None, k, v, pos, rot, apart, pages, 0, None))
    def by_parts():
        for lo in range(0, 4400, 400):
            part = [max(0, min(400, n - lo)) for n in news]
            at = torch.cat([torch.arange(cu[r] + lo, cu[r] + lo + n) for r, n in enumerate(part)]).cuda()
            x, _ = cu_.make_batch(c, part, n_q, lens=[length - n + lo + m for length, n, m in zip(c.lens, news, part)])
            b.codecomp_append(None, k[at].contiguous(), v[at].contiguous(), pos[at].contiguous(), rot, x, pages, 0, None)
    again(by_parts)
