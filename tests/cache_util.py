"""Paged caches with known contents for the tests: tensors on the GPU, the same numbers in fp64 on the CPU."""
import numpy as np
import torch

from paper_2604_10235_amd import binding as b


def bf16(x):
    return torch.as_tensor(np.asarray(x, dtype=np.float32)).to(torch.bfloat16)


def f64(t):
    return (t.view(torch.float8_e4m3fn) if t.dtype == torch.uint8 else t).float().double().cpu().numpy()


class Cache:
    """A pool of random rows and a table of pages in no order; `spare` pages are nobody's."""

    def __init__(self, rng, lens, *, n_kv=2, d=128, page=16, fp8=False, layers=1, spare=3, width_more=0, k_scale=1.0, v_scale=1.0, sharp=1.0):
        need = [-(-n // page) for n in lens]
        self.n_pages, self.page, self.d, self.fp8, self.lens = sum(need) + spare, page, d, fp8, list(lens)
        self.k_scale, self.v_scale = k_scale, v_scale
        order = rng.permutation(self.n_pages)[: sum(need)]
        self.table = np.full((len(lens), max(need + [1]) + width_more), -1, np.int32)
        for r, n in enumerate(need):
            self.table[r, :n] = order[sum(need[:r]): sum(need[: r + 1])]
        shape = (layers, self.n_pages, n_kv, page, d)
        self.k, self.v = (self._fill(rng, shape, s) for s in (sharp, 1.0))

    def _fill(self, rng, shape, sharp):
        x = torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)) * sharp
        return (x * 30).clamp(-448, 448).to(torch.float8_e4m3fn).cuda() if self.fp8 else x.to(torch.bfloat16).cuda()

    def pages(self):
        return b.make_pages(self.k, self.v, k_scale=self.k_scale, v_scale=self.v_scale)

    def dev_table(self):
        return torch.from_numpy(self.table).cuda()

    def values(self, layer=0):
        return f64(self.k[layer]) * self.k_scale, f64(self.v[layer]) * self.v_scale


def make_batch(cache, news, n_q, *, lens=None, max_kv=None, **kw):
    cu = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    lens = cache.lens if lens is None else lens
    x = b.make_batch(n_q_heads=n_q, cu_q_host=cu, cu_q=torch.from_numpy(cu).cuda(), kv_lens=torch.tensor(lens, dtype=torch.int32).cuda(),
                     table=cache.dev_table(), max_kv_len=max(list(cache.lens) + [1]) if max_kv is None else max_kv, **kw)
    return x, cu


def workspace(batch, pages):
    n = b.codecomp_attend_workspace_bytes(batch, pages)
    return torch.full((max(256, n),), 0xFF, dtype=torch.uint8, device="cuda")        # NaN, were it read as floats


# Half a step of the output type, and what fp32 arithmetic may add.  An attention weight is exp of a logit: the logit's own error (d products
# and sums of fp32, each half a step, of at most `reach` in all, and its scaling) is a relative error of the weight; exp itself is good
# to 2^-20.  Every weight is rounded to bf16 (2^-8) or to two bf16 (2^-16) on its way into the second product.
HALF_BF16 = 2.0 ** -8


def attend_tolerance(out, lse, spread, reach, d, weight_bits):
    logit = 2.0 ** -24 * (d + 16) * reach + 2.0 ** -23 * np.abs(np.where(np.isfinite(lse), lse, 0.0))
    weight = 2.0 * (logit + 2.0 ** -20) + 2.0 ** -weight_bits
    tol = HALF_BF16 * np.abs(out) + (1 + HALF_BF16) * weight[..., None] * spread + 2.0 ** -130
    return tol, logit + 2.0 ** -20


def assert_attended(got, got_lse, want, d, weight_bits=8):
    out, lse, spread, reach = want
    tol, tol_lse = attend_tolerance(out, lse, spread, reach, d, weight_bits)
    got = got.float().double().cpu().numpy()
    off = np.abs(got - out)
    assert np.all(off <= tol), (float((off / tol).max()), np.unravel_index(np.argmax(off / tol), off.shape))
    if got_lse is not None:
        g = got_lse.double().cpu().numpy()
        assert np.array_equal(np.isneginf(g), np.isneginf(lse))
        fin = np.isfinite(lse)
        assert np.all(np.abs(g[fin] - lse[fin]) <= tol_lse[fin]), float((np.abs(g[fin] - lse[fin]) / tol_lse[fin]).max())
