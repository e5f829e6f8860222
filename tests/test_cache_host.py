"""Operators on a paged cache, what needs no GPU: symbols and structures of the header, rotary frequencies, and every refusal with its code
(checked on the host before anything is launched)."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from oracle import cache_oracle as orc
from paper_2604_10235_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "codecomp_cache.h")
D = 0x1000          # a device pointer that is never followed: the calls below are refused, or launch nothing


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(b.LIB_PATH):
        from paper_2604_10235_amd import build
        build.build_library(verbose=False)


def test_header_is_c99_and_every_declared_function_is_exported():
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-fsyntax-only", "-x", "c", HEADER], check=True)
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(codecomp_[a-z_]+)\s*\(", text)))
    assert names == ["codecomp_append", "codecomp_attend", "codecomp_attend_validate", "codecomp_attend_workspace_bytes", "codecomp_pages_compact",
                     "codecomp_pages_copy", "codecomp_pages_load", "codecomp_pages_store", "codecomp_rotary_init", "codecomp_rotate"]
    for n in names:
        assert hasattr(b.lib(), n), n


def test_structures_are_laid_out_as_in_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    fields = {"codecomp_pages": b.codecomp_pages, "codecomp_batch": b.codecomp_batch, "codecomp_rotary": b.codecomp_rotary}
    lines = [f'printf("%zu\\n", sizeof({n})); ' + " ".join(f'printf("%zu\\n", offsetof({n}, {f[0]}));' for f in s._fields_) for n, s in fields.items()]
    src.write_text('#include <stdio.h>\n#include "codecomp_cache.h"\nint main(void) {' + "\n".join(lines) + "return 0; }\n")
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = [x for s in fields.values() for x in [C.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]]
    assert got == want


@pytest.mark.parametrize("dim", [16, 64, 128])
@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "wavelength", "ramp"])
def test_rotary_frequencies(dim, scaling):
    kw = dict(factor=4.0, context=8192.0, low=1.0, high=32.0 if scaling == "ramp" else 4.0)
    r = b.make_rotary(dim, base=50000.0, scaling=b.ROTARY_SCALINGS[scaling], **kw)
    assert (r.dim, r.interleaved, r.inverse, r.magnitude) == (dim, 0, 0, 1.0)
    np.testing.assert_allclose(np.array(r.freq[: dim // 2]), orc.frequencies(dim, 50000.0, scaling, **kw), rtol=1e-13)
    assert all(f == 0.0 for f in r.freq[dim // 2:])


def test_scaled_frequencies_lie_between_plain_and_slowed():
    for s in (b.ROTARY_WAVELENGTH, b.ROTARY_RAMP):
        plain = np.array(b.make_rotary(128).freq)
        got = np.array(b.make_rotary(128, scaling=s, factor=8.0, context=4096.0, low=1.0, high=32.0).freq)
        assert got[0] == plain[0] and got[63] == pytest.approx(plain[63] / 8.0, rel=1e-14)
        assert np.all(got <= plain) and np.all(got >= plain / 8.0 * (1 - 1e-14))
    # a factor of one changes nothing, whatever the way
    for s in b.ROTARY_SCALINGS.values():
        np.testing.assert_allclose(b.make_rotary(64, scaling=s, factor=1.0, context=4096.0).freq[:32], b.make_rotary(64).freq[:32], rtol=1e-14)


@pytest.mark.parametrize("bad", [dict(dim=0), dict(dim=24), dict(dim=144), dict(dim=-16), dict(base=1.0), dict(base=float("nan")), dict(scaling=5),
                                 dict(scaling=1, factor=0.5), dict(scaling=3, context=0.0), dict(scaling=3, context=100.0, low=4.0, high=4.0),
                                 dict(scaling=4, context=100.0, low=0.0, high=4.0), dict(scaling=2, factor=float("inf"))])
def test_rotary_init_refuses(bad):
    kw = dict(dim=64, base=10000.0, scaling=0, factor=2.0, context=4096.0, low=1.0, high=4.0)
    kw.update(bad)
    with pytest.raises(b.CodecompError) as e:
        b.make_rotary(kw.pop("dim"), **kw)
    assert e.value.status == -11
    assert b.lib().codecomp_rotary_init(None, 64, 0, 10000.0, 0, 1.0, 1.0, 1.0, 4.0) == -1


def pool(**over):
    p = b.codecomp_pages()
    p.k, p.v, p.n_layers, p.n_pages, p.page_size, p.n_kv_heads, p.head_dim, p.kv_dtype = D, D, 2, 9, 16, 4, 128, 0
    for k, v in over.items():
        setattr(p, k, v)
    return p


def batch(cu=(0, 1, 3), **over):
    x = b.codecomp_batch()
    host = np.array(cu, np.int32)
    x.n_seqs, x.n_q_heads, x.table_width, x.max_kv_len, x.causal = len(cu) - 1, 28, 4, 64, 1
    x.cu_q_host, x.cu_q_dev, x.kv_lens_dev, x.table_dev = host.ctypes.data, D, D, D
    x._keep = host
    for k, v in over.items():
        setattr(x, k, v)
    return x


def attend(x, p, layer=0, q=D, out=D, lse=None, ws=D, size=1 << 40):
    return b.lib().codecomp_attend(q, C.byref(x) if x else None, C.byref(p) if p else None, layer, out, lse, ws, size, None)


def append(x, p, layer=0, q=D, k=D, v=D, pos=D, rot="default", q_out=D):
    rot = b.make_rotary(64) if rot == "default" else rot
    return b.lib().codecomp_append(q, k, v, pos, C.byref(rot) if rot else None, C.byref(x) if x else None, C.byref(p) if p else None, layer, q_out, None)


POOLS = [(dict(k=None), -1), (dict(v=None), -1), (dict(head_dim=96), -7), (dict(kv_dtype=2), -11), (dict(n_kv_heads=0), -6), (dict(n_layers=0), -2),
         (dict(n_layers=20000), -2), (dict(n_pages=0), -12), (dict(page_size=0), -12), (dict(page_size=24), -12), (dict(page_size=1 << 17), -12),
         (dict(k=D + 8), -2), (dict(stride_tok=124), -2), (dict(stride_tok=64), -2), (dict(stride_head=-8), -2), (dict(stride_page=12), -2),
         (dict(kv_dtype=1, stride_tok=136), -2), (dict(k_scale=-1.0), -10), (dict(v_scale=float("nan")), -10), (dict(k_scale=float("inf")), -10)]
BATCHES = [(dict(cu_q_host=None), -1), (dict(cu_q_dev=None), -1), (dict(kv_lens_dev=None), -1), (dict(table_dev=None), -1), (dict(n_seqs=0), -2),
           (dict(n_seqs=65536), -2), (dict(n_q_heads=30), -6), (dict(n_q_heads=0), -6), (dict(causal=2), -11), (dict(softmax_scale=-0.5), -10),
           (dict(softmax_scale=float("inf")), -10), (dict(table_width=0), -12), (dict(max_kv_len=65), -12), (dict(max_kv_len=-1), -12),
           (dict(q_stride_tok=12), -2), (dict(q_stride_head=64), -2), (dict(out_stride_tok=-8), -2), (dict(new_stride_head=120), -2)]


@pytest.mark.parametrize("bad, code", POOLS, ids=str)
def test_a_bad_pool_is_refused_by_every_call(bad, code):
    x, p = batch(), pool(**bad)
    assert attend(x, p) == code and append(x, p) == code
    assert b.lib().codecomp_attend_validate(C.byref(x), C.byref(p)) == code
    assert b.lib().codecomp_attend_workspace_bytes(C.byref(x), C.byref(p)) == 0
    assert b.lib().codecomp_pages_copy(C.byref(p), D, 1, None) == code


@pytest.mark.parametrize("bad, code", BATCHES, ids=str)
def test_a_bad_batch_is_refused(bad, code):
    x, p = batch(**bad), pool()
    assert attend(x, p) == code and append(x, p) == code
    assert b.lib().codecomp_attend_validate(C.byref(x), C.byref(p)) == code


def test_token_offsets_are_checked():
    for cu in [(1, 2, 3), (0, 3, 2), (0, -1, 4)]:
        assert attend(batch(cu), pool()) == -8 and append(batch(cu), pool()) == -8
    assert attend(batch((0, 2**31 - 1)), pool()) == -2


def test_attend_refuses_pointers_layers_and_workspaces():
    x, p = batch(), pool()
    assert attend(x, p, q=None) == -1 and attend(x, p, out=None) == -1 and attend(None, p) == -1 and attend(x, None) == -1
    assert attend(x, p, layer=2) == -12 and attend(x, p, layer=-1) == -12
    assert attend(x, p, q=D + 2) == -2 and attend(x, p, out=D + 8) == -2 and attend(x, p, lse=D + 2) == -2
    need = b.lib().codecomp_attend_workspace_bytes(C.byref(x), C.byref(p))
    if need:
        assert attend(x, p, ws=None) == -9 and attend(x, p, ws=D + 16) == -9 and attend(x, p, size=need - 1) == -9


def test_calls_without_tokens_do_nothing():
    x, p = batch((0, 0, 0)), pool()
    assert attend(x, p) == 0 and append(x, p) == 0
    assert b.lib().codecomp_pages_copy(C.byref(p), None, 0, None) == 0
    r = b.make_rotary(64)
    assert b.lib().codecomp_rotate(D, D, C.byref(r), 0, 4, 128, 0, 0, D, 0, 0, None) == 0
    # empty tensors have no address
    assert b.lib().codecomp_rotate(None, None, C.byref(r), 0, 4, 128, 0, 0, None, 0, 0, None) == 0
    assert attend(x, p, q=None, out=None) == 0 and append(x, p, q=None, k=None, v=None, pos=None, q_out=None) == 0
    assert attend(x, p, layer=7) == -12 and append(x, p, layer=7) == -12
    assert b.lib().codecomp_attend_workspace_bytes(C.byref(x), C.byref(p)) == 0


def test_sizes_beyond_a_launch_are_refused():
    huge = pool(n_kv_heads=4096, n_layers=1)
    x = batch([0] + [1] * 60000, n_q_heads=4096)
    assert attend(x, huge) == -2 and b.lib().codecomp_attend_validate(C.byref(x), C.byref(huge)) == -2
    wide = pool(n_layers=1, n_kv_heads=65535, page_size=65536, head_dim=64, stride_tok=64, n_pages=1)
    assert b.lib().codecomp_pages_copy(C.byref(wide), D, 2, None) == -2
    assert b.lib().codecomp_pages_copy(C.byref(pool()), D, 2**30, None) == -2
    assert attend(batch(), pool(page_size=65536, stride_tok=1 << 16)) == -2          # 8 GB in a page
    # many requests of long tables: chunks grow until a launch holds them
    x = batch(list(range(60001)), table_width=1 << 16, max_kv_len=1 << 20)
    assert 0 < b.lib().codecomp_attend_workspace_bytes(C.byref(x), C.byref(pool()))


def test_workspace_follows_lengths_and_tokens():
    size = lambda cu, **kw: b.lib().codecomp_attend_workspace_bytes(C.byref(batch(cu, table_width=1 << 14, **kw)), C.byref(pool()))  # noqa: E731
    assert size((0, 1), max_kv_len=100) == 0                                          # one chunk: written at once
    assert 0 < size((0, 1), max_kv_len=5000) < size((0, 1), max_kv_len=100000)
    assert size((0, 400), max_kv_len=500) == 0                                        # blocks of rows that nobody shares
    assert size((0, 400), max_kv_len=5000) > 0


def test_append_refuses():
    x, p = batch(), pool()
    assert append(x, p, k=None) == -1 and append(x, p, v=None) == -1 and append(x, p, q=None) == -1 and append(x, p, q_out=None) == -1
    assert append(x, p, pos=None) == -1 and append(None, p) == -1 and append(x, None) == -1
    assert append(x, p, layer=2) == -12
    assert append(x, p, k=D + 4) == -2 and append(x, p, q=D + 4) == -2
    for change in [dict(dim=136), dict(dim=24), dict(dim=-16), dict(interleaved=2), dict(inverse=-1), dict(magnitude=float("inf"))]:
        r = b.make_rotary(64)
        for k, v in change.items():
            setattr(r, k, v)
        assert append(x, p, rot=r) == -11
    r = b.make_rotary(64)
    r.freq[31] = float("nan")
    assert append(x, p, rot=r) == -11
    assert append(x, pool(head_dim=64), rot=b.make_rotary(128)) == -11


def test_rotate_refuses():
    r = b.make_rotary(64)
    call = lambda x=D, pos=D, rot=r, T=3, H=4, d=128, s=(0, 0), out=D, o=(0, 0): b.lib().codecomp_rotate(  # noqa: E731
        x, pos, C.byref(rot) if rot else None, T, H, d, *s, out, *o, None)
    assert call(x=None) == -1 and call(pos=None) == -1 and call(rot=None) == -1 and call(out=None) == -1
    assert call(d=96) == -7 and call(H=0) == -6 and call(T=-1) == -2 and call(T=2**30) == -2
    assert call(x=D + 2) == -2 and call(out=D + 4) == -2 and call(s=(0, 64)) == -2 and call(s=(4, 0)) == -2 and call(o=(-8, 0)) == -2
    assert call(d=64, rot=b.make_rotary(128)) == -11


def rows_params(**over):
    cu, cb = np.array([0, 100, 130], np.int32), np.array([0, 10, 16], np.int32)
    kw = dict(n_layers=2, n_q_heads=28, n_kv_heads=4, head_dim=128, window=1, pool_kernel=1, prior_weight=0.0, cu_seqlens_host=cu, cu_budgets_host=cb,
              cu_seqlens_dev=D, cu_budgets_dev=D)
    kw.update(over)
    return b.make_params(**kw)


def test_moves_of_rows_refuse():
    l, q, p = b.lib(), rows_params(), pool()
    store = lambda k=D, v=D, idx=None, q=q, p=p, t=D, w=4: l.codecomp_pages_store(k, v, idx, C.byref(q), C.byref(p), t, w, None, None)  # noqa: E731
    load = lambda p=p, t=D, w=4, idx=None, q=q, k=D, v=D: l.codecomp_pages_load(C.byref(p), t, w, None, idx, C.byref(q), k, v, None)  # noqa: E731
    compact = lambda p=p, t=D, w=4, idx=D, q=q, to=p, tt=D, tw=4: l.codecomp_pages_compact(C.byref(p), t, w, None, idx, C.byref(q), C.byref(to), tt, tw, None, None)  # noqa: E731
    for f in (store, load):
        assert f(k=None) == -1 and f(v=None) == -1 and f(t=None) == -1 and f(w=0) == -12 and f(k=D + 8) == -2
    assert compact(idx=None) == -1 and compact(t=None) == -1 and compact(tt=None) == -1 and compact(w=0) == -12 and compact(tw=-3) == -12
    for f in (store, load, compact):
        assert f(p=pool(n_layers=3)) == -2 and f(p=pool(n_kv_heads=2)) == -2 and f(p=pool(head_dim=64)) == -7 and f(p=pool(kv_dtype=1)) == -11
        assert f(p=pool(page_size=20)) == -12
        assert f(q=rows_params(window=0)) == -3 and f(q=rows_params(cu_seqlens_host=np.array([0, 100, 90], np.int32))) == -8
    assert compact(to=pool(page_size=20)) == -12 and compact(to=pool(k_scale=0.5)) == -11 and compact(to=pool(n_layers=1)) == -2
    assert l.codecomp_pages_copy(C.byref(p), None, 2, None) == -1 and l.codecomp_pages_copy(C.byref(p), D, -1, None) == -2


def test_the_new_status_has_a_description():
    assert "page" in b.status_string(-12) and b.STATUS[-12] == "CODECOMP_EINVAL_PAGES"


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    k = torch.zeros(1, 3, 2, 16, 64, dtype=torch.bfloat16)
    p = b.make_pages(k, k.clone())
    with pytest.raises(ValueError):
        b.make_pages(k, k[:, :2])
    with pytest.raises(ValueError):
        b.make_pages(k.float(), k.float())
    with pytest.raises(ValueError):
        b.make_pages(k[..., ::2], k[..., ::2])
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    cu = np.array([0, 2, 3], np.int32)
    x = b.make_batch(n_q_heads=4, cu_q_host=cu, cu_q=i32(3), kv_lens=i32(2), table=i32(2, 3), max_kv_len=48)
    for bad in (dict(cu_q=i32(4)), dict(kv_lens=i32(3)), dict(table=i32(3, 3)), dict(table=i32(2, 6)[:, ::2]), dict(kv_lens=torch.zeros(2))):
        with pytest.raises(ValueError):
            b.make_batch(**{**dict(n_q_heads=4, cu_q_host=cu, cu_q=i32(3), kv_lens=i32(2), table=i32(2, 3), max_kv_len=48), **bad})
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    for bad in (q[:2], q.float(), torch.zeros(3, 8, 64, dtype=torch.bfloat16)[:, ::2]):
        with pytest.raises(ValueError):
            b.codecomp_attend(bad, x, p, 0, q, None)
        with pytest.raises(ValueError):
            b.codecomp_attend(q, x, p, 0, bad, None)
    if not torch.cuda.is_available():
        return
    with pytest.raises(ValueError):           # everything there, but on the CPU
        b.codecomp_attend(q, x, p, 0, q.clone(), None)


def test_products_of_sizes_that_wrap_around_are_refused():
    """Each of these passes every bound by itself; multiplied in 64 bits they would come out small or negative."""
    r, most = b.make_rotary(64), 2**31 - 1
    rotate = lambda T, H: b.lib().codecomp_rotate(D, D, C.byref(r), T, H, 128, 0, 0, D, 0, 0, None)  # noqa: E731
    assert rotate(most, most) == -6 and rotate(2**30, 2**30) == -6 and rotate(1, 65536) == -6 and rotate(most, 65535) == -2
    for cu, heads, code in [((0, 2**30), 2**30, -6), ((0, 1), 1 << 16, -6), ((0, most), 65532, -2)]:
        x, p = batch(cu, n_q_heads=heads), pool()
        assert attend(x, p) == code and append(x, p) == code
    for stride in (2**62, 2**47, 2**31):
        assert attend(batch(), pool(stride_tok=stride, page_size=65536)) == -2


def test_binding_refuses_broadcast_and_scattered_tensors():
    """A stride of zero is not the dense layout that a zero stands for in the C interface."""
    import torch
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    r, pos = b.make_rotary(64), torch.zeros(5, dtype=torch.int32)
    for bad in (bf(1, 4, 64).expand(5, 4, 64), bf(5, 1, 64).expand(5, 4, 64)):
        with pytest.raises(ValueError, match="broadcast"):
            b.codecomp_rotate(bad, pos, r, bf(5, 4, 64))
        with pytest.raises(ValueError, match="broadcast"):
            b.codecomp_rotate(bf(5, 4, 64), pos, r, bad)
    for bad in (bf(1, 3, 2, 16, 64).expand(2, 3, 2, 16, 64), bf(2, 3, 1, 16, 64).expand(2, 3, 2, 16, 64), bf(2, 3, 2, 1, 64).expand(2, 3, 2, 16, 64)):
        with pytest.raises(ValueError, match="broadcast"):
            b.make_pages(bad, bad)
    one = b.make_pages(*[bf(1, 3, 1, 16, 64).as_strided((1, 3, 1, 16, 64), (3, 1024, 5, 64, 1))] * 2)          # strides of single places say nothing
    assert (one.stride_layer, one.stride_page, one.stride_head, one.stride_tok) == (0, 1024, 0, 64)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    good = dict(n_q_heads=4, cu_q_host=np.array([0, 2, 3], np.int32), cu_q=i32(3), kv_lens=i32(2), table=i32(2, 3), max_kv_len=48)
    for name in ("cu_q", "kv_lens", "table"):                                                                     # not all on one device
        with pytest.raises(ValueError, match="device"):
            b.make_batch(**{**good, name: good[name].to("meta")})
    with pytest.raises(TypeError):
        b.make_batch(**good, q_strides_tok=8)
    x, p = b.make_batch(**good), b.make_pages(bf(1, 3, 2, 16, 64), bf(1, 3, 2, 16, 64))
    with pytest.raises(ValueError, match="workspace"):
        b.codecomp_attend(bf(3, 4, 64), x, p, 0, bf(3, 4, 64), torch.zeros(1, dtype=torch.uint8).expand(1 << 20))


@pytest.mark.parametrize("cu, over, kv", [((0, 1), dict(max_kv_len=5000), {}), ((0, 1, 2), dict(max_kv_len=1 << 18), {}), ((0, 400), dict(max_kv_len=5000), {}),
                                           ((0, 9), dict(max_kv_len=1 << 18), {}), ((0, 9, 400), dict(max_kv_len=1 << 18), dict(kv_dtype=1))])
def test_attend_refuses_workspaces_that_do_not_hold_its_parts(cu, over, kv):
    """One token over chunks of keys, tokens over equal parts, a prompt, a short chunk, both kernels."""
    x, p = batch(cu, table_width=1 << 14, **over), pool(**kv)
    need = b.lib().codecomp_attend_workspace_bytes(C.byref(x), C.byref(p))
    assert need > 0
    for bad in (dict(ws=None), dict(ws=D + 16), dict(ws=D + 128), dict(size=need - 1), dict(size=0)):
        assert attend(x, p, **bad) == -9, bad


def test_a_batch_keeps_its_own_token_offsets():
    """The array that sizes the launches may be used again for the next batch: the tensors of the first are still checked against what it was made with."""
    import torch
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    cu = np.array([0, 2, 3], np.int32)
    x = b.make_batch(n_q_heads=4, cu_q_host=cu, cu_q=i32(3), kv_lens=i32(2), table=i32(2, 3), max_kv_len=48)
    cu[1:] = 1000, 2000
    assert (C.c_int32 * 3).from_address(x.cu_q_host)[:] == [0, 2, 3] and x._tokens == 3


def test_tensors_of_no_tokens_have_no_strides_to_be_checked():
    import torch
    for t in (torch.from_numpy(np.empty((0, 6, 64), np.float32)).bfloat16()[:, :4], torch.empty(0, 4, 64, dtype=torch.bfloat16).as_strided((0, 4, 64), (0, 0, 0))):
        b._vectors(t, "q", (0, 4, 64), 6 * 64, 0)
    with pytest.raises(ValueError):
        b._vectors(torch.empty(1, 4, 64, dtype=torch.bfloat16).as_strided((1, 4, 64), (0, 0, 0)), "q", (1, 4, 64), 0, 0)
