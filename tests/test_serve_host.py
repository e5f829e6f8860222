"""Operators for shared and evicted caches, what needs no GPU: symbols and structures of the header, and every refusal with its code (checked on the host
before anything is launched)."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from paper_2604_10235_amd import binding as b
from tests.test_cache_host import BATCHES, D, POOLS, ROOT, batch, pool

HEADER = os.path.join(ROOT, "include", "codecomp_serve.h")


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(b.LIB_PATH):
        from paper_2604_10235_amd import build
        build.build_library(verbose=False)


def test_header_is_c99_and_every_declared_function_is_exported():
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-fsyntax-only", "-x", "c", HEADER], check=True)
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(codecomp_[a-z_]+)\s*\(", text)))
    assert names == ["codecomp_attend_mass", "codecomp_attend_mass_validate", "codecomp_attend_mass_workspace_bytes", "codecomp_attend_shared",
                     "codecomp_attend_shared_validate", "codecomp_attend_shared_workspace_bytes", "codecomp_evict"]
    for n in names:
        assert hasattr(b.lib(), n), n


def test_structures_are_laid_out_as_in_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    fields = {"codecomp_groups": b.codecomp_groups, "codecomp_mass": b.codecomp_mass, "codecomp_eviction": b.codecomp_eviction}
    lines = [f'printf("%zu\\n", sizeof({n})); ' + " ".join(f'printf("%zu\\n", offsetof({n}, {f[0]}));' for f in s._fields_) for n, s in fields.items()]
    src.write_text('#include <stdio.h>\n#include "codecomp_serve.h"\nint main(void) {' + "\n".join(lines) + "return 0; }\n")
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [x for s in fields.values() for x in [C.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]]


def groups(cu=(0, 2), **over):
    g = b.codecomp_groups()
    host = np.array(cu, np.int32)
    g.n_groups, g.max_prefix_len, g.max_own_len = len(cu) - 1, 48, 16
    g.cu_groups_host, g.cu_groups_dev, g.prefix_lens_dev = host.ctypes.data, D, D
    g._keep = host
    for k, v in over.items():
        setattr(g, k, v)
    return g


def mass(**over):
    m = b.codecomp_mass()
    m.sums, m.n_layers, m.n_seqs, m.n_kv_heads, m.width = D, 2, 2, 4, 64
    for k, v in over.items():
        setattr(m, k, v)
    return m


def eviction(**over):
    e = b.codecomp_eviction()
    e.n_seqs, e.table_width, e.max_kv_len, e.max_budget, e.recent = 2, 4, 64, 32, 8
    e.kv_lens_dev, e.table_dev, e.budgets_dev = D, D, D
    for k, v in over.items():
        setattr(e, k, v)
    return e


def ref(x):
    return C.byref(x) if x is not None else None


def shared(x, g, p, layer=0, q=D, out=D, lse=None, ws=D, size=1 << 40):
    return b.lib().codecomp_attend_shared(q, ref(x), ref(g), ref(p), layer, out, lse, ws, size, None)


def weigh(x, p, m, layer=0, q=D, lse=D, first=None, decay=1.0, ws=D, size=1 << 40):
    return b.lib().codecomp_attend_mass(q, lse, ref(x), ref(p), layer, first, decay, ref(m), ws, size, None)


def evict(m, e, p, kept=D, lens=D + 64, to=None):
    return b.lib().codecomp_evict(ref(m), ref(e), ref(p), kept, lens, ref(to), None)


@pytest.mark.parametrize("bad, code", POOLS, ids=str)
def test_a_bad_pool_is_refused_by_every_call(bad, code):
    x, p = batch(), pool(**bad)
    assert shared(x, groups(), p) == code and weigh(x, p, mass()) == code and evict(mass(), eviction(), p) == code
    assert b.lib().codecomp_attend_shared_workspace_bytes(ref(x), ref(groups()), ref(p)) == 0
    assert b.lib().codecomp_attend_mass_workspace_bytes(ref(x), ref(p), ref(mass())) == 0


@pytest.mark.parametrize("bad, code", BATCHES, ids=str)
def test_a_bad_batch_is_refused(bad, code):
    x, p = batch(**bad), pool()
    assert shared(x, groups(), p) == code and weigh(x, p, mass()) == code
    assert b.lib().codecomp_attend_shared_validate(ref(x), ref(groups()), ref(p)) == code
    assert b.lib().codecomp_attend_mass_validate(ref(x), ref(p), ref(mass())) == code


@pytest.mark.parametrize("bad, code", [(dict(cu_groups_host=None), -1), (dict(cu_groups_dev=None), -1), (dict(prefix_lens_dev=None), -1), (dict(n_groups=0), -2), (dict(n_groups=65536), -2),
                                       (dict(max_prefix_len=65), -12), (dict(max_prefix_len=-1), -12), (dict(max_own_len=65), -12), (dict(max_own_len=-1), -12)], ids=str)
def test_bad_groups_are_refused(bad, code):
    assert shared(batch(), groups(**bad), pool()) == code
    assert b.lib().codecomp_attend_shared_validate(ref(batch()), ref(groups(**bad)), ref(pool())) == code


def test_group_offsets_are_checked():
    for cu in [(1, 2), (0, 1), (0, 3), (0, 2, 1), (0, -1, 2), (0, 2, 1, 2)]:
        assert shared(batch(), groups(cu), pool()) == -8, cu
    assert shared(batch(), None, pool()) == -1 and shared(None, groups(), pool()) == -1 and shared(batch(), groups(), None) == -1


def test_shared_refuses_pointers_layers_and_workspaces():
    x, g, p = batch(), groups(), pool()
    assert shared(x, g, p, q=None) == -1 and shared(x, g, p, out=None) == -1
    assert shared(x, g, p, layer=2) == -12 and shared(x, g, p, layer=-1) == -12
    assert shared(x, g, p, q=D + 2) == -2 and shared(x, g, p, out=D + 8) == -2 and shared(x, g, p, lse=D + 2) == -2
    assert b.lib().codecomp_attend_shared_workspace_bytes(ref(x), ref(g), ref(p)) == 0             # short: no parts
    x, g = batch(table_width=64, max_kv_len=1024), groups(max_prefix_len=700)
    need = b.lib().codecomp_attend_shared_workspace_bytes(ref(x), ref(g), ref(p))
    assert need >= 3 * 28 * 130 * 4                                  # a part at least of every row
    for bad in (dict(ws=None), dict(ws=D + 16), dict(ws=D + 128), dict(size=need - 1), dict(size=0)):
        assert shared(x, g, p, **bad) == -9, bad


@pytest.mark.parametrize("bad, code", [(dict(sums=None), -1), (dict(sums=D + 2), -2), (dict(n_layers=0), -2), (dict(n_layers=3), -2), (dict(n_seqs=0), -2), (dict(n_seqs=3), -2),
                                       (dict(n_kv_heads=0), -2), (dict(n_kv_heads=2), -2), (dict(width=63), -2), (dict(width=-1), -2), (dict(stride_layer=-1), -2),
                                       (dict(stride_seq=-4), -2), (dict(stride_head=-64), -2), (dict(n_layers=2**31 - 1), -2)], ids=str)
def test_bad_sums_are_refused(bad, code):
    m = mass(**bad)
    assert weigh(batch(), pool(), m) == code and evict(m, eviction(), pool()) == code and evict(mass(), eviction(), pool(), to=m) == code
    assert b.lib().codecomp_attend_mass_validate(ref(batch()), ref(pool()), ref(m)) == code


def test_mass_refuses_pointers_layers_decay_and_workspaces():
    x, p, m = batch(), pool(), mass()
    assert weigh(x, p, None) == -1 and weigh(x, None, m) == -1 and weigh(None, p, m) == -1 and weigh(x, p, m, q=None) == -1 and weigh(x, p, m, lse=None) == -1
    assert weigh(x, p, m, layer=2) == -12 and weigh(x, p, m, layer=-1) == -12
    for decay in (-0.1, 1.0001, float("nan"), float("inf")):
        assert weigh(x, p, m, decay=decay) == -10
    assert weigh(x, p, m, q=D + 8) == -2 and weigh(x, p, m, lse=D + 1) == -2 and weigh(x, p, m, first=D + 2) == -2
    x = batch((0, 4000), table_width=1 << 10, max_kv_len=4000)
    m = mass(n_seqs=1, width=4000)
    need = b.lib().codecomp_attend_mass_workspace_bytes(ref(x), ref(p), ref(m))
    assert need > 0
    for bad in (dict(ws=None), dict(ws=D + 128), dict(size=need - 1)):
        assert weigh(x, p, m, **bad) == -9, bad


def test_evict_refuses():
    m, e, p = mass(), eviction(), pool()
    assert evict(None, e, p) == -1 and evict(m, None, p) == -1 and evict(m, e, None) == -1 and evict(m, e, p, kept=None) == -1 and evict(m, e, p, lens=None) == -1
    for name in ("kv_lens_dev", "table_dev", "budgets_dev"):
        assert evict(m, eviction(**{name: None}), p) == -1
    for bad, code in [(dict(n_seqs=0), -2), (dict(n_seqs=3), -2), (dict(n_seqs=65536), -2), (dict(table_width=0), -12), (dict(max_kv_len=65), -12), (dict(max_kv_len=-1), -12),
                      (dict(max_budget=0), -4), (dict(recent=-1), -4), (dict(recent=33), -4), (dict(max_budget=2**31 - 1), -4)]:
        assert evict(m, eviction(**bad), p) == code, bad
    assert evict(mass(width=2**31 - 1), eviction(table_width=2**31 - 1, max_kv_len=2**31 - 1), p) == -12
    assert evict(m, e, p, kept=D + 2) == -2 and evict(m, e, p, lens=D + 1) == -2
    assert evict(m, e, p, lens=D) == -2                              # the lengths themselves, the budgets, the numbers of protected rows
    assert evict(m, eviction(budgets_dev=D + 128), p, lens=D + 128) == -2 and evict(m, eviction(first_dev=D + 192), p, lens=D + 192) == -2
    assert evict(m, e, p, to=mass(width=65)) == -2
    assert evict(m, e, p, to=mass(stride_head=128)) == -2            # the same place with other strides


def test_calls_without_tokens_do_nothing():
    x, g, p = batch((0, 0, 0)), groups(), pool()
    assert shared(x, g, p, q=None, out=None, ws=None, size=0) == 0 and weigh(x, p, mass(), q=None, lse=None, ws=None, size=0) == 0
    assert shared(x, g, p, layer=7) == -12 and weigh(x, p, mass(), layer=7) == -12
    assert b.lib().codecomp_attend_shared_workspace_bytes(ref(x), ref(g), ref(p)) == 0


def test_sizes_beyond_a_launch_are_refused():
    huge = pool(n_kv_heads=4096, n_layers=1)
    x = batch([0] + [1] * 60000, n_q_heads=4096)
    assert shared(x, groups((0, 60000)), huge) == -2
    for n in (x, batch([0] * 60000 + [1], n_q_heads=4096)):                               # shares of all work: as many workgroups whatever there is
        assert b.lib().codecomp_attend_mass_validate(ref(n), ref(huge), ref(mass(n_layers=1, n_seqs=60000, n_kv_heads=4096))) == 0
    assert evict(mass(n_layers=15, n_seqs=65535, n_kv_heads=4096), eviction(n_seqs=65535), pool(n_kv_heads=4096, n_layers=15)) == -2
    # one prompt of very many tokens is none too many: what is behind the shared rows is joined where it is attended to
    assert b.lib().codecomp_attend_shared_validate(ref(batch([0, 1 << 20], n_q_heads=64)), ref(groups((0, 1))), ref(pool(head_dim=128))) == 0
    # many groups without tokens beside one with some; many requests, each a group of its own, under long bounds
    for tokens, cu in ((1000, [0] * 60000 + [1]), (1, [0] * 60000 + [1])):
        x = batch([0, tokens], n_q_heads=64, table_width=1 << 16, max_kv_len=1 << 20)
        for bound in (600, 1 << 20):
            assert b.lib().codecomp_attend_shared_validate(ref(x), ref(groups(cu, max_prefix_len=bound, max_own_len=bound)), ref(pool())) == 0
    x = batch(list(range(60001)), table_width=1 << 16, max_kv_len=1 << 20)
    assert b.lib().codecomp_attend_shared_validate(ref(x), ref(groups(range(60001), max_prefix_len=1 << 20, max_own_len=1 << 20)), ref(pool())) == 0
    # many requests of long tables: chunks grow until a launch holds them
    x = batch(list(range(60001)), table_width=1 << 16, max_kv_len=1 << 20)
    assert b.lib().codecomp_attend_shared_workspace_bytes(ref(x), ref(groups((0, 60000), max_prefix_len=1 << 20, max_own_len=1 << 20)), ref(pool())) > 0
    assert b.lib().codecomp_attend_mass_validate(ref(x), ref(pool()), ref(mass(n_seqs=60000, width=1 << 20))) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    p = b.make_pages(bf(1, 3, 2, 16, 64), bf(1, 3, 2, 16, 64))
    cu = np.array([0, 2, 3], np.int32)
    x = b.make_batch(n_q_heads=4, cu_q_host=cu, cu_q=i32(3), kv_lens=i32(2), table=i32(2, 3), max_kv_len=48)
    good = dict(cu_groups_host=np.array([0, 2]), cu_groups=i32(2), prefix_lens=i32(1), max_prefix_len=20, max_own_len=20)
    g = b.make_groups(**good)
    for bad in (dict(cu_groups=i32(3)), dict(prefix_lens=i32(2)), dict(prefix_lens=torch.zeros(1)), dict(cu_groups=i32(4)[::2]), dict(prefix_lens=i32(1).to("meta"))):
        with pytest.raises(ValueError):
            b.make_groups(**{**good, **bad})
    host = good["cu_groups_host"]
    host[:] = 7
    assert (C.c_int32 * 2).from_address(g.cu_groups_host)[:] == [0, 2]                 # a copy
    sums = torch.zeros(1, 2, 2, 48)
    m = b.make_mass(sums)
    assert (m.n_layers, m.n_seqs, m.n_kv_heads, m.width, m.stride_head) == (1, 2, 2, 48, 48)
    for bad in (sums.double(), sums[0], torch.zeros(1, 2, 2, 96)[..., ::2], torch.zeros(1, 1, 2, 48).expand(1, 2, 2, 48), torch.zeros(1, 2, 1, 48).expand(1, 2, 2, 48),
                torch.zeros(200).as_strided((1, 2, 2, 48), (0, 24, 48, 1)), torch.zeros(200).as_strided((1, 2, 2, 48), (0, 60, 40, 1))):
        with pytest.raises(ValueError):
            b.make_mass(bad)
    b.make_mass(torch.zeros(2, 2, 1, 96)[..., 3:50].permute(2, 1, 0, 3))                 # another order, and room between
    q, lse = bf(3, 4, 64), torch.zeros(3, 4)
    for bad in (q[:2], q.float(), bf(3, 8, 64)[:, ::2]):
        with pytest.raises(ValueError):
            b.codecomp_attend_shared(bad, x, g, p, 0, q, None)
        with pytest.raises(ValueError):
            b.codecomp_attend_shared(q, x, g, p, 0, bad, None)
        with pytest.raises(ValueError):
            b.codecomp_attend_mass(bad, lse, x, p, 0, m, None)
    for bad in (lse[:2], lse.double(), torch.zeros(4, 3).T):
        with pytest.raises(ValueError):
            b.codecomp_attend_mass(q, bad, x, p, 0, m, None)
        with pytest.raises(ValueError):
            b.codecomp_attend_shared(q, x, g, p, 0, q.clone(), None, lse=bad)
    with pytest.raises(ValueError):
        b.codecomp_attend_mass(q, lse, x, p, 0, m, None, first=i32(3))
    with pytest.raises(ValueError, match="workspace"):
        b.codecomp_attend_shared(q, x, g, p, 0, q.clone(), torch.zeros(1, dtype=torch.uint8).expand(1 << 20))
    ev = dict(kv_lens=i32(2), table=i32(2, 3), budgets=i32(2), max_kv_len=48, max_budget=8, recent=2)
    e = b.make_eviction(**ev)
    for bad in (dict(budgets=i32(3)), dict(table=i32(3, 3)), dict(first=i32(1)), dict(kv_lens=torch.zeros(2)), dict(budgets=i32(2).to("meta"))):
        with pytest.raises(ValueError):
            b.make_eviction(**{**ev, **bad})
    for kept, lens in ((i32(1, 2, 2, 9), i32(2)), (i32(1, 2, 2, 8), i32(3)), (torch.zeros(1, 2, 2, 8), i32(2)), (i32(1, 2, 2, 16)[..., ::2], i32(2))):
        with pytest.raises(ValueError):
            b.codecomp_evict(m, e, p, kept, lens)
    if not torch.cuda.is_available():
        return
    with pytest.raises(ValueError):           # everything there, but on the CPU
        b.codecomp_evict(m, e, p, i32(1, 2, 2, 8), i32(2))


@pytest.mark.parametrize("news, members, prefix, own", [
    ([1] * 64 + [1], [64, 1], 32768, 700), ([1] * 200 + [1], [200, 1], 32768, 700), ([512, 1], [1, 1], 32768, 700), ([4096] * 16 + [1], [16, 1], 8192, 4096),
    ([1] + [600] * 4, [1, 2, 2], 20000, 3000), ([1] * 1000 + [90], [4] * 250 + [1], 9000, 300)])
def test_workspace_of_both_kinds_of_groups_is_that_of_each(news, members, prefix, own):
    """A group of few rows has as many chunks of its shared rows as it needs, and one of many; neither number is every row's.  Own rows and places of tokens come on top."""
    cu, cg = np.concatenate([[0], np.cumsum(news)]), np.concatenate([[0], np.cumsum(members)])

    def need(these):
        """Bytes where only some of the groups have tokens."""
        host = np.concatenate([[0], np.cumsum([n if these[int(np.searchsorted(cg, r, side="right")) - 1] else 0 for r, n in enumerate(news)])])
        x = batch(host, table_width=(prefix + own) // 16 + 1, max_kv_len=prefix + own)
        return b.lib().codecomp_attend_shared_workspace_bytes(ref(x), ref(groups(cg, max_prefix_len=prefix, max_own_len=own)), ref(pool()))

    rows = [7 * int(cu[cg[g + 1]] - cu[cg[g]]) for g in range(len(members))]
    both, many, few = need([True] * len(members)), need([n > 64 for n in rows]), need([n <= 64 for n in rows])
    assert many > 0 and few > 0
    assert both <= 1.25 * (many + few) + 4 * int(cu[-1]) + (1 << 20), (both, many, few)
