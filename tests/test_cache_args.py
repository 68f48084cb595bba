"""Argument checks of the dm_cache_* entry points, made before any CUDA call:
they run without a GPU, on a library that is only loaded."""

import ctypes as C

import pytest


@pytest.fixture(scope="module")
def D():
    import __graft_entry__ as g
    g.build()
    from paper_2602_06502_gb300 import dualmap
    return dualmap


def cache(D, **kw):
    """A cache whose pointers are never followed."""
    base = dict(k=1 << 20, v=1 << 21, dtype=D.DM_BF16, layout=D.DM_PAGES_HEADS, layers=2, pages=64, page_tokens=16, kv_heads=4,
                head_dim=128, max_seqs=8, max_blocks=16, layer_stride=64 * 8192, page_stride=8192, tables=1 << 22, lengths=1 << 23,
                refs=1 << 24, status=1 << 25, work=1 << 26, work_bytes=1 << 20)
    base.update(kw)
    return D.dm_cache(**base)


BAD_SHAPES = [dict(dtype=2), dict(layout=2), dict(layers=0), dict(pages=0), dict(pages=(1 << 30) + 1), dict(page_tokens=24),
              dict(page_tokens=128), dict(page_tokens=0), dict(kv_heads=0), dict(kv_heads=65536), dict(head_dim=96), dict(head_dim=256),
              dict(max_seqs=0), dict(max_blocks=0), dict(max_blocks=1 << 27), dict(reserved0=1), dict(layer_stride=4),
              dict(page_stride=8191), dict(page_stride=8184), dict(page_stride=0)]
BAD_POINTERS = [dict(k=None), dict(v=None), dict(k=(1 << 20) + 8), dict(v=(1 << 20) + 2), dict(tables=None), dict(lengths=None),
                dict(refs=None), dict(refs=(1 << 24) + 4), dict(status=None), dict(work=None), dict(work=(1 << 26) + 8), dict(work_bytes=16)]


@pytest.mark.parametrize("bad", BAD_SHAPES, ids=str)
def test_shapes(D, bad):
    c = cache(D, **bad)
    assert D.dm_cache_work_bytes(c) == 0
    assert D.dm_plan_bytes(c, 4, 0, 4, 8) == 0
    assert D.dm_cache_free(c, 64, 1) == D.DM_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", BAD_POINTERS, ids=str)
def test_pointers(D, bad):
    c = cache(D, **bad)
    i = 1 << 27
    inv = D.DM_ERR_INVALID_ARG
    assert D.dm_cache_work_bytes(c) > 0
    assert D.dm_cache_extend(c, i, i, 1) == inv
    assert D.dm_cache_fork(c, i, i, i, 1) == inv
    assert D.dm_cache_free(c, i, 1) == inv
    assert D.dm_cache_compact(c) == inv
    assert D.dm_cache_append(c, D.dm_append_args()) == inv
    assert D.dm_cache_plan(c, D.dm_plan()) == inv
    assert D.dm_cache_attend(c, D.dm_plan(), D.dm_attend_args()) == inv


def test_null_structs(D):
    inv = D.DM_ERR_INVALID_ARG
    L, c = D.lib(), cache(D)
    assert L.dm_cache_work_bytes(None) == 0 and L.dm_plan_bytes(None, 1, 0, 1, 4) == 0
    assert L.dm_cache_last_error(None, None) == inv
    assert L.dm_cache_extend(None, None, None, 0, None) == inv
    assert L.dm_cache_append(C.byref(c), None, None) == inv
    assert L.dm_cache_plan(C.byref(c), None, None) == inv
    assert L.dm_cache_attend(C.byref(c), None, None, None) == inv


def test_page_calls(D):
    c, i, inv = cache(D), 1 << 27, D.DM_ERR_INVALID_ARG
    assert D.dm_cache_extend(c, None, None, 0) == D.DM_OK          # nothing to do
    assert D.dm_cache_fork(c, None, None, None, 0) == D.DM_OK
    assert D.dm_cache_free(c, None, 0) == D.DM_OK
    assert D.dm_cache_extend(c, i, None, 1) == inv and D.dm_cache_extend(c, None, i, 1) == inv
    assert D.dm_cache_extend(c, i, i, 9) == inv                    # more than the sequences there are
    assert D.dm_cache_fork(c, i, i, None, 1) == inv and D.dm_cache_fork(c, None, i, i, 1) == inv
    assert D.dm_cache_fork(c, i, None, i, 1) == inv and D.dm_cache_free(c, None, 1) == inv
    assert D.dm_cache_compact(c, None, i + 4) == inv


def test_append(D):
    c, a16, inv = cache(D), 1 << 27, D.DM_ERR_INVALID_ARG

    def args(**kw):
        base = dict(seqs=a16, offsets=a16, n=2, tokens=5, layer=0, q_heads=8, q=a16, k=a16, v=a16, q_out=a16, q_token=1024, q_head=128,
                    k_token=512, k_head=128, v_token=512, v_head=128, q_out_token=1024, q_out_head=128, q_weight=a16, k_weight=a16,
                    cos=a16, sin=a16, rope_rows=100, rope_dim=128, interleaved=0, eps=1e-6)
        base.update(kw)
        return D.dm_append_args(**base)

    for bad in (dict(layer=2), dict(q_heads=6), dict(eps=-1.0), dict(eps=float("nan")), dict(rope_dim=8), dict(rope_dim=144),
                dict(rope_rows=0), dict(cos=None), dict(sin=None), dict(n=9), dict(interleaved=2), dict(seqs=None), dict(offsets=None),
                dict(q=None), dict(k=None), dict(v=None), dict(q_out=None), dict(q=a16 + 8), dict(k=a16 + 2), dict(v=a16 + 8),
                dict(q_out=a16 + 4), dict(q_weight=a16 + 8), dict(cos=a16 + 4), dict(q_token=1025), dict(q_head=4), dict(k_token=2),
                dict(v_head=1), dict(q_out_token=7), dict(tokens=1 << 31)):
        assert D.dm_cache_append(c, args(**bad)) == inv, bad
    assert D.dm_cache_append(c, args(n=0)) == D.DM_OK and D.dm_cache_append(c, args(tokens=0)) == D.DM_OK


def test_plan_and_attend(D):
    c, a, inv = cache(D), 1 << 27, D.DM_ERR_INVALID_ARG
    size = D.dm_plan_bytes(c, 4, 2, 6, 8)
    assert size > 0
    assert D.dm_plan_bytes(c, 9, 0, 6, 8) == 0 and D.dm_plan_bytes(c, 4, 5, 6, 8) == 0      # sequences, groups
    assert D.dm_plan_bytes(c, 4, 2, 6, 6) == 0 and D.dm_plan_bytes(c, 4, 2, 6, 0) == 0      # heads
    assert D.dm_plan_bytes(c, 4, 2, 1 << 31, 8) == 0

    def plan(**kw):
        base = dict(seqs=a, offsets=a, n=4, tokens=6, q_heads=8, groups=2, group_offsets=a, group_prefix=a, work=a, work_bytes=size)
        base.update(kw)
        return D.dm_plan(**base)

    for bad in (dict(seqs=None), dict(offsets=None), dict(group_offsets=None), dict(group_prefix=None), dict(work=None),
                dict(work=a + 128), dict(work_bytes=size - 1), dict(n=9), dict(groups=5), dict(q_heads=7)):
        assert D.dm_cache_plan(c, plan(**bad)) == inv, bad
        assert D.dm_cache_attend(c, plan(**bad), D.dm_attend_args(0, 1.0, a, a, None, 1024, 128, 1024, 128)) == inv, bad
    assert D.dm_cache_plan(c, plan(n=0, groups=0)) == D.DM_OK

    def attend(**kw):
        base = dict(layer=0, scale=0.1, q=a, o=a, lse=None, q_token=1024, q_head=128, o_token=1024, o_head=128)
        base.update(kw)
        return D.dm_attend_args(**base)

    for bad in (dict(layer=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(q=None),
                dict(o=None), dict(q=a + 8), dict(o=a + 8), dict(lse=a + 2), dict(q_token=4), dict(o_head=2), dict(q_head=1),
                dict(o_token=12)):
        assert D.dm_cache_attend(c, plan(), attend(**bad)) == inv, bad
    assert D.dm_cache_attend(c, plan(n=0, groups=0), attend()) == D.DM_OK


def test_struct_layouts_match_header(D, tmp_path):
    import os
    import subprocess
    hdr = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dualmap.h")
    structs = {n: getattr(D, n) for n in ("dm_cache", "dm_append_args", "dm_plan", "dm_attend_args")}
    lines = ["#include <stdio.h>", "#include <stddef.h>", f'#include "{hdr}"', "int main(void) {"]
    for n, cls in structs.items():
        lines.append(f'printf("{n} %zu\\n", sizeof({n}));')
        lines += [f'printf("{n}.{f[0]} %zu\\n", offsetof({n}, {f[0]}));' for f in cls._fields_]
    for k in ("DM_BF16", "DM_F16", "DM_PAGES_HEADS", "DM_PAGES_TOKENS"):
        lines.append(f'printf("{k} %d\\n", (int){k});')
    lines.append("return 0; }")
    (tmp_path / "l.c").write_text("\n".join(lines))
    subprocess.run(["gcc", "-Wall", "-Werror", str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    out = dict(x.rsplit(" ", 1) for x in subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, check=True).stdout.split("\n") if x)
    for n, cls in structs.items():
        assert int(out[n]) == C.sizeof(cls), n
        for f in cls._fields_:
            assert int(out[f"{n}.{f[0]}"]) == getattr(cls, f[0]).offset, (n, f[0])
    for k in ("DM_BF16", "DM_F16", "DM_PAGES_HEADS", "DM_PAGES_TOKENS"):
        assert int(out[k]) == getattr(D, k)
