"""Refusals of the budget operators, which come before anything is launched, and their arguments through the binding (no GPU)."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from paper_2404_09336_b200 import build, ssa

P = C.c_void_p(0x1000)      # never dereferenced: validation fails first
NUL = None


def good():
    d = ssa.AttnDesc()
    d.B, d.H, d.H_kv, d.D, d.max_ctx = 2, 8, 2, 128, 512
    d.kv_dtype, d.out_dtype, d.scale = ssa.BF16, ssa.BF16, 0.0
    d.q_stride_b, d.q_stride_h = 8 * 4 * 128, 4 * 128
    d.k_stride_b, d.k_stride_h, d.k_stride_t = 2 * 512 * 128, 512 * 128, 128
    d.v_stride_b, d.v_stride_h, d.v_stride_t = 2 * 512 * 128, 512 * 128, 128
    d.o_stride_b, d.o_stride_h = 8 * 4 * 128, 4 * 128
    w = ssa.Window()
    w.n_q, w.window, w.sinks, w.q_stride_t, w.o_stride_t = 4, 100, 4, 128, 128
    return d, w


def window(d, w, q=P, k=P, v=P, ctx=P, out=P, ws=P, ws_bytes=1 << 40):
    return ssa.lib.ssa_attn_window(d and C.byref(d), w and C.byref(w), q, k, v, ctx, out, NUL, ws, ws_bytes, NUL, NUL)


def mass(d, w, q=P, m_in=P, m_out=P, stride=512, ws=P, ws_bytes=1 << 40):
    return ssa.lib.ssa_attn_mass(d and C.byref(d), w and C.byref(w), q, P, P, P, P, NUL, m_in, m_out, stride, 1.0, ws, ws_bytes, NUL, NUL)


def paged(w, size=16, stride=32, pages=64, table=0x1000):
    pg = ssa.Paging()
    pg.page_table, pg.page_table_stride, pg.page_size, pg.n_pages = table, stride, size, pages
    w.paging = C.pointer(pg)
    return w


def test_attention_refuses_bad_arguments_before_launching():
    before = ssa.launch_count()
    for call in (window, mass):
        d, w = good()
        assert call(None, w) == ssa.ERR_NULL and call(d, None) == ssa.ERR_NULL and call(d, w, q=NUL) == ssa.ERR_NULL
        assert call(d, w, q=C.c_void_p(0x1008)) == ssa.ERR_ALIGN
        assert call(d, w, ws=NUL) == ssa.ERR_WORKSPACE and call(d, w, ws=C.c_void_p(0x1004)) == ssa.ERR_ALIGN
        for field, val, err in [("n_q", 0, ssa.ERR_SHAPE), ("n_q", -1, ssa.ERR_SHAPE), ("n_q", 1 << 30, ssa.ERR_SHAPE), ("window", -1, ssa.ERR_SHAPE),
                                ("sinks", -1, ssa.ERR_SHAPE), ("q_stride_t", 4, ssa.ERR_ALIGN), ("o_stride_t", 129, ssa.ERR_ALIGN),
                                ("q_stride_t", -128, ssa.ERR_SHAPE), ("o_stride_t", -128, ssa.ERR_SHAPE)]:
            d, w = good()
            setattr(w, field, val)
            assert call(d, w) == err, field
            assert ssa.attn_window_workspace_bytes(d, w) == 0 and ssa.attn_mass_workspace_bytes(d, w) == 0
        for field, val, err in [("D", 96, ssa.ERR_UNSUPPORTED), ("H_kv", 3, ssa.ERR_UNSUPPORTED), ("kv_dtype", ssa.F32, ssa.ERR_DTYPE),
                                ("out_dtype", ssa.F16, ssa.ERR_DTYPE), ("k_stride_t", 132, ssa.ERR_ALIGN), ("B", 0, ssa.ERR_SHAPE),
                                ("max_ctx", (1 << 30) + 1, ssa.ERR_SHAPE)]:
            d, w = good()
            setattr(d, field, val)
            assert call(d, w) == err, field
        for bad, err in [(dict(table=0), ssa.ERR_NULL), (dict(size=12), ssa.ERR_SHAPE), (dict(pages=0), ssa.ERR_SHAPE), (dict(stride=31), ssa.ERR_SHAPE),
                         (dict(pages=1 << 27), ssa.ERR_SHAPE)]:
            d, w = good()
            assert call(d, paged(w, **bad)) == err, bad
    d, w = good()
    for missing in ("k", "v", "ctx", "out"):
        assert window(d, w, **{missing: NUL}) == ssa.ERR_NULL
    need = ssa.attn_window_workspace_bytes(d, w)
    assert need > 0 and window(d, w, ws_bytes=need - 1) == ssa.ERR_WORKSPACE
    need = ssa.attn_mass_workspace_bytes(d, w)
    assert need >= 4 * 2 * 8 * 4 * 512 and mass(d, w, ws_bytes=need - 1) == ssa.ERR_WORKSPACE
    assert mass(d, w, m_out=NUL) == ssa.ERR_NULL and mass(d, w, stride=511) == ssa.ERR_SHAPE
    w.n_q = ssa.MASS_MAX_ROWS // 8 + 1
    assert mass(d, w) == ssa.ERR_SHAPE and ssa.attn_mass_workspace_bytes(d, w) == 0 and ssa.attn_window_workspace_bytes(d, w) > 0
    assert ssa.launch_count() == before


def test_selection_refuses_bad_arguments():
    f = ssa.lib.ssa_mass_to_index
    good = dict(mass=P, mass_stride=512, ctx=P, B=2, max_ctx=512, budget=64, sinks=4, recent=32, index=P, index_stride=64, counts=P)
    call = lambda **k: f(*{**good, **k}.values(), NUL, NUL)
    before = ssa.launch_count()
    for k in ("mass", "ctx", "index", "counts"):
        assert call(**{k: NUL}) == ssa.ERR_NULL
    for k in (dict(B=0), dict(B=65536), dict(max_ctx=0), dict(index_stride=0), dict(mass_stride=511),
              dict(max_ctx=(1 << 30) + 1, mass_stride=1 << 31)):
        assert call(**k) == ssa.ERR_SHAPE
    for k in (dict(budget=0), dict(budget=65), dict(sinks=-1), dict(recent=-1), dict(sinks=33), dict(sinks=2**31 - 1, recent=2**31 - 1)):
        assert call(**k) == ssa.ERR_CAPACITY
    assert ssa.launch_count() == before


def test_compaction_refuses_bad_arguments():
    f = ssa.lib.ssa_cache_compact
    before = ssa.launch_count()

    def call(d=None, pg=None, **k):
        a = {**dict(k=P, v=C.c_void_p(0x2000), ctx=P, index=P, index_stride=64, counts=P, max_selected=64, mass=P, mass_stride=512), **k}
        return f(C.byref(d or good()[0]), pg, *a.values(), NUL, NUL)

    assert f(None, None, P, P, P, P, 64, P, 64, P, 512, NUL, NUL) == ssa.ERR_NULL
    for k in ("k", "v", "ctx", "index", "counts"):
        assert call(**{k: NUL}) == ssa.ERR_NULL
    assert call(mass_stride=511) == ssa.ERR_SHAPE
    assert call(max_selected=65) == call(max_selected=0) == call(index_stride=0) == ssa.ERR_CAPACITY
    assert call(k=C.c_void_p(0x1008)) == call(v=C.c_void_p(0x1001)) == ssa.ERR_ALIGN
    assert call(v=P) == ssa.ERR_UNSUPPORTED                  # K and V in one place
    for field, val, err in (("D", 32, ssa.ERR_UNSUPPORTED), ("k_stride_t", 0, ssa.ERR_UNSUPPORTED), ("v_stride_h", 0, ssa.ERR_UNSUPPORTED),
                            ("k_stride_b", 0, ssa.ERR_UNSUPPORTED), ("max_ctx", (1 << 30) + 1, ssa.ERR_SHAPE)):
        d, w = good()
        setattr(d, field, val)
        assert call(d) == err, field
    d, w = good()
    assert call(pg=paged(w, size=3).paging) == ssa.ERR_SHAPE and call(pg=paged(w, table=0).paging) == ssa.ERR_NULL
    assert ssa.launch_count() == before


def test_errors_raise_through_the_binding():
    d, w = good()
    i = torch.zeros(2, 64, dtype=torch.int32)
    sums = torch.zeros(2, 512)
    for f, args in ((ssa.attn_window, (d, w, None, None, None, None, None)), (ssa.attn_mass, (d, w, None, None, None, None, None, None, None, sums)),
                    (ssa.mass_to_index, (torch.zeros(2, 9), i[:, 0], 65, 0, 0, i, i[:, 0])), (ssa.cache_compact, (d, None, None, None, i, None, 5))):
        with pytest.raises(ssa.SsaError, match=f.__name__):
            f(*args, stream=0)
        assert f(*args, stream=0, check=False) != ssa.OK
    with pytest.raises(ValueError, match="row stride"):
        ssa.attn_mass(d, w, None, None, None, None, None, None, sums, torch.zeros(2, 513), stream=0)
    for bad in (i, sums[:, :511], sums.double(), torch.zeros(512, 2).t()):
        with pytest.raises(ValueError, match="fp32"):
            ssa.attn_mass(d, w, None, None, None, None, None, None, None, bad, stream=0)
        with pytest.raises(ValueError, match="fp32"):
            ssa.cache_compact(d, None, None, None, i, None, 5, mass=bad, stream=0)
    with pytest.raises(ValueError, match="fp32"):
        ssa.mass_to_index(i, i[:, 0], 5, 0, 0, i, i[:, 0], stream=0)
    q = torch.zeros(2, 8, 4, 128)
    with pytest.raises(ValueError, match="int32"):
        ssa.make_window(q, q, q_lens=torch.zeros(2, dtype=torch.int64))
    with pytest.raises(TypeError, match="ssa_window"):
        ssa.attn_window(d, d, None, None, None, None, None, stream=0)
    with pytest.raises(TypeError):
        ssa.attn_mass(d, w, None, None, None, None, None, None, None, sums, "much", stream=0)


def test_struct_layout_matches_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "ssa.h"\nint main(void) {\n'
                   '  printf("%zu %zu %zu %zu %d\\n", sizeof(ssa_window), offsetof(ssa_window, q_stride_t), offsetof(ssa_window, q_lens),\n'
                   "         offsetof(ssa_window, paging), SSA_MASS_MAX_ROWS);\n  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run([cc, "-I", os.path.join(build.ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    W = ssa.Window
    assert got == [C.sizeof(W), W.q_stride_t.offset, W.q_lens.offset, W.paging.offset, ssa.MASS_MAX_ROWS]


# the calls' arguments, and the entry points' as they should arrive ("#x" elements, "/x" row stride, "*x" bytes of x)
CALLS = {
    "attn_window": ("desc win q k v ctx out lse ws status 7", "desc win q k v ctx out lse ws *ws status 7"),
    "attn_mass": ("desc win q k v ctx out lse min mout 0.75 ws status 7", "desc win q k v ctx out lse min mout /mout 0.75 ws *ws status 7"),
    "mass_to_index": ("mout ctx 36 20 3 5 idx cnt status 7", "mout /mout ctx #ctx 36 20 3 5 idx /idx cnt status 7"),
    "cache_compact": ("desc paging k v ctx idx cnt 11 mout status 7", "desc paging k v ctx idx /idx cnt 11 mout /mout status 7"),
}


@pytest.mark.parametrize("through", ["binding", "ctypes"])
@pytest.mark.parametrize("name", sorted(CALLS))
def test_arguments_arrive(name, through):
    import importlib.util
    import types
    got = []
    entry = getattr(ssa.lib, "ssa_" + name)
    kinds = [C.c_void_p if t.__name__.startswith("LP_") else t for t in entry.argtypes]
    callback = C.CFUNCTYPE(C.c_int32, *kinds)(lambda *a: got.append(list(a)) or 3)
    if through == "binding":
        spec = importlib.util.spec_from_file_location("apart._ssa_call", build.build_binding())
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.bind({"ssa_" + name: C.cast(callback, C.c_void_p).value})
        other = next(n for n in CALLS if n != name)
        with pytest.raises(RuntimeError, match="no library bound"):
            getattr(module, other)(*CALLS[other][0].split())
    else:
        module = ssa._CtypesCalls(types.SimpleNamespace(**{"ssa_" + name: callback}))
    for rows in (1, 3):
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
        d = {n: torch.zeros(4, 2) for n in ("q", "k", "v", "out", "lse", "min", "status")}
        d.update(ctx=i32(rows), cnt=i32(rows), ws=torch.zeros(321), idx=i32(rows, 2, 40)[:, 1, :36], mout=torch.zeros(rows, 50)[:, :36],
                 desc=ssa.AttnDesc(), win=ssa.Window(), paging=ssa.Paging())

        def want(word):
            if word[0] == "#":
                return d[word[1:]].numel()
            if word[0] == "/":
                return (80 if word == "/idx" else 50) if rows > 1 else 36
            if word[0] == "*":
                return 4 * 321
            if word in d:
                return C.addressof(d[word]) if isinstance(d[word], C.Structure) else d[word].data_ptr()
            return float(word) if "." in word else int(word)

        args, params = (w.split() for w in CALLS[name])
        for absent in (set(), {"lse", "ws", "status", "min", "paging"} | ({"mout"} if name == "cache_compact" else set())):
            given = [None if w in absent else d[w] if w in d else want(w) for w in args]
            assert getattr(module, name)(*given) == 3
            assert got.pop() == [(None if w in absent else 0 if w.strip("/*") in absent else want(w)) for w in params]
