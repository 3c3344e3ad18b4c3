"""Refusals of the operators that fill a cache and read its blocks, which come before anything is launched, and their arguments through
the binding (no GPU)."""
import ctypes as C
import os
import shutil
import subprocess
import types

import pytest
import torch

from paper_2404_09336_b200 import build, ssa

P, P2 = C.c_void_p(0x1000), C.c_void_p(0x2000)      # never dereferenced: validation fails first
NUL, ODD = None, C.c_void_p(0x1008)


def desc(dtype=ssa.FP4_E2M1):
    d = ssa.AttnDesc()
    d.B, d.H, d.H_kv, d.D, d.max_ctx = 2, 8, 2, 128, 512
    d.kv_dtype, d.out_dtype, d.scale = dtype, ssa.F16 if dtype == ssa.F16 else ssa.BF16, 0.0
    d.q_stride_b, d.q_stride_h = 8 * 4 * 128, 4 * 128
    d.k_stride_b, d.k_stride_h, d.k_stride_t = 2 * 512 * 128, 512 * 128, 128
    d.v_stride_b, d.v_stride_h, d.v_stride_t = 2 * 512 * 128, 512 * 128, 128
    d.o_stride_b, d.o_stride_h = 8 * 4 * 128, 4 * 128
    return d


def good_window():
    w = ssa.Window()
    w.n_q, w.window, w.sinks, w.q_stride_t, w.o_stride_t = 4, 100, 4, 128, 128
    return w


def good_blocks():
    k = ssa.Blocks()
    k.n_q, k.block_size, k.budget, k.sinks, k.recent, k.q_stride_t, k.o_stride_t = 4, 64, 4, 1, 1, 128, 128
    k.bounds_stride_b, k.bounds_stride_h = 2 * 8 * 256, 8 * 256
    return k


def good_append():
    a = ssa.Append()
    a.n_q, a.rotary_dims, a.n_positions, a.k_factor, a.v_factor, a.q_stride_t, a.cos_sin = 4, 64, 512, 1.0, 1.0, 128, 0x3000
    for n in ("qo", "kn", "vn"):
        for d in "bht":
            setattr(a, f"{n}_stride_{d}", 128)
    return a


def pages(s, size=16, stride=32, pages=64, table=0x1000):
    pg = ssa.Paging()
    pg.page_table, pg.page_table_stride, pg.page_size, pg.n_pages = table, stride, size, pages
    s.paging = C.pointer(pg)
    return s


def ref(x):
    return x and C.byref(x)


def window(d, w, q=P, k=P, v=P, ks=P, vs=P, ctx=P, out=P, ws=P, ws_bytes=1 << 40):
    return ssa.lib.ssa_attn_window_fp4(ref(d), ref(w), q, k, v, ks, vs, ctx, out, NUL, ws, ws_bytes, NUL, NUL)


def bounds(d, k, key=P, ks=P, ctx=P, to=P):
    return ssa.lib.ssa_block_bounds(ref(d), ref(k), key, ks, ctx, to, NUL, NUL)


def select(d, k, q=P, b=P, ctx=P, index=P, counts=P):
    return ssa.lib.ssa_block_select(ref(d), ref(k), q, b, ctx, index, counts, NUL, NUL, NUL)


def attend(d, k, q=P, key=P, v=P, ks=P, vs=P, ctx=P, index=P, counts=P, out=P, ws=P, ws_bytes=1 << 40):
    return ssa.lib.ssa_attn_blocks(ref(d), ref(k), q, key, v, ks, vs, ctx, index, counts, out, NUL, ws, ws_bytes, NUL, NUL)


def append(d, a, kn=P, vn=P, ctx=P, k=P, v=P2, q=P, qo=P, ks=P, vs=P2):
    return ssa.lib.ssa_cache_append(ref(d), ref(a), kn, vn, ctx, k, v, q, qo, ks, vs, NUL, NUL)


CALLS = {"window": (window, good_window), "bounds": (bounds, good_blocks), "select": (select, good_blocks), "attend": (attend, good_blocks),
         "append": (append, good_append)}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_what_is_refused_by_every_call(name):
    call, good = CALLS[name]
    before = ssa.launch_count()
    assert call(None, good()) == ssa.ERR_NULL and call(desc(), None) == ssa.ERR_NULL
    params = {p: v for p, v in zip(call.__code__.co_varnames[2:], call.__defaults__) if p not in ("ws", "ws_bytes")}
    for p in params:
        assert call(desc(), good(), **{p: NUL}) == ssa.ERR_NULL, p
        if p not in ("ctx", "index", "counts"):
            assert call(desc(), good(), **{p: ODD}) == ssa.ERR_ALIGN, p
    for field, val, err in [("D", 96, ssa.ERR_UNSUPPORTED), ("H_kv", 3, ssa.ERR_UNSUPPORTED), ("kv_dtype", ssa.F32, ssa.ERR_DTYPE), ("kv_dtype", 5, ssa.ERR_DTYPE),
                            ("out_dtype", ssa.F16, ssa.ERR_DTYPE), ("k_stride_t", 64, ssa.ERR_ALIGN), ("v_stride_h", 512 * 128 + 32, ssa.ERR_ALIGN),
                            ("k_stride_b", -128, ssa.ERR_SHAPE), ("B", 0, ssa.ERR_SHAPE), ("max_ctx", (1 << 30) + 1, ssa.ERR_SHAPE), ("max_ctx", 0, ssa.ERR_SHAPE)]:
        d = desc()
        setattr(d, field, val)
        assert call(d, good()) == err, field
    for n_q in (0, -1) + (() if name == "bounds" else (1 << 30,)):
        s = good()
        s.n_q = n_q
        assert call(desc(), s) == ssa.ERR_SHAPE
    if name != "select":
        for bad, err in [(dict(table=0), ssa.ERR_NULL), (dict(size=12), ssa.ERR_SHAPE), (dict(pages=0), ssa.ERR_SHAPE), (dict(stride=31), ssa.ERR_SHAPE),
                         (dict(pages=1 << 27), ssa.ERR_SHAPE)]:
            assert call(desc(), pages(good(), **bad)) == err, bad
    if name in ("bounds", "attend", "append"):               # (scales belong to 4-bit caches only)
        d = desc(ssa.BF16)
        d.out_dtype = 77
        assert call(d, good(), ks=NUL) == ssa.ERR_DTYPE
    assert ssa.launch_count() == before


def test_windows_over_4_bit_values():
    d, w = desc(), good_window()
    need = ssa.attn_window_fp4_workspace_bytes(d, w)
    assert need > 0 and window(d, w, ws_bytes=need - 1) == ssa.ERR_WORKSPACE and window(d, w, ws=NUL) == ssa.ERR_WORKSPACE
    assert window(d, w, ws=ODD) == ssa.ERR_ALIGN
    for field, val, err in [("window", -1, ssa.ERR_SHAPE), ("sinks", -1, ssa.ERR_SHAPE), ("q_stride_t", 4, ssa.ERR_ALIGN), ("o_stride_t", -8, ssa.ERR_SHAPE)]:
        w = good_window()
        setattr(w, field, val)
        assert window(d, w) == err and ssa.attn_window_fp4_workspace_bytes(d, w) == 0
    for dtype in (ssa.BF16, ssa.F16, ssa.FP8_E4M3):
        assert window(desc(dtype), good_window()) == ssa.ERR_DTYPE and ssa.attn_window_fp4_workspace_bytes(desc(dtype), good_window()) == 0


def test_other_calls_refuse_a_4_bit_cache():
    d, w = desc(), good_window()
    assert ssa.lib.ssa_attn_window(C.byref(d), C.byref(w), P, P, P, P, P, NUL, P, 1 << 40, NUL, NUL) == ssa.ERR_DTYPE
    assert ssa.lib.ssa_decode_attn_dense(C.byref(d), P, P, P, P, P, NUL, P, 1 << 40, NUL, NUL) == ssa.ERR_DTYPE
    assert ssa.lib.ssa_cache_compact(C.byref(d), None, P, P2, P, P, 64, P, 64, P, 512, NUL, NUL) == ssa.ERR_DTYPE
    assert ssa.attn_window_workspace_bytes(d, w) == 0 == ssa.decode_workspace_bytes(d, 64)


@pytest.mark.parametrize("call", [bounds, select, attend])
def test_blocks(call):
    before = ssa.launch_count()
    for size in (0, 16, 48, 512, -64):
        k = good_blocks()
        k.block_size = size
        assert call(desc(), k) == ssa.ERR_UNSUPPORTED
    d, k = desc(), good_blocks()
    d.max_ctx = 64 * ssa.MAX_BLOCKS + 1
    assert call(d, k) == ssa.ERR_SHAPE
    for field, val, err in [("bounds_stride_b", -8, ssa.ERR_SHAPE), ("bounds_stride_h", 4, ssa.ERR_ALIGN)] if call is not attend else [
            ("q_stride_t", 4, ssa.ERR_ALIGN), ("o_stride_t", -8, ssa.ERR_SHAPE), ("budget", 0, ssa.ERR_CAPACITY), ("budget", -4, ssa.ERR_CAPACITY)]:
        k = good_blocks()
        setattr(k, field, val)
        assert call(desc(), k) == err, field
    if call is select:
        for change in (dict(budget=0), dict(sinks=-1), dict(recent=-1), dict(sinks=3, recent=2), dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1)):
            k = good_blocks()
            for field, val in change.items():
                setattr(k, field, val)
            assert select(desc(), k) == ssa.ERR_CAPACITY, change
        for stride, err in ((4, ssa.ERR_ALIGN), (-8, ssa.ERR_SHAPE)):
            k = good_blocks()
            k.q_stride_t = stride
            assert select(desc(), k) == err
    if call is attend:
        need = ssa.attn_blocks_workspace_bytes(desc(), good_blocks())
        assert need > 0 and attend(desc(), good_blocks(), ws_bytes=need - 1) == ssa.ERR_WORKSPACE and attend(desc(), good_blocks(), ws=NUL) == ssa.ERR_WORKSPACE
        assert attend(desc(), good_blocks(), ws=ODD) == ssa.ERR_ALIGN
        k.block_size = 31
        assert ssa.attn_blocks_workspace_bytes(desc(), k) == 0
        k.block_size, k.budget = 64, 1 << 25                 # (2^31 positions: tiles and positions of a list are counted in 32 bits)
        assert attend(desc(), k) == ssa.ERR_CAPACITY and ssa.attn_blocks_workspace_bytes(desc(), k) == 0
        k.budget -= 1
        assert ssa.attn_blocks_workspace_bytes(desc(), k) > 0
    assert ssa.launch_count() == before


def test_appending():
    before = ssa.launch_count()
    for field, val, err in [("rotary_dims", 16, ssa.ERR_SHAPE), ("rotary_dims", 160, ssa.ERR_SHAPE), ("rotary_dims", -32, ssa.ERR_SHAPE), ("cos_sin", None, ssa.ERR_NULL),
                            ("cos_sin", 0x3008, ssa.ERR_ALIGN), ("n_positions", 0, ssa.ERR_SHAPE), ("q_stride_t", 4, ssa.ERR_ALIGN), ("qo_stride_h", -8, ssa.ERR_SHAPE),
                            ("kn_stride_b", 9, ssa.ERR_ALIGN), ("vn_stride_t", -128, ssa.ERR_SHAPE)]:
        a = good_append()
        setattr(a, field, val)
        assert append(desc(), a) == err, field
    assert append(desc(), good_append(), v=P) == append(desc(), good_append(), vs=P) == ssa.ERR_UNSUPPORTED      # K and V in one place
    for field in ("k_stride_t", "v_stride_t", "k_stride_h", "v_stride_h", "k_stride_b", "v_stride_b"):
        d = desc()
        setattr(d, field, 0)
        assert append(d, good_append()) == ssa.ERR_UNSUPPORTED, field
    for field in ("qo_stride_b", "qo_stride_h", "qo_stride_t"):
        a = good_append()
        setattr(a, field, 0)
        assert append(desc(), a) == ssa.ERR_UNSUPPORTED, field
    for field in ("bounds_stride_b", "bounds_stride_h"):
        k = good_blocks()
        setattr(k, field, 0)
        assert bounds(desc(), k) == ssa.ERR_UNSUPPORTED, field
    assert ssa.launch_count() == before


def test_struct_layout_matches_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    fields = [(n, f) for n, c in (("ssa_blocks", ssa.Blocks), ("ssa_append", ssa.Append)) for f, _ in c._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ssa.h"\nint main(void) {\n  printf("%zu %zu %d %d", sizeof(ssa_blocks), sizeof(ssa_append), SSA_MAX_BLOCKS, SSA_FP4_E2M1);\n'
                   + "".join(f'  printf(" %zu", offsetof({n}, {f}));\n' for n, f in fields) + "  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run([cc, "-I", os.path.join(build.ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    of = {"ssa_blocks": ssa.Blocks, "ssa_append": ssa.Append}
    assert got == [C.sizeof(ssa.Blocks), C.sizeof(ssa.Append), ssa.MAX_BLOCKS, ssa.FP4_E2M1, *(getattr(of[n], f).offset for n, f in fields)]


# the calls' arguments, and the entry points' as they should arrive ("*x" bytes of x)
ARRIVE = {
    "attn_window_fp4": ("desc win q k v ks vs ctx out lse ws status 7", "desc win q k v ks vs ctx out lse ws *ws status 7"),
    "block_bounds": ("desc blocks k ks ctx out status 7",) * 2,
    "block_select": ("desc blocks q k ctx idx cnt lse status 7",) * 2,
    "attn_blocks": ("desc blocks q k v ks vs ctx idx cnt out lse ws status 7", "desc blocks q k v ks vs ctx idx cnt out lse ws *ws status 7"),
    "cache_append": ("desc append ks vs ctx k v q out idx cnt status 7",) * 2,
}


@pytest.mark.parametrize("through", ["binding", "ctypes"])
@pytest.mark.parametrize("name", sorted(ARRIVE))
def test_arguments_arrive(name, through):
    import importlib.util
    got = []
    entry = getattr(ssa.lib, "ssa_" + name)
    kinds = [C.c_void_p if t.__name__.startswith("LP_") else t for t in entry.argtypes]
    callback = C.CFUNCTYPE(C.c_int32, *kinds)(lambda *a: got.append(list(a)) or 3)
    if through == "binding":
        spec = importlib.util.spec_from_file_location("apart._ssa_call", build.build_binding())
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.bind({"ssa_" + name: C.cast(callback, C.c_void_p).value, "ssa_attn_desc": ssa.AttnDesc, "ssa_window": ssa.Window, "ssa_blocks": ssa.Blocks,
                     "ssa_append": ssa.Append})
        with pytest.raises(TypeError, match="wanted, not"):
            getattr(module, name)(*[ssa.AttnDesc()] * 2, *[None] * (len(ARRIVE[name][0].split()) - 3), 7)
    else:
        module = ssa._CtypesCalls(types.SimpleNamespace(**{"ssa_" + name: callback}))
    d = {n: torch.zeros(4, 2) for n in ("q", "k", "v", "ks", "vs", "ctx", "out", "lse", "idx", "cnt", "status")}
    d.update(ws=torch.zeros(321), desc=ssa.AttnDesc(), win=ssa.Window(), blocks=ssa.Blocks(), append=ssa.Append())

    def want(word):
        if word[0] == "*":
            return 4 * 321
        return int(word) if word not in d else C.addressof(d[word]) if isinstance(d[word], C.Structure) else d[word].data_ptr()

    args, params = (w.split() for w in ARRIVE[name])
    for absent in (set(), {"lse", "ws", "status", "ks", "vs"}):
        assert getattr(module, name)(*[None if w in absent else d.get(w, 7) for w in args]) == 3
        assert got.pop() == [(None if w in absent else 0 if w.strip("*") in absent else want(w)) for w in params]


def test_errors_raise_through_the_binding():
    d, x = desc(), torch.zeros(2, 8, 4, 128).bfloat16()
    b, i = torch.zeros(2, 2, 8, 2, 128).bfloat16(), torch.zeros(2, 2, 4, 4, dtype=torch.int32)
    k = good_blocks()
    for f, args in ((ssa.attn_window_fp4, (d, good_window(), *[None] * 7)), (ssa.block_bounds, (d, k, None, None, b)), (ssa.block_select, (d, k, None, b, None, i, i[..., 0].contiguous())),
                    (ssa.attn_blocks, (d, k, None, None, None, None, i, i[..., 0].contiguous(), None)), (ssa.cache_append, (d, good_append(), *[None] * 5))):
        with pytest.raises(ssa.SsaError, match=f.__name__):
            f(*args, stream=0)
        assert f(*args, stream=0, check=False) != ssa.OK
    other, c = x.half(), i[..., 0].contiguous()              # another type than the cache's queries have
    for call in (lambda: ssa.attn_window_fp4(d, good_window(), other, *[None] * 6, stream=0), lambda: ssa.block_bounds(d, k, None, None, b.half(), stream=0),
                 lambda: ssa.block_select(d, k, other, b, None, i, c, stream=0), lambda: ssa.block_select(d, k, x, b.float(), None, i, c, stream=0),
                 lambda: ssa.attn_blocks(d, k, other, None, None, None, i, c, None, stream=0), lambda: ssa.cache_append(d, good_append(), other, *[None] * 4, stream=0),
                 lambda: ssa.cache_append(desc(ssa.F16), good_append(), x, *[None] * 4, stream=0)):
        with pytest.raises(ValueError, match="where the cache goes with"):
            call()
    few = [(b[:1], "bounds"), (b[:, :1], "bounds"), (b[:, :, :7], "bounds"), (b[..., :64], "bounds")]
    for bad, word in few:
        with pytest.raises(ValueError, match=word):
            ssa.block_bounds(d, k, None, None, bad, stream=0)
    for bad in (i[:1], i[..., :3].contiguous(), i.long(), i.transpose(0, 1)):
        with pytest.raises(ValueError, match="lists"):
            ssa.attn_blocks(d, k, x, x, x, i, bad, torch.zeros(2, 2, 4, dtype=torch.int32), x, stream=0)
    with pytest.raises(ValueError, match="lists"):
        ssa.block_select(d, k, x, b, i, i, torch.zeros(15, dtype=torch.int32), stream=0)
    for bad in (torch.zeros(2, 2, 4, 7), torch.zeros(2, 2, 4, 8).half(), torch.zeros(2, 2, 3, 8)):
        with pytest.raises(ValueError, match="scores"):
            ssa.block_select(d, k, x, b, i, i, torch.zeros(16, dtype=torch.int32), bad, stream=0)


def test_what_the_makers_refuse():
    q, kv = torch.zeros(2, 8, 3, 128).bfloat16(), torch.zeros(2, 2, 3, 128).bfloat16()
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    a = ssa.make_append(kv, kv, q, q, torch.zeros(9, 64), True, i32(2, 3), i32(2))
    assert (a.n_q, a.rotary_dims, a.n_positions, a.interleaved, a.q_stride_t, a.kn_stride_h) == (3, 64, 9, 1, 128, 384)
    for bad in (dict(v_new=kv[:1]), dict(q=q[:, :, :2]), dict(q_out=q.float()), dict(v_new=kv.transpose(2, 3)), dict(cos_sin=torch.zeros(9, 64).double()), dict(cos_sin=torch.zeros(9, 128)[:, :64]),
                dict(positions=i32(2, 2)), dict(positions=i32(2, 3).long()), dict(positions=i32(2, 6)[:, ::2]), dict(q_lens=i32(1)), dict(q_lens=i32(2).long())):
        with pytest.raises(ValueError):
            ssa.make_append(**{**dict(k_new=kv, v_new=kv), **bad})
    bounds = torch.zeros(2, 2, 5, 2, 128)
    k = ssa.make_blocks(3, 64, 4, 1, 2, q, q, bounds[:, :, :4], i32(2))
    assert (k.q_stride_t, k.o_stride_t, k.bounds_stride_b, k.bounds_stride_h) == (128, 128, 2560, 1280)
    for bad in (dict(n_q=2), dict(bounds=bounds[..., :64]), dict(bounds=bounds[0]), dict(bounds=bounds.transpose(2, 3)), dict(q_lens=i32(1)), dict(q_lens=i32(2).long())):
        with pytest.raises(ValueError):
            ssa.make_blocks(**{**dict(n_q=3, block_size=64, budget=4, q=q, bounds=bounds), **bad})
    codes, scales = torch.zeros(2, 2, 10, 64, dtype=torch.uint8), torch.zeros(2, 2, 10, 8, dtype=torch.uint8)
    d = ssa.make_desc_fp4(q[:, :, 0], codes, codes, scales, scales, q[:, :, 0])
    assert (d.kv_dtype, d.k_stride_t, d.v_stride_h, d.k_stride_b, d.max_ctx) == (ssa.FP4_E2M1, 128, 1280, 2560, 10)
    pool, pool_scales = torch.zeros(7, 16, 2, 64, dtype=torch.uint8), torch.zeros(7, 16, 2, 8, dtype=torch.uint8)
    d = ssa.make_desc_fp4(q[:, :, 0], pool, pool, pool_scales, pool_scales, q[:, :, 0], 100, paged=True)
    assert (d.kv_dtype, d.k_stride_t, d.k_stride_h, d.k_stride_b, d.H_kv, d.max_ctx) == (ssa.FP4_E2M1, 256, 128, 0, 2, 100)
    for bad in (dict(k=codes[..., :32]), dict(k_scales=scales[..., :4]), dict(v_scales=scales[:, :, :9]), dict(v_scales=torch.zeros(2, 10, 2, 8, dtype=torch.uint8).transpose(1, 2)),
                dict(k=codes.float()), dict(k_scales=torch.zeros(2, 2, 10, 16, dtype=torch.uint8)[..., ::2])):
        with pytest.raises(ValueError):
            ssa.make_desc_fp4(**{**dict(q=q[:, :, 0], k=codes, v=codes, k_scales=scales, v_scales=scales, out=q[:, :, 0]), **bad})
