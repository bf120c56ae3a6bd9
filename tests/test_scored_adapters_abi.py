"""Entry points of scored routing, of layers on given routing and of adapters on the host: struct layouts, sizes, and what they
refuse before anything is launched (CPU only)."""
import ctypes
import os
import subprocess

import pytest

import paper_2511_10054_amd as bm

HDR = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
ONE = ctypes.c_void_p(256)       # non-null and aligned, never dereferenced on these paths
ODD = ctypes.c_void_p(264)
NULL, SHAPE, DTYPE, WORKSPACE, ALIGN = -1, -2, -3, -4, -7
BIG = 1 << 60


def test_struct_layouts_match_header(tmp_path):
    structs = {"bm_router_desc": bm.RouterDesc, "bm_adapter_desc": bm.AdapterDesc}
    lines = []
    for name, cls in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
    for name in ("BM_SCORE_SOFTMAX", "BM_SCORE_SIGMOID"):
        lines.append(f'printf("{name} %d\\n", (int){name});')
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "buddymoe.h"\nint main(void){' + "".join(lines) + "return 0;}\n")
    subprocess.run(["gcc", "-I", HDR, "-o", str(tmp_path / "layout"), str(src)], check=True)
    got = dict(l.split() for l in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines())
    for name, cls in structs.items():
        assert int(got[name]) == ctypes.sizeof(cls)
        for f in cls._fields_:
            assert int(got[f"{name}.{f[0]}"]) == getattr(cls, f[0]).offset
    assert int(got["BM_SCORE_SOFTMAX"]) == bm.BM_SCORE_SOFTMAX and int(got["BM_SCORE_SIGMOID"]) == bm.BM_SCORE_SIGMOID


def _router(**over):
    return bm.RouterDesc(**dict(dict(T=4, d=64, E=64, K=8, n_groups=8, keep_groups=4, group_top=2, scoring=bm.BM_SCORE_SIGMOID,
                                     dtype=bm.BM_BF16, flags=bm.BM_RENORM_TOPK, scale=2.5), **over))


@pytest.mark.parametrize("over,want", [
    (dict(dtype=2), DTYPE), (dict(T=-1), SHAPE), (dict(d=0), SHAPE), (dict(d=48), SHAPE), (dict(d=(1 << 20) + 32), SHAPE), (dict(E=0), SHAPE),
    (dict(E=260, n_groups=1, keep_groups=1), SHAPE), (dict(K=0), SHAPE), (dict(K=33), SHAPE), (dict(T=1 << 30), SHAPE), (dict(n_groups=0), SHAPE),
    (dict(n_groups=7), SHAPE), (dict(E=256, n_groups=128, keep_groups=64, group_top=1), SHAPE), (dict(keep_groups=0), SHAPE), (dict(keep_groups=9), SHAPE),
    (dict(keep_groups=1, K=9), SHAPE), (dict(group_top=0), SHAPE), (dict(group_top=3), SHAPE), (dict(n_groups=64, keep_groups=64, group_top=2), SHAPE),
    (dict(scoring=2), SHAPE), (dict(scoring=-1), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(T=0), 0),
])
def test_router_refuses_descriptors(over, want):
    d = _router(**over)
    # x, w_router, bias, balance, ids, w, workspace
    assert bm.load_library().bm_route_scored(ctypes.byref(d), *(ONE,) * 7, BIG, None) == want
    assert (bm.bm_workspace_bytes_scored(d) == 0) == (want != 0 or d.T == 0)


def test_router_refuses_pointers():
    lib = bm.load_library()
    d = _router()

    def but(i, v):
        return [v if j == i else ONE for j in range(7)]

    for i in (0, 1, 4, 5):
        assert lib.bm_route_scored(ctypes.byref(d), *but(i, None), BIG, None) == NULL, i
    for i in (0, 1):
        assert lib.bm_route_scored(ctypes.byref(d), *but(i, ODD), BIG, None) == ALIGN, i
    for ws, n in ((None, BIG), (ODD, BIG), (ONE, bm.bm_workspace_bytes_scored(d) - 1)):
        assert lib.bm_route_scored(ctypes.byref(d), *(ONE,) * 6, ws, n, None) == WORKSPACE
    assert lib.bm_route_scored(None, *(ONE,) * 7, BIG, None) == NULL
    assert lib.bm_workspace_bytes_scored(None) == 0
    assert lib.bm_route_scored(ctypes.byref(_router(T=0)), *(None,) * 7, 0, None) == 0


@pytest.mark.parametrize("E,dtype", [(8, 1), (256, 1), (60, 0)])
def test_router_workspace_serves_smaller_batches(E, dtype):
    last = 0
    for T in (1, 2, 15, 16, 17, 64, 65, 100, 255, 256, 257, 1000, 2047, 2048, 2049, 8192, 16384, 16385, 40000, 1 << 20):
        now = bm.bm_workspace_bytes_scored(_router(T=T, E=E, K=1, n_groups=1, keep_groups=1, dtype=dtype))
        assert now >= last and now % 256 == 0, T
        last = now


def _adapters(**over):
    return bm.AdapterDesc(**dict(dict(rows=10, Kd=64, N=96, n=4, rank=16, dtype=bm.BM_BF16, y_dtype=bm.BM_F32), **over))


@pytest.mark.parametrize("over,want", [
    (dict(dtype=2), DTYPE), (dict(y_dtype=-1), DTYPE), (dict(rows=-1), SHAPE), (dict(rows=(1 << 24) + 1), SHAPE), (dict(Kd=0), SHAPE), (dict(N=0), SHAPE),
    (dict(Kd=(1 << 20) + 1), SHAPE), (dict(N=(1 << 20) + 1), SHAPE), (dict(n=0), SHAPE), (dict(n=1025), SHAPE), (dict(rank=0), SHAPE), (dict(rank=129), SHAPE),
    (dict(x_stride=63), SHAPE), (dict(x_stride=-64), SHAPE), (dict(base_stride=95), SHAPE), (dict(y_stride=95), SHAPE), (dict(rows=0), 0),
])
def test_adapters_refuse_descriptors(over, want):
    # x, adapter, a, b, ranks, scale, base, y, workspace
    d = _adapters(**over)
    args = [ONE] * 7 + [ctypes.c_void_p(512), ONE]
    assert bm.load_library().bm_add_adapters(ctypes.byref(d), *args, BIG, None) == want
    assert (bm.bm_workspace_bytes_adapters(d) == 0) == (want != 0 or d.rows == 0)


def test_adapters_refuse_pointers():
    lib = bm.load_library()
    d = _adapters()
    for i in (0, 1, 2, 3, 6, 7):
        args = [None if j == i else ONE for j in range(9)]
        assert lib.bm_add_adapters(ctypes.byref(d), *args, BIG, None) == NULL, i
    for ws, n in ((None, BIG), (ODD, BIG), (ONE, bm.bm_workspace_bytes_adapters(d) - 1)):
        assert lib.bm_add_adapters(ctypes.byref(d), ctypes.c_void_p(512), *(ONE,) * 7, ws, n, None) == WORKSPACE
    # in place, the rows of base are those of y; x is read while y is written
    two = ctypes.c_void_p(512)
    assert lib.bm_add_adapters(ctypes.byref(_adapters(base_stride=96, y_stride=128)), two, *(ONE,) * 8, BIG, None) == SHAPE
    assert lib.bm_add_adapters(ctypes.byref(d), *(ONE,) * 6, two, ONE, ONE, BIG, None) == SHAPE
    assert lib.bm_add_adapters(None, *(ONE,) * 9, BIG, None) == NULL
    assert lib.bm_workspace_bytes_adapters(None) == 0
    assert lib.bm_add_adapters(ctypes.byref(_adapters(rows=0)), *(None,) * 9, 0, None) == 0


@pytest.mark.parametrize("Kd,n,rank,dtype", [(64, 4, 16, 1), (4096, 1, 128, 1), (4096, 1024, 64, 1), (1442, 5, 12, 0), (1 << 20, 3, 8, 0)])
def test_adapter_workspace_serves_smaller_batches(Kd, n, rank, dtype):
    last = 0
    for rows in list(range(1, 70)) + [100, 127, 128, 129, 500, 1000, 1023, 1024, 1025, 1100, 2047, 2048, 2049, 5000, 20000, 32768, 40000, 100000, 1 << 24]:
        now = bm.bm_workspace_bytes_adapters(_adapters(rows=rows, Kd=Kd, n=n, rank=rank, dtype=dtype))
        assert now >= last and now % 256 == 0, rows
        last = now


def _layer(**over):
    return bm.LayerDesc(**dict(dict(T=16, d=64, E=8, F=128, K=2, n_shared=0, R=3, H=3, dtype=bm.BM_BF16, flags=0), **over))


def test_routed_layer_refusals():
    lib = bm.load_library()
    names = [f[0] for f in bm.Weights._fields_]
    need = bm.bm_workspace_bytes(_layer())

    def weights(missing=()):
        return bm.Weights(*[0 if n in missing + ("w_router", "router_bias", "buddy_q") or n.startswith("wp_") or n.startswith("wsp_") else 256 for n in names])

    def call(d=None, x=ONE, ids=ONE, w=ONE, wt=None, bitmap=ONE, table=ONE, y=ONE, ws=ONE, nbytes=need):
        return lib.bm_moe_forward_routed(ctypes.byref(d or _layer()), x, ids, w, ctypes.byref(wt or weights()), bitmap, table, y, ws, nbytes, None, None)

    for kw in (dict(x=None), dict(ids=None), dict(w=None), dict(bitmap=None), dict(table=None), dict(y=None)):
        assert call(**kw) == NULL, kw
    for name in ("w_gate", "w_up", "w_down"):
        assert call(wt=weights((name,))) == NULL
    assert call(_layer(flags=bm.BM_PSI_TOKEN)) in (NULL, SHAPE) and call(_layer(K=9)) == SHAPE and call(_layer(dtype=5)) == DTYPE
    full = bm.Weights(*[256] * len(names))
    assert call(_layer(flags=bm.BM_PSI_TOKEN), wt=full) == SHAPE
    assert call(ws=None) == WORKSPACE and call(ws=ODD) == WORKSPACE and call(nbytes=need - 1) == WORKSPACE
    assert call(_layer(T=0), x=None, ids=None, w=None, y=None, ws=None, nbytes=0) == 0


def test_routed_quantized_layer_refusals():
    lib = bm.load_library()
    names = [f[0] for f in bm.QuantizedWeights._fields_]
    need = bm.bm_workspace_bytes_quantized(_layer())

    def weights(missing=()):
        return bm.QuantizedWeights(*[0 if n in missing + ("w_router", "router_bias", "buddy_q") else 256 for n in names])

    def call(d=None, x=ONE, xq=ONE, xs=ONE, ids=ONE, w=ONE, wt=None, bitmap=ONE, table=ONE, y=ONE, ws=ONE, nbytes=need):
        return lib.bm_moe_forward_routed_quantized(ctypes.byref(d or _layer()), x, xq, xs, ids, w, ctypes.byref(wt or weights()), bitmap, table, y, ws,
                                                   nbytes, None, None)

    for kw in (dict(ids=None), dict(w=None), dict(bitmap=None), dict(table=None), dict(y=None), dict(xq=None), dict(xs=None), dict(x=None, xq=None, xs=None)):
        assert call(**kw) == NULL, kw
    for name in ("w_gate", "gate_scale", "w_up", "up_scale", "w_down", "down_scale"):
        assert call(wt=weights((name,))) == NULL
    assert call(_layer(flags=bm.BM_PSI_TOKEN)) == SHAPE and call(_layer(dtype=bm.BM_F32)) == DTYPE
    assert call(xq=ODD) == ALIGN and call(x=ODD) == ALIGN
    assert call(x=None, nbytes=need - 1) == WORKSPACE        # the 8-bit form alone will do
    assert call(_layer(T=0), x=None, xq=None, xs=None, ids=None, w=None, y=None, ws=None, nbytes=0) == 0
