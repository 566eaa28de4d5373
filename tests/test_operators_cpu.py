"""CPU checks of the layer operators' entry points: every argument that they refuse is refused with its code before any
GPU work, empty calls are accepted, struct layouts match the C compiler's, and the binding's own checks."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_1910_01578_amd import gdp, rel_layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                                # an aligned address that no refused call reads
BIG = 1 << 40
INVALID, UNSUPPORTED, WORKSPACE = gdp.GDP_E_INVALID_ARG, gdp.GDP_E_UNSUPPORTED, gdp.GDP_E_WORKSPACE
ref = ctypes.byref


def _refused(code, status, *words):
    assert code == status, (code, gdp.last_error())
    for w in words:
        assert w in gdp.last_error(), gdp.last_error()


# LayerNorm -----------------------------------------------------------------------------------

def _norm(**kw):
    a = dict(rows=5, width=12, dtype=gdp.GDP_BF16, x=P, ld_x=12, residual=P, ld_res=12, gamma=P, beta=P, eps=1e-5, y=P,
             ld_y=12, sum=P, ld_sum=12)
    a.update(kw)
    return gdp.lib.gdp_layer_norm(*a.values(), None)


def _norm_backward(**kw):
    a = dict(rows=5, width=12, dtype=gdp.GDP_BF16, h=P, ld_h=12, gamma=P, eps=1e-5, dy=P, ld_dy=12, dsum=P, ld_dsum=12,
             dh=P, ld_dh=12, dgamma=P, dbeta=P, ws=P, bytes=BIG)
    a.update(kw)
    return gdp.lib.gdp_layer_norm_backward(*a.values(), None)


@pytest.mark.parametrize("call", [_norm, _norm_backward])
@pytest.mark.parametrize("status, word, kw", [
    (INVALID, "rows", dict(rows=-1)), (UNSUPPORTED, "rows", dict(rows=2 ** 62)), (INVALID, "width", dict(width=0)),
    (UNSUPPORTED, "GDP_MAX_NORM_WIDTH", dict(width=8193)), (INVALID, "dtype", dict(dtype=7)),
    (INVALID, "eps", dict(eps=-1e-9)), (INVALID, "eps", dict(eps=float("nan"))), (INVALID, "eps", dict(eps=float("inf"))),
    (INVALID, "gamma", dict(gamma=None)), (INVALID, "gamma", dict(gamma=P + 1))])
def test_norm_refusals(call, status, word, kw):
    _refused(call(**kw), status, word)


@pytest.mark.parametrize("name, kw", [
    ("x", dict(x=None)), ("x", dict(x=P + 1)), ("beta", dict(beta=None)), ("y", dict(y=None)), ("residual", dict(residual=P + 1)),
    ("sum", dict(sum=P + 1)), ("ld_x", dict(ld_x=11)), ("ld_res", dict(ld_res=0)), ("ld_y", dict(ld_y=11)),
    ("ld_sum", dict(ld_sum=-12))])
def test_norm_array_refusals(name, kw):
    _refused(_norm(**kw), INVALID, name)


@pytest.mark.parametrize("name, kw", [
    ("h", dict(h=None)), ("dy", dict(dy=None)), ("dh", dict(dh=None)), ("dgamma", dict(dgamma=None)),
    ("dbeta", dict(dbeta=P + 2)), ("ld_h", dict(ld_h=11)), ("ld_dy", dict(ld_dy=11)), ("ld_dsum", dict(ld_dsum=11)),
    ("ld_dh", dict(ld_dh=11))])
def test_norm_backward_array_refusals(name, kw):
    _refused(_norm_backward(**kw), INVALID, name)


def test_norm_workspace():
    assert gdp.lib.gdp_layer_norm_workspace_bytes(-1, 4) == 0
    assert gdp.lib.gdp_layer_norm_workspace_bytes(4, 8193) == 0
    for rows, width in ((0, 1), (1, 1), (5, 12), (52000, 256), (7, 8192), (2 ** 33, 64)):
        assert gdp.lib.gdp_layer_norm_workspace_bytes(rows, width) >= 256
    _refused(_norm_backward(ws=None), INVALID, "workspace")
    _refused(_norm_backward(bytes=8), WORKSPACE)
    _refused(_norm(rows=5, ld_x=BIG + 1), UNSUPPORTED, "ld_x")


# FC layer --------------------------------------------------------------------------------------

def _layer(**kw):
    f = gdp.GdpFcLayer(100, 24, 40, gdp.GDP_BF16, 1, 24, 40, 40, 40, 40, 24, 24)
    for k, v in kw.items():
        setattr(f, k, v)
    return f


FC_SIZES = [
    (INVALID, "rows", dict(rows=-1)), (UNSUPPORTED, "rows", dict(rows=2 ** 31)), (INVALID, "in_dim", dict(in_dim=0)),
    (INVALID, "out_dim", dict(out_dim=-3)), (INVALID, "act", dict(act=2)), (INVALID, "dtype", dict(dtype=-1)),
    (UNSUPPORTED, "tiles", dict(rows=2 ** 31 - 1, out_dim=2 ** 20, ld_y=2 ** 20)),
    (UNSUPPORTED, "tiles", dict(rows=1, in_dim=2 ** 22, out_dim=2 ** 22))]


@pytest.mark.parametrize("status, word, kw", FC_SIZES)
def test_fc_size_refusals(status, word, kw):
    f = _layer(**kw)
    _refused(gdp.lib.gdp_fc(ref(f), P, P, P, P, P, P, None), status, word)
    assert gdp.lib.gdp_fc_workspace_bytes(ref(f)) == 0 and word in gdp.last_error()
    _refused(gdp.lib.gdp_fc_backward(ref(f), P, P, P, P, P, P, P, P, P, BIG, None), status, word)


def test_fc_array_refusals():
    f = _layer()
    names = ("x", "w", "b", "residual", "y", "act_out")
    for i, n in enumerate(names):
        args = [P] * 6
        args[i] = P + 1
        _refused(gdp.lib.gdp_fc(ref(f), *args, None), INVALID, n)
        args[i] = None
        if n in ("x", "w", "y"):
            _refused(gdp.lib.gdp_fc(ref(f), *args, None), INVALID, n)
    for n, least in (("ld_x", 24), ("ld_y", 40), ("ld_res", 40), ("ld_act", 40)):
        _refused(gdp.lib.gdp_fc(ref(_layer(**{n: least - 1})), P, P, P, P, P, P, None), INVALID, n)
    assert gdp.lib.gdp_fc(None, P, P, P, P, P, P, None) == INVALID


def test_fc_backward_array_refusals():
    names = ("dy", "x", "w", "act_out", "dx_add", "dx", "dw", "db")
    for i, n in enumerate(names):
        args = [P] * 8
        args[i] = P + 1
        _refused(gdp.lib.gdp_fc_backward(ref(_layer()), *args, P, BIG, None), INVALID, n)
        args[i] = None
        if n in ("dy", "x", "w", "act_out"):
            _refused(gdp.lib.gdp_fc_backward(ref(_layer()), *args, P, BIG, None), INVALID, n)
    for n, least in (("ld_dy", 40), ("ld_x", 24), ("ld_act", 40), ("ld_dx", 24), ("ld_dx_add", 24)):
        _refused(gdp.lib.gdp_fc_backward(ref(_layer(**{n: least - 1})), *[P] * 8, P, BIG, None), INVALID, n)
    need = gdp.lib.gdp_fc_workspace_bytes(ref(_layer()))
    assert need >= 256
    _refused(gdp.lib.gdp_fc_backward(ref(_layer()), *[P] * 8, P, need - 1, None), WORKSPACE)
    _refused(gdp.lib.gdp_fc_backward(ref(_layer()), *[P] * 8, None, need, None), INVALID, "workspace")


@pytest.mark.parametrize("dtype", [gdp.GDP_F32, gdp.GDP_BF16])
@pytest.mark.parametrize("rows", [0, 1, 64, 65, 257, 100003])
@pytest.mark.parametrize("k, n", [(1, 1), (3, 1000), (256, 1024), (1001, 515)])
def test_fc_workspace_holds_its_parts(dtype, rows, k, n):
    """At least the copies that the products read and one set of partial sums."""
    for act, ld_x, ld_dy in ((0, k, n), (1, k + 1, n), (0, k, n + 3)):
        f = _layer(rows=rows, in_dim=k, out_dim=n, dtype=dtype, act=act, ld_x=ld_x, ld_dy=ld_dy)
        least = 256
        if dtype == gdp.GDP_BF16:
            least = max(256, 4 * (n * k + n))
            if act or n % 8 or ld_dy % 8:
                least += rows * n * 2
            if k % 8 or ld_x % 8:
                least += rows * k * 2
        elif act:
            least += rows * n * 4
        assert gdp.lib.gdp_fc_workspace_bytes(ref(f)) >= least


# attention --------------------------------------------------------------------------------------

def _attn(**kw):
    a = dict(lengths=[70, 0, 33], heads=6, d_head=16, bounds=[1, 2, 9], kv_heads=2, seg_len=32, mem_len=16)
    a.update(kw)
    return gdp.RelAttention(**a)


def _calls(c):
    fwd = gdp.lib.gdp_rel_attention(ref(c), P, P, P, P, P, P, P, P, BIG, None), gdp.last_error()
    bwd = gdp.lib.gdp_rel_attention_backward(ref(c), P, P, P, P, P, P, P, P, P, P, P, P, P, BIG, None), gdp.last_error()
    return fwd, bwd


ATTN = [
    (INVALID, "n_graphs", dict(n_graphs=0)), (UNSUPPORTED, "GDP_MAX_GRAPHS", dict(n_graphs=100000)),
    (INVALID, "NULL", dict(len_h=None)), (INVALID, "NULL", dict(key_start_h=None)), (INVALID, "n_kv_heads", dict(n_kv_heads=4)),
    (INVALID, "n_kv_heads", dict(n_kv_heads=0)), (INVALID, "n_heads", dict(n_heads=-2)), (UNSUPPORTED, "head_dim", dict(head_dim=24)),
    (INVALID, "seg_len", dict(seg_len=0)), (INVALID, "mem_len", dict(mem_len=-1)), (INVALID, "causal", dict(causal=2)),
    (INVALID, "n_bounds", dict(n_bounds=-1)), (UNSUPPORTED, "GDP_MAX_REL_BOUNDS", dict(n_bounds=64)),
    (INVALID, "bounds_h", dict(bounds_h=None)), (INVALID, "scale", dict(scale=float("nan"))),
    (INVALID, "scale", dict(scale=float("inf"))), (INVALID, "dtype", dict(dtype=5)), (INVALID, "ld_q", dict(ld_q=95)),
    (INVALID, "ld_k", dict(ld_k=31)), (INVALID, "ld_v", dict(ld_v=0)), (INVALID, "ld_o", dict(ld_o=95)),
    (UNSUPPORTED, "ld_q", dict(ld_q=BIG + 1))]


@pytest.mark.parametrize("status, word, kw", ATTN)
def test_attention_refusals(status, word, kw):
    p = _attn()
    for k, v in kw.items():
        setattr(p._c, k, v)
    for code, error in _calls(p._c):
        assert code == status and word in error, (code, error)
    for backward in (0, 1):
        assert gdp.lib.gdp_rel_attention_workspace_bytes(ref(p._c), backward) == 0 and word in gdp.last_error()


@pytest.mark.parametrize("status, word, kw", [
    (INVALID, "ascend", dict(bounds=[0, 4])), (INVALID, "ascend", dict(bounds=[4, 4])), (INVALID, "ascend", dict(bounds=[5, 4])),
    (INVALID, "negative", dict(lengths=[-1, 5], starts=[0, 0])), (INVALID, "negative", dict(lengths=[5], starts=[-2])),
    (UNSUPPORTED, "GDP_MAX_REL_LEN", dict(lengths=[2 ** 28 + 1])), (INVALID, "n_query_h", dict(lengths=[5], queries=[6])),
    (INVALID, "n_query_h", dict(lengths=[5], queries=[-1])),
    (UNSUPPORTED, "too many", dict(lengths=[2 ** 28] * 8, heads=64, kv_heads=64, starts=[0] * 8))])
def test_attention_batch_refusals(status, word, kw):
    with pytest.raises(gdp.GdpError) as e:
        _attn(**kw)
    assert word in str(e.value)
    assert gdp.lib.gdp_rel_attention_workspace_bytes(None, 0) == 0
    assert gdp.lib.gdp_rel_attention_workspace_bytes(ref(_attn()._c), 2) == 0


def test_attention_array_refusals():
    p = _attn()
    fwd = ["q", "k", "v", "table", None, "o", "lse"]
    for i, n in enumerate(fwd):
        if n is None:
            continue
        args = [P] * 7
        args[i] = P + 1
        _refused(gdp.lib.gdp_rel_attention(ref(p._c), *args, P, BIG, None), INVALID, n)
        args[i] = None
        if n != "lse":
            _refused(gdp.lib.gdp_rel_attention(ref(p._c), *args, P, BIG, None), INVALID, n)
    bwd = ["dout", "q", "k", "v", "table", None, "o", "lse", "dq", "dk", "dv", "dtable"]
    for i, n in enumerate(bwd):
        if n is None:
            continue
        for bad in (P + 1, None):
            args = [P] * 12
            args[i] = bad
            _refused(gdp.lib.gdp_rel_attention_backward(ref(p._c), *args, P, BIG, None), INVALID, n)
    for n in ("ld_do", "ld_dq", "ld_dk", "ld_dv"):
        c = gdp.GdpRelAttn.from_buffer_copy(p._c)
        setattr(c, n, 1)
        _refused(gdp.lib.gdp_rel_attention_backward(ref(c), *[P] * 12, P, BIG, None), INVALID, n)
    for backward, call, n in ((0, gdp.lib.gdp_rel_attention, 7), (1, gdp.lib.gdp_rel_attention_backward, 12)):
        need = gdp.lib.gdp_rel_attention_workspace_bytes(ref(p._c), backward)
        assert need >= 256
        _refused(call(ref(p._c), *[P] * n, P, need - 1, None), WORKSPACE)
        _refused(call(ref(p._c), *[P] * n, None, need, None), INVALID, "workspace")


def test_attention_backward_refuses_shared_key_rows():
    """Two graphs may read the same rows; their gradients would have no place."""
    p = _attn(lengths=[10, 10], starts=[0, 9])
    assert gdp.lib.gdp_rel_attention_workspace_bytes(ref(p._c), 1) == 0 and "overlap" in gdp.last_error()
    assert gdp.lib.gdp_rel_attention_workspace_bytes(ref(_attn(lengths=[10, 10], starts=[10, 0])._c), 1) > 0


# empty calls, bounds, layouts --------------------------------------------------------------------

def test_no_rows_is_no_work():
    assert _norm(rows=0, x=None, gamma=None, beta=None, y=None) == gdp.GDP_OK
    assert gdp.lib.gdp_fc(ref(_layer(rows=0)), None, None, None, None, None, None, None) == gdp.GDP_OK
    p = _attn(queries=[0, 0, 0])
    assert gdp.lib.gdp_rel_attention(ref(p._c), None, None, None, None, None, None, None, None, 0, None) == gdp.GDP_OK


@pytest.mark.parametrize("buckets, reach", [(1, 5), (2, 100), (8, 48), (16, 128), (32, 128), (64, 1 << 20), (64, 10)])
def test_rel_bounds(buckets, reach):
    b = gdp.rel_bounds(buckets, reach)
    assert len(b) == buckets - 1 and all(x < y for x, y in zip([0] + b, b))
    half = max(1, buckets // 2) if buckets > 1 else 0
    assert b[:half] == list(range(1, half + 1))
    if reach > 2 * buckets and buckets > 2:
        assert b[-1] == reach
    gdp.RelAttention([4], 1, 16, b)
    with pytest.raises(gdp.GdpError):
        gdp.rel_bounds(0, reach)


def test_struct_layouts_match_c_compiler(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = {"gdp_fc_layer": gdp.GdpFcLayer, "gdp_rel_attn": gdp.GdpRelAttn}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "gdp.h"', "int main(void) {"]
    for cname, py in structs.items():
        lines.append(f'printf("{cname} size %zu\\n", sizeof({cname}));')
        lines += [f'printf("{cname} {f} %zu\\n", offsetof({cname}, {f}));' for f, _ in py._fields_]
    lines.append('printf("limits norm %d\\nlimits bounds %d\\n", GDP_MAX_NORM_WIDTH, GDP_MAX_REL_BOUNDS); return 0; }')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines))
    exe = tmp_path / "layout"
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    want = {"limits norm": 8192, "limits bounds": 63}
    for cname, py in structs.items():
        want[f"{cname} size"] = ctypes.sizeof(py)
        want.update({f"{cname} {f}": getattr(py, f).offset for f, _ in py._fields_})
    assert {l.rsplit(" ", 1)[0]: int(l.rsplit(" ", 1)[1]) for l in out if l} == want


# the binding -----------------------------------------------------------------------------------

@pytest.mark.parametrize("call", [
    lambda x, g: gdp.layer_norm(x, g, g), lambda x, g: gdp.layer_norm_backward(x, g, x), lambda x, g: gdp.fc(x, x),
    lambda x, g: gdp.fc_backward(x, x, x)])
def test_tensors_off_the_gpu_are_refused(call):
    with pytest.raises(gdp.GdpError, match="not on a GPU"):
        call(torch.zeros(4, 4), torch.zeros(4))


def test_binding_refusals():
    x, g = torch.zeros(4, 6), torch.zeros(6)
    for bad, word in (
            (lambda: gdp.layer_norm(x.double(), g, g), "float64"), (lambda: gdp.layer_norm(x[0], g, g), "matrix"),
            (lambda: gdp.fc(x, x, act="gelu"), "act"), (lambda: gdp.fc(x.half(), x), "float16"),
            (lambda: gdp.fc_backward(x, x, x, act="tanh"), "act"),
            (lambda: gdp.RelAttention([4, 5], 2, 16, [], starts=[0]), "length"),
            (lambda: gdp.RelAttention([4, 5], 2, 16, [], queries=[1]), "length"),
            (lambda: gdp.RelAttention([4], 2, 20, []), "head_dim"),
            (lambda: gdp.RelAttention([4], 3, 16, [], kv_heads=2), "n_kv_heads"),
            (lambda: gdp.RelAttention([4], 2, 16, []).forward(x, x, x, g), "GPU"),
            (lambda: gdp.RelAttention([5], 2, 16, []).forward(x, x, x, g), "5 rows"),
            (lambda: gdp.RelAttention([4], 2, 16, []).forward(torch.zeros(4, 32), torch.zeros(4, 32), torch.zeros(4, 32),
                                                              torch.zeros(2, 2)), "GPU"),
            (lambda: rel_layer.RelPlacerLayer(gdp.RelAttention([4], 2, 16, []), {}), "w_qkv")):
        with pytest.raises(gdp.GdpError) as e:
            bad()
        assert word in str(e.value)
    weights = {n: None for n in rel_layer.FIELDS}
    for kw in (dict(queries=[1]), dict(starts=[2])):
        with pytest.raises(gdp.GdpError, match="same rows"):
            rel_layer.RelPlacerLayer(gdp.RelAttention([4], 2, 16, [], **kw), weights)
    rel_layer.RelPlacerLayer(gdp.RelAttention([4], 2, 16, []), weights)


def test_plan_counts():
    p = _attn(queries=[3, 0, 33])
    assert (p.n_queries, p.n_rows, p.n_keys, p.n_buckets) == (36, 103, 103, 8)
    assert _attn(causal=True).n_buckets == 4
    assert _attn(lengths=[0, 0]).n_rows == 0
    assert gdp.RelAttention([7, 9], 1, 16, [], starts=[20, 2]).n_rows == 27
    assert isinstance(p.lengths, np.ndarray) and p.lengths.dtype == np.int32
