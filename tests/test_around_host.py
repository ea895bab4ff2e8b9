"""Refusals of the operators around the layer: every call fails its host checks
before any HIP call (CPU)."""
import ctypes
import os

import numpy as np
import pytest

from paper_2608_02989_amd import _lib as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="HIP library not built")

V = ctypes.c_void_p
A, B, C, D, E = (V(0x100000 + i * 0x10000000) for i in range(5))  # aligned, apart, never dereferenced


def refused(rc, code, word):
    assert rc == code and word in L.lib().acceptmoe_last_error().decode()


def norm(hidden=A, dtype=L.BF16, y=B, weight=C, T=4, H=64, eps=1e-6, group=0, hidden_out=A, norm_out=D, scale=E):
    return L.lib().acceptmoe_residual_norm(hidden, dtype, y, weight, T, H, eps, group, hidden_out, norm_out, scale, None)


@pytest.mark.parametrize("change,code,word", [
    ({"dtype": 7}, L.ERR_INVALID_ARG, "dtype"), ({"T": -1}, L.ERR_INVALID_ARG, "sizes"),
    ({"H": 0}, L.ERR_INVALID_ARG, "sizes"), ({"H": 66}, L.ERR_UNSUPPORTED, "multiple of 4"),
    ({"H": 65540}, L.ERR_UNSUPPORTED, "65536"), ({"eps": -1.0}, L.ERR_INVALID_ARG, "eps"),
    ({"eps": float("nan")}, L.ERR_INVALID_ARG, "eps"), ({"group": 48}, L.ERR_UNSUPPORTED, "group"),
    ({"group": 128}, L.ERR_UNSUPPORTED, "multiple of the group"), ({"hidden": None}, L.ERR_INVALID_ARG, "null"),
    ({"weight": None}, L.ERR_INVALID_ARG, "null"), ({"norm_out": None}, L.ERR_INVALID_ARG, "null"),
    ({"hidden_out": None}, L.ERR_INVALID_ARG, "hidden_out"), ({"group": 32, "scale": None}, L.ERR_INVALID_ARG, "scale"),
    ({"y": V(0x100008)}, L.ERR_INVALID_ARG, "aligned"), ({"norm_out": A}, L.ERR_INVALID_ARG, "overlaps"),
    ({"hidden_out": V(0x100010)}, L.ERR_INVALID_ARG, "overlaps"), ({"hidden_out": D}, L.ERR_INVALID_ARG, "overlaps")])
def test_residual_norm_rejects(change, code, word):
    refused(norm(**change), code, word)


@pytest.mark.parametrize("scale", [A, B, C, D, V(A.value + 4 * 64 * 2 - 4), V(D.value - 4)],
                         ids=["hidden", "y", "weight", "norm_out", "hidden's end", "norm_out's start"])
@pytest.mark.parametrize("group", [32, -1])
def test_residual_norm_rejects_overlapping_scales(scale, group):
    refused(norm(group=group, scale=scale), L.ERR_INVALID_ARG, "scale_out overlaps")
    refused(norm(group=group, scale=scale, hidden_out=V(E.value + 0x10000000)), L.ERR_INVALID_ARG, "scale_out overlaps")


def test_no_ops():
    assert norm(T=0) == L.OK
    assert sample(R=0) == L.OK
    assert accept(T=0, trees=0) == L.OK


def sample(logits=A, dtype=L.F32, stride=100, R=2, vocab=100, u=B, token=C, prob=D, ws=E, nbytes=1 << 30):
    return L.lib().acceptmoe_sample(logits, dtype, stride, R, vocab, u, None, None, None, None, token, prob, ws, nbytes,
                                    None)


@pytest.mark.parametrize("change,code,word", [
    ({"dtype": 2}, L.ERR_INVALID_ARG, "dtype"), ({"R": -1}, L.ERR_INVALID_ARG, "sizes"),
    ({"vocab": 0}, L.ERR_INVALID_ARG, "sizes"), ({"vocab": L.MAX_VOCAB + 1, "stride": 1 << 21}, L.ERR_UNSUPPORTED, "V must"),
    ({"R": L.MAX_SAMPLE_ROWS + 1}, L.ERR_UNSUPPORTED, "R <="), ({"stride": 99}, L.ERR_INVALID_ARG, "row_stride"),
    ({"logits": None}, L.ERR_INVALID_ARG, "null"), ({"u": None}, L.ERR_INVALID_ARG, "null"),
    ({"token": None}, L.ERR_INVALID_ARG, "null"), ({"prob": None}, L.ERR_INVALID_ARG, "null"),
    ({"logits": V(0x100002)}, L.ERR_INVALID_ARG, "aligned"), ({"ws": None}, L.ERR_WORKSPACE, "workspace"),
    ({"nbytes": 0}, L.ERR_WORKSPACE, "workspace"), ({"ws": V(0x100010)}, L.ERR_WORKSPACE, "aligned")])
def test_sample_rejects(change, code, word):
    refused(sample(**change), code, word)


def test_sample_workspace_size():
    f = L.lib().acceptmoe_sample_workspace_size
    assert f(4, 0) == 0 and f(-1, 10) == 0 and f(4, L.MAX_VOCAB + 1) == 0
    for vocab in (1, 1000, 32000, 131072, L.MAX_VOCAB):
        sizes = [f(r, vocab) for r in range(0, 600)]
        assert sizes == sorted(sizes) and sizes[1] > 0


def accept(token=A, parent=B, target=C, offs=None, trees=1, T=5, on=D, path=E, path_len=5, length=A, bonus=B):
    arr = None if offs is None else np.ascontiguousarray(offs, np.int32)
    return L.lib().acceptmoe_accept(token, parent, target, None if arr is None else arr.ctypes.data, trees, T, on, path,
                                    path_len, length, bonus, None)


@pytest.mark.parametrize("change,code,word", [
    ({"T": -1}, L.ERR_INVALID_ARG, "T must"), ({"trees": 0}, L.ERR_UNSUPPORTED, "B must"),
    ({"trees": 257}, L.ERR_UNSUPPORTED, "B must"), ({"trees": 2}, L.ERR_INVALID_ARG, "NULL"),
    ({"offs": [1, 5]}, L.ERR_INVALID_ARG, "must be 0"), ({"offs": [0, 4]}, L.ERR_INVALID_ARG, "equal T"),
    ({"offs": [0, 7, 5], "trees": 2}, L.ERR_INVALID_ARG, "non-decreasing"),
    ({"T": 1025, "path_len": 1025}, L.ERR_UNSUPPORTED, "nodes"), ({"path_len": 4}, L.ERR_INVALID_ARG, "path_len"),
    ({"token": None}, L.ERR_INVALID_ARG, "null"), ({"parent": None}, L.ERR_INVALID_ARG, "null"),
    ({"target": None}, L.ERR_INVALID_ARG, "null"), ({"on": None}, L.ERR_INVALID_ARG, "null"),
    ({"path": None}, L.ERR_INVALID_ARG, "null"), ({"length": None}, L.ERR_INVALID_ARG, "null"),
    ({"bonus": None}, L.ERR_INVALID_ARG, "null")])
def test_accept_rejects(change, code, word):
    refused(accept(**change), code, word)


# ---------------------------------------------------------------------------
# experts in 4 bits
# ---------------------------------------------------------------------------
def fwd(hidden=A, wgu=B, wd=C, T=4, H=64, I=32, experts=8, k=2, idx=D, gate=D, out=E, ws=V(0x200000000), nbytes=1 << 40):
    return L.lib().acceptmoe_moe_forward_q4(hidden, wgu, wd, T, H, I, experts, k, idx, gate, out, ws, nbytes, None)


@pytest.mark.parametrize("change,code,word", [
    ({"T": -1}, L.ERR_INVALID_ARG, "T must"), ({"H": 48}, L.ERR_UNSUPPORTED, "multiples of 32"),
    ({"I": 0}, L.ERR_UNSUPPORTED, "multiples of 32"), ({"H": 65568}, L.ERR_UNSUPPORTED, "65536"),
    ({"experts": 513}, L.ERR_UNSUPPORTED, "E must"), ({"k": 0}, L.ERR_UNSUPPORTED, "k must"),
    ({"k": 33}, L.ERR_UNSUPPORTED, "k must"), ({"T": 1 << 30}, L.ERR_UNSUPPORTED, "too large"),
    ({"hidden": None}, L.ERR_INVALID_ARG, "null"), ({"wgu": None}, L.ERR_INVALID_ARG, "null"),
    ({"wd": None}, L.ERR_INVALID_ARG, "null"), ({"idx": None}, L.ERR_INVALID_ARG, "null"),
    ({"gate": None}, L.ERR_INVALID_ARG, "null"), ({"out": None}, L.ERR_INVALID_ARG, "null"),
    ({"out": V(0x100008)}, L.ERR_INVALID_ARG, "aligned"), ({"ws": None}, L.ERR_WORKSPACE, "needs"),
    ({"nbytes": 100}, L.ERR_WORKSPACE, "needs"), ({"ws": V(0x200000010)}, L.ERR_WORKSPACE, "aligned")])
def test_forward_q4_rejects(change, code, word):
    refused(fwd(**change), code, word)


@pytest.mark.parametrize("change", [{"T": 1 << 25, "k": 32, "I": 128}, {"T": 1 << 25, "k": 8, "I": 1024, "H": 32},
                                    {"T": 32767, "k": 32, "H": 65536, "I": 65536, "experts": 512, "nbytes": 100}])
def test_forward_q4_more_workgroups_than_a_launch_takes(change):
    """Refused before the first launch, also where T * ceil(H / 1024) is small."""
    T, k, I, H, E = (change.get(n, d) for n, d in (("T", 4), ("k", 2), ("I", 32), ("H", 32), ("experts", 8)))
    fits = (T * k // 64 + E + 16) * -(-max(I, H // 2) // 128) < 1 << 24
    if fits:  # a large call that stays within the limits gets as far as its workspace
        refused(fwd(**change), L.ERR_WORKSPACE, "needs")
    else:
        refused(fwd(**{"H": H, **change}), L.ERR_UNSUPPORTED, "workgroups")


def test_q4_sizes():
    lib = L.lib()
    # a quad of 16-row tiles takes 4,352 bytes per 128 columns
    assert lib.acceptmoe_q4_gate_up_bytes(8, 96, 256) == 8 * 3 * 2 * 4352
    assert lib.acceptmoe_q4_down_bytes(8, 256, 96) == 8 * 4 * 1 * 4352
    assert lib.acceptmoe_q4_down_bytes(8, 96, 160) == 8 * 2 * 2 * 4352
    for bad in ((0, 96, 256), (8, 40, 256), (8, 96, 0), (513, 96, 256), (8, 65568, 32)):
        assert lib.acceptmoe_q4_gate_up_bytes(*bad) == 0 and lib.acceptmoe_q4_down_bytes(*bad) == 0
    sizes = [lib.acceptmoe_moe_forward_q4_workspace_size(t, 2048, 768, 128, 8) for t in range(300)]
    assert sizes == sorted(sizes) and fwd(T=0) == L.OK
    assert lib.acceptmoe_moe_forward_q4_workspace_size(-1, 2048, 768, 128, 8) == 0


def test_q4_packing_rejects():
    lib = L.lib()
    refused(lib.acceptmoe_quantize_q4(A, 5, 64, B, C, None), L.ERR_INVALID_ARG, "dtype")
    refused(lib.acceptmoe_quantize_q4(A, L.F32, 65, B, C, None), L.ERR_INVALID_ARG, "multiple of 32")
    refused(lib.acceptmoe_quantize_q4(A, L.F32, 64, None, C, None), L.ERR_INVALID_ARG, "null")
    refused(lib.acceptmoe_quantize_q4(A, L.F32, 64, V(0x100010), C, None), L.ERR_INVALID_ARG, "overlap")
    refused(lib.acceptmoe_quantize_q4(V(0x100004), L.F32, 64, B, C, None), L.ERR_INVALID_ARG, "aligned")
    assert lib.acceptmoe_quantize_q4(None, L.F32, 0, None, None, None) == L.OK
    up = lib.acceptmoe_pack_gate_up_q4
    refused(up(A, B, C, D, 4, 40, 64, E, None), L.ERR_UNSUPPORTED, "multiples of 32")
    refused(up(A, B, C, None, 4, 32, 64, E, None), L.ERR_INVALID_ARG, "null")
    refused(up(A, B, C, D, 4, 32, 64, A, None), L.ERR_INVALID_ARG, "overlaps")
    refused(up(A, B, C, D, 4, 32, 64, V(0x100004), None), L.ERR_INVALID_ARG, "aligned")
    down = lib.acceptmoe_pack_down_q4
    refused(down(A, B, 0, 64, 32, E, None), L.ERR_UNSUPPORTED, "E must")
    refused(down(None, B, 4, 64, 32, E, None), L.ERR_INVALID_ARG, "null")
    refused(down(A, B, 4, 64, 32, B, None), L.ERR_INVALID_ARG, "overlaps")
    refused(down(V(0x100008), B, 4, 64, 32, E, None), L.ERR_INVALID_ARG, "aligned")
