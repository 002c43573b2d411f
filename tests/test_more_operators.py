"""Rotary positions, root-mean-square norm, rows in 8 bits: what is decided on the host (no compute calls here)."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2309_12578_amd as sp
from paper_2309_12578_amd.binding import _RotaryParams

PI = Fraction("3.14159265358979323846264338327950288419716939937510582")


@pytest.mark.parametrize("head_dim,sections,base,ladder", [
    (64, (32,), 10000.0, "shared"), (64, (8, 12, 12), 10000.0, "shared"), (64, (16, 16), 100.0, "own"), (16, (1,), 2.0, "own"),
    (256, (5, 6, 7, 8), 500000.0, "own"), (32, (3, 2), 10000.0, "shared")])
@pytest.mark.parametrize("neighbours", [False, True])
def test_axes_by_their_definition(head_dim, sections, base, ladder, neighbours):
    a = sp.rotary_axes(head_dim, sections, base, ladder, neighbours)
    assert (a.head_dim, a.count, a.neighbours) == (head_dim, len(sections), neighbours)
    i, pairs = 0, head_dim // 2
    for axis, n in enumerate(sections):
        for j in range(n):
            frequency = base ** -(j / n) if ladder == "own" else base ** -(i / pairs)
            turns = int(a.turns[i]) % 2 ** 64
            assert abs(Fraction(turns, 2 ** 64) - Fraction(frequency) / (2 * PI)) <= Fraction(1, 2 ** 65)
            assert int(a.axis_of[i]) == axis
            i += 1
    assert not a.turns[i:].any() and a.turns.dtype == torch.int64 and a.axis_of.dtype == torch.uint8


@pytest.mark.parametrize("arguments", [
    dict(head_dim=64, sections=()), dict(head_dim=64, sections=(0, 4)), dict(head_dim=64, sections=(16, 17)), dict(head_dim=24, sections=(4,)),
    dict(head_dim=272, sections=(4,)), dict(head_dim=64, sections=(4,), base=1.0), dict(head_dim=64, sections=(4,), base=math.inf),
    dict(head_dim=64, sections=(4,), ladder="none"), dict(head_dim=0, sections=(4,))])
def test_axes_that_are_refused(arguments):
    with pytest.raises(ValueError):
        sp.rotary_axes(**arguments)


@pytest.mark.parametrize("yes,no", [(True, False), (1, 0), (np.True_, np.False_), (torch.tensor(True), torch.tensor(0))])
def test_pairing_by_any_truth_value(yes, no):
    for given, want in ((yes, True), (no, False)):
        axes = sp.rotary_axes(64, (32,), neighbours=given)
        assert axes.neighbours is want and sp.RotaryAxes(64, 1, axes.turns, axes.axis_of, given).neighbours is want
        assert sp.SparseMHA(64, 1, rotary=axes).rotary.neighbours is want
    with pytest.raises(ValueError):
        sp.rotary_axes(64, (32,), neighbours=np.zeros(2))


def test_axes_and_packed_rows_are_looked_at():
    t, u = torch.zeros(32, dtype=torch.int64), torch.zeros(32, dtype=torch.uint8)
    sp.RotaryAxes(64, 1, t, u)
    for bad in ((64, 0, t, u), (64, 256, t, u), (64, 1, t.int(), u), (64, 1, t, u.int()), (128, 1, t, u), (64, 1, t[None], u)):
        with pytest.raises(ValueError):
            sp.RotaryAxes(*bad)
    c, e = torch.zeros((3, 128), dtype=torch.int8), torch.zeros((3, 2), dtype=torch.uint8)
    assert sp.Packed8(c, e, 65).shape == (3, 65) and sp.Packed8(c, e, 128, torch.ones(128)).shape == (3, 128)
    for bad in ((c, e, 64), (c, e, 129), (c, e, 0), (c.int(), e, 128), (c, e.int(), 128), (c, e[:2], 128), (c, e, 65, torch.ones(64))):
        with pytest.raises(ValueError):
            sp.Packed8(*bad)


def test_tensors_that_are_not_on_a_device_are_refused():
    """Before anything is computed, with the package's own errors."""
    x, w = torch.zeros(2, 3, 64), torch.zeros(64)
    axes = sp.rotary_axes(64, (32,))
    p = sp.Packed8(torch.zeros((2, 64), dtype=torch.int8), torch.ones((2, 1), dtype=torch.uint8), 64)
    for call in (lambda: sp.rotary(x[None], axes, torch.zeros((1, 3), dtype=torch.int64)), lambda: sp.pack8(x), lambda: sp.unpack8(p),
                 lambda: sp.rms_norm(x, w), lambda: sp.rms_norm8(x, w), lambda: sp.linear8(x, torch.zeros(8, 64)), lambda: sp.pack8(3),
                 lambda: sp.unpack8(p, torch.float16), lambda: sp.linear8(x, torch.zeros(8, 64), checkpoint=p)):
        with pytest.raises(ValueError):
            call()


def test_sub_layer_options_that_are_refused():
    for bad in (dict(norm="none"), dict(rotary=sp.rotary_axes(128, (64,)))):
        with pytest.raises(ValueError):
            sp.SparseMHA(128, 2, **bad)
    mha = sp.SparseMHA(128, 2, norm="rms", rotary=sp.rotary_axes(64, (16, 16)), eight_bit=True)
    assert {n for n, _ in mha.named_parameters()} == {"norm.weight", "w_qkv.weight", "w_o.weight"}
    assert set(mha.state_dict()) == {"norm.weight", "w_qkv.weight", "w_o.weight"}
    assert mha.rotary.count == 2 and sp.SparseMHA(128, 2).rotary is None
    with pytest.raises(ValueError):
        sp.SparseMHA(128, 2)(torch.zeros(1, 32, 128), None, residual=torch.zeros(1, 32, 128))


FAKE, NONE = ctypes.c_void_p(256), ctypes.c_void_p(None)   # non-NULL, never dereferenced: validation fails first
SIZE = ctypes.c_size_t


def _rotary(**changes):
    p = _RotaryParams()
    p.B, p.H, p.L, p.d, p.rotated, p.axes, p.dtype, p.position_bytes = 2, 4, 8, 64, 4, 2, sp.SPION_BF16, 8
    for name, value in changes.items():
        setattr(p, name, value)
    return p


@pytest.mark.parametrize("changes,code", [
    (dict(B=0), -2), (dict(H=0), -2), (dict(H=65536, rotated=1), -2), (dict(L=0), -2), (dict(d=8), -2), (dict(d=24), -2), (dict(d=272), -2),
    (dict(B=1 << 16, L=1 << 15), -2), (dict(rotated=5), -5), (dict(rotated=-1), -5), (dict(axes=0), -5), (dict(axes=256), -5), (dict(dtype=2), -3),
    (dict(position_bytes=2), -5), (dict(flags=4), -5), (dict(reserved=1), -5)])
def test_rotary_refuses(changes, code):
    p = _rotary(**changes)
    assert sp.load().spion_rotary(FAKE, FAKE, FAKE, FAKE, FAKE, ctypes.byref(p), NONE) == code


def test_rotary_refuses_missing_and_misaligned_pointers():
    good = [FAKE] * 5 + [ctypes.byref(_rotary()), NONE]
    for i in range(6):
        bad = list(good)
        bad[i] = None
        assert sp.load().spion_rotary(*bad) == -1
    for i, at in ((0, 257), (1, 257), (2, 260), (4, 260)):
        bad = list(good)
        bad[i] = ctypes.c_void_p(at)
        assert sp.load().spion_rotary(*bad) == -5


@pytest.mark.parametrize("rows,D,dtype,code", [(0, 64, 0, -2), (-1, 64, 0, -2), (1, 0, 0, -2), (1, (1 << 20) + 1, 0, -2), (1 << 60, 64, 0, -2), (1, 64, 2, -3)])
def test_eight_bits_refuse(rows, D, dtype, code):
    lib = sp.load()
    assert lib.spion_pack_eight(FAKE, FAKE, FAKE, rows, D, dtype, NONE) == code
    assert lib.spion_unpack_eight(FAKE, FAKE, NONE, 0, FAKE, rows, D, dtype, NONE) == code


def test_eight_bits_refuse_missing_and_misaligned_pointers():
    lib = sp.load()
    for i in range(3):
        a = [FAKE] * 3
        a[i] = NONE
        assert lib.spion_pack_eight(*a, 1, 64, 0, NONE) == -1
        assert lib.spion_unpack_eight(a[0], a[1], NONE, 0, a[2], 1, 64, 0, NONE) == -1
    assert lib.spion_unpack_eight(FAKE, FAKE, FAKE, 7, FAKE, 1, 64, 0, NONE) == -3
    odd = ctypes.c_void_p(260)
    assert lib.spion_pack_eight(FAKE, odd, FAKE, 1, 64, 0, NONE) == -5
    assert lib.spion_unpack_eight(odd, FAKE, NONE, 0, FAKE, 1, 64, 0, NONE) == -5


def _norm(lib, x=FAKE, residual=FAKE, w=FAKE, y=FAKE, h=FAKE, rstd=FAKE, codes=FAKE, exponents=FAKE, rows=4, D=64, eps=1e-6, dtype=0, flags=0):
    return lib.spion_rms_norm(x, residual, w, y, h, rstd, codes, exponents, rows, D, eps, dtype, flags, NONE)


def test_norm_refuses():
    lib = sp.load()
    for bad in (dict(x=NONE), dict(w=NONE), dict(codes=NONE), dict(exponents=NONE), dict(y=NONE, h=NONE, rstd=NONE, codes=NONE, exponents=NONE)):
        assert _norm(lib, **bad) == -1
    for bad in (dict(rows=0), dict(D=0), dict(D=16385), dict(rows=1 << 60)):
        assert _norm(lib, **bad) == -2
    assert _norm(lib, dtype=5) == -3
    for bad in (dict(eps=-1e-9), dict(eps=math.nan), dict(eps=math.inf), dict(flags=2), dict(codes=ctypes.c_void_p(260))):
        assert _norm(lib, **bad) == -5


def test_norm_gradient_refuses():
    lib = sp.load()
    need = lib.spion_rms_norm_workspace_bytes(1000, 640)
    assert need >= 640 * 4 and sp.spion_rms_norm_workspace_bytes(1000, 640) == need
    assert lib.spion_rms_norm_workspace_bytes(0, 640) == SIZE(-1).value and lib.spion_rms_norm_workspace_bytes(5, 16385) == SIZE(-1).value
    with pytest.raises(sp.SpionError):
        sp.spion_rms_norm_workspace_bytes(5, 16385)

    def call(dy=FAKE, dh=FAKE, h=FAKE, codes=FAKE, exponents=FAKE, w=FAKE, rstd=FAKE, dx=FAKE, dw=FAKE, rows=1000, D=640, dtype=0, ws=FAKE, size=need):
        return lib.spion_rms_norm_grad(dy, dh, h, codes, exponents, w, rstd, dx, dw, rows, D, dtype, ws, size, NONE)
    for bad in (dict(dy=NONE), dict(w=NONE), dict(rstd=NONE), dict(dx=NONE), dict(codes=NONE), dict(exponents=NONE), dict(codes=NONE, exponents=NONE, h=NONE)):
        assert call(**bad) == -1
    assert call(rows=0) == -2 and call(D=16385) == -2 and call(dtype=9) == -3 and call(codes=ctypes.c_void_p(260)) == -5
    for bad in (dict(ws=NONE), dict(ws=ctypes.c_void_p(264)), dict(size=need - 1)):
        assert call(**bad) == -4


def test_weight_gradient_refuses():
    lib = sp.load()
    bytes_ = lib.spion_weight_grad_eight_workspace_bytes
    need = bytes_(5000, 300, 70)
    assert need >= 300 * 128 * 4 and sp.spion_weight_grad_eight_workspace_bytes(5000, 300, 70) == need
    for bad in ((0, 8, 8), (8, 0, 8), (8, 8, 0), (0x7fffffff - 4096, 8, 8), (8, (1 << 20) + 1, 8), (8, 8, (1 << 20) + 1), (8, 1 << 19, 1 << 19)):
        assert bytes_(*bad) == SIZE(-1).value
        with pytest.raises(sp.SpionError):
            sp.spion_weight_grad_eight_workspace_bytes(*bad)
        assert lib.spion_weight_grad_eight(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, *bad, 0, FAKE, 1 << 40, NONE) == -2

    def call(*pointers, rows=5000, N=300, M=70, dtype=0, ws=FAKE, size=need):
        return lib.spion_weight_grad_eight(*pointers, rows, N, M, dtype, ws, size, NONE)
    for i in (0, 1, 2, 4):
        a = [FAKE] * 6
        a[i] = NONE
        assert call(*a) == -1
    good = [FAKE] * 6
    assert call(*good, dtype=3) == -3 and call(FAKE, ctypes.c_void_p(264), *good[2:]) == -5
    for bad in (dict(ws=NONE), dict(ws=ctypes.c_void_p(264)), dict(size=need - 1)):
        assert call(*good, **bad) == -4


@pytest.mark.parametrize("rows,N,M", [(16384, 131072, 4096), (32768, 152064, 8192), (65536, 28672, 8192), (2 ** 30, 2 ** 13, 2 ** 13), (2 ** 20, 2 ** 20, 2 ** 16), (300, 2 ** 20, 64)])
def test_weight_gradient_of_large_projections_needs_little_room(rows, N, M):
    """Where dW has tiles enough to fill the machine, only the bias' sums: 2 numbers an output and 128 columns, a 16th of dW in bf16 (M up to 64: as much as dW)."""
    assert sp.spion_weight_grad_eight_workspace_bytes(rows, N, M) <= 2 * 4 * N * ((M + 127) // 128)
