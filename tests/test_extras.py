"""Relative position bias, dropout and lengths: what is decided on the host (no compute calls here)."""
import ctypes
import math
from fractions import Fraction

import pytest
import torch

import paper_2309_12578_amd as sp
from paper_2309_12578_amd.binding import _AttnExtras, _AttnParams


def _bucket_of(distance, count, max_distance, bidirectional):
    """The usual formula, with powers compared as fractions."""
    n = count // 2 if bidirectional else count
    far = abs(distance) if bidirectional else max(-distance, 0)
    exact = n // 2
    if far < exact:
        b = far
    else:
        b = exact   # the largest b with far >= exact (max_distance / exact)^((b - exact) / (n - exact))
        while b + 1 < n and Fraction(far, exact) ** (n - exact) >= Fraction(max_distance, exact) ** (b + 1 - exact):
            b += 1
    return b + (n if bidirectional and distance > 0 else 0)


@pytest.mark.parametrize("length,count,max_distance,bidirectional", [
    (300, 32, 128, True), (300, 32, 128, False), (1, 4, 2, True), (2, 2, 2, False), (50, 7, 20, False), (700, 256, 500, True),
    (400, 16, 64, True), (100, 32, 9, True)])
def test_buckets_by_their_definition(length, count, max_distance, bidirectional):
    b = sp.relative_buckets(length, count, max_distance, bidirectional)
    assert (b.length, b.count, b.map.dtype, tuple(b.map.shape)) == (length, count, torch.uint8, (2 * length - 1,))
    want = [_bucket_of(d, count, max_distance, bidirectional) for d in range(-(length - 1), length)]
    assert b.map.tolist() == want


@pytest.mark.parametrize("arguments", [
    dict(length=0), dict(length=5, count=0), dict(length=5, count=258), dict(length=5, count=31), dict(length=5, count=2),
    dict(length=5, count=1, bidirectional=False), dict(length=5, count=32, max_distance=8)])
def test_buckets_that_are_refused(arguments):
    with pytest.raises(ValueError):
        sp.relative_buckets(**arguments)


def test_bucket_maps_are_looked_at():
    m = torch.zeros(9, dtype=torch.uint8)
    assert sp.RelativeBuckets(5, 1, m).map is m
    for bad in ((5, 0, m), (5, 257, m), (4, 1, m), (5, 1, m.int()), (5, 1, m[None])):
        with pytest.raises(ValueError):
            sp.RelativeBuckets(*bad)


def test_map_of_shorter_sequences_is_the_middle():
    from paper_2309_12578_amd.extras import _map_for
    table, long, short = torch.zeros(32, 2), sp.relative_buckets(100), sp.relative_buckets(37)
    assert torch.equal(_map_for(table, long, 37), short.map) and _map_for(table, long, 100) is long.map
    for bad in (lambda: _map_for(table, short, 38), lambda: _map_for(table, None), lambda: _map_for(torch.zeros(31, 2), long)):
        with pytest.raises(ValueError):
            bad()


FAKE, NONE = ctypes.c_void_p(256), ctypes.c_void_p(None)   # non-NULL, never dereferenced: validation fails first


def _params(**changes):
    p = _AttnParams(2, 4, 256, 64, 32, sp.SPION_BF16, 0.0, 0)
    for name, value in changes.items():
        setattr(p, name, value)
    return p


def _extras(**changes):
    x = _AttnExtras(256, 256, 256, 256, None, 0.1, 32, sp.SPION_F32, 0, 0)
    for name, value in changes.items():
        setattr(x, name, value)
    return x


def _calls(p, x, nnzb=10):
    lib, P, X = sp.load(), ctypes.byref(p), ctypes.byref(x)
    fwd = [FAKE] * 7 + [nnzb, P, X, NONE, 0, NONE]
    bwd = [FAKE] * 15 + [nnzb, P, X, NONE, 0, NONE]
    return (lib.spion_attn_fwd_with, fwd), (lib.spion_attn_bwd_with, bwd)


@pytest.mark.parametrize("params,extras,code", [
    (dict(flags=1), {}, -5), (dict(d=32), {}, -2), (dict(block=48), {}, -2), (dict(L=250), {}, -2), (dict(dtype=2), {}, -3),
    (dict(B=0), {}, -2), (dict(L=65536 + 64, block=64), {}, -2), ({}, dict(reserved=1), -5),
    ({}, dict(dropout=1.0), -5), ({}, dict(dropout=-0.1), -5), ({}, dict(dropout=math.nan), -5), ({}, dict(dropout=1 - 2.0 ** -18), -5),
    ({}, dict(rng=None), -1), ({}, dict(bucket_of=None), -1), ({}, dict(n_buckets=0), -5), ({}, dict(n_buckets=257), -5),
    ({}, dict(table_dtype=7), -3), ({}, dict(o_rest=264), -5)])
def test_attention_calls_that_are_refused(params, extras, code):
    p, x = _params(**params), _extras(**extras)
    for call, args in _calls(p, x):
        assert call(*args) == code
    for is_bwd in (0, 1):
        assert sp.load().spion_attn_with_workspace_bytes(ctypes.byref(p), ctypes.byref(x), 10, is_bwd) == ctypes.c_size_t(-1).value


def test_attention_calls_without_their_pointers():
    for call, args in _calls(_params(), _extras()):
        for i, a in enumerate(args):
            if a is FAKE and not (call is sp.load().spion_attn_bwd_with and i == 9):   # dtable may be missing
                assert call(*args[:i], NONE, *args[i + 1:]) == -1, i
        for i in (-5, -4):   # the parameters themselves
            bad = list(args)
            bad[i] = None
            assert call(*bad) == -1
        odd = list(args)
        odd[0] = ctypes.c_void_p(264)
        assert call(*odd) == -5


def test_backward_needs_its_workspace():
    (_, _), (bwd, args) = _calls(_params(), _extras())
    assert bwd(*args) == -4
    need = sp.load().spion_attn_with_workspace_bytes(ctypes.byref(_params()), ctypes.byref(_extras()), 10, 1)
    assert need > 0
    for ptr, n in ((256, need - 1), (264, need), (None, need)):
        bad = list(args)
        bad[-3:-1] = ctypes.c_void_p(ptr), n
        assert bwd(*bad) == -4
    no_table = list(args)   # a gradient of a table that the call does not have
    no_table[-4] = ctypes.byref(_extras(table=None))
    assert bwd(*no_table) == -1


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), -3), (dict(n_buckets=0), -5), (dict(n_buckets=257), -5), (dict(H=0), -2), (dict(q_len=0), -2), (dict(k_len=0), -2),
    (dict(q_start=-1), -2), (dict(q_start=93), -2), (dict(k_len=101), -2), (dict(reach=0), -2), (dict(reach=2 ** 20 + 1), -2)])
def test_dense_bias_calls_that_are_refused(change, code):
    lib = sp.load()
    v = dict(reach=100, n_buckets=32, H=4, q_len=8, k_len=100, q_start=92, dtype=0)
    sizes = list({**v, **change}.values())
    assert lib.spion_relative_bias(FAKE, FAKE, FAKE, *sizes, NONE) == code
    assert lib.spion_relative_bias_grad(FAKE, FAKE, FAKE, *sizes, FAKE, 1 << 30, NONE) == code


def test_dense_bias_pointers_and_workspace():
    lib, sizes = sp.load(), [100, 32, 4, 8, 100, 92, 0]
    for i in range(3):
        args = [FAKE] * 3
        args[i] = NONE
        assert lib.spion_relative_bias(*args, *sizes, NONE) == -1
        assert lib.spion_relative_bias_grad(*args, *sizes, FAKE, 1 << 30, NONE) == -1
    need = sp.spion_relative_bias_workspace_bytes(32, 4, 8, 100)
    for ws, n in ((NONE, need), (FAKE, need - 1), (ctypes.c_void_p(264), need)):
        assert lib.spion_relative_bias_grad(FAKE, FAKE, FAKE, *sizes, ws, n, NONE) == -4
    with pytest.raises(sp.SpionError):
        sp.spion_relative_bias_workspace_bytes(0, 4, 8, 100)


def test_dropout_calls_that_are_refused():
    call = sp.load().spion_dropout_add
    for args, code in (((NONE, FAKE, FAKE, 8, 0, 0.1, FAKE), -1), ((FAKE, FAKE, NONE, 8, 0, 0.1, FAKE), -1), ((FAKE, FAKE, FAKE, 8, 0, 0.1, NONE), -1),
                       ((FAKE, FAKE, FAKE, 8, 2, 0.1, FAKE), -3), ((FAKE, FAKE, FAKE, 0, 0, 0.1, FAKE), -2), ((FAKE, FAKE, FAKE, 8, 0, 1.0, FAKE), -5),
                       ((FAKE, FAKE, FAKE, 8, 0, -1.0, FAKE), -5), ((FAKE, FAKE, FAKE, 8, 0, math.nan, FAKE), -5)):
        assert call(*args, NONE, 0, NONE) == code, args


def test_host_tensors_are_refused():
    q = torch.zeros(1, 1, 32, 64)
    index = torch.zeros(2, dtype=torch.int32)
    pattern = sp.Pattern(32, 32, None, index, index, index, index, index, None, None, 1)
    with pytest.raises(ValueError):
        sp.sparse_attention(q, q, q, pattern, lengths=torch.ones(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        sp.relative_bias(torch.zeros(32, 1), sp.relative_buckets(8), 8, 8)
    with pytest.raises(ValueError):
        sp.dropout_add(q, None, 0.1, torch.zeros(2, dtype=torch.int64))


def test_sub_layer_arguments():
    with pytest.raises(ValueError):
        sp.SparseMHA(128, 2, attn_dropout=1.0)
    mha = sp.SparseMHA(128, 2, buckets=sp.relative_buckets(64))
    assert mha.bias_table.shape == (32, 2) and mha.buckets.length == 64
    assert "bias_table" in mha.state_dict() and "bucket_map" not in mha.state_dict()
    assert set(sp.SparseMHA(128, 2).state_dict()) == {"norm.weight", "norm.bias", "w_qkv.weight", "w_o.weight"}
    with pytest.raises(ValueError):
        mha(torch.zeros(1, 64, 128), None, sp.SPION_ATTN_PAPER_DENOM)


@pytest.mark.parametrize("more", [{}, dict(lengths=torch.ones(1, dtype=torch.int32)), dict(dropout=0.1)])
def test_buckets_without_their_table_are_refused(more):
    q = torch.zeros(1, 1, 32, 64)
    index = torch.zeros(2, dtype=torch.int32)
    pattern = sp.Pattern(32, 32, None, index, index, index, index, index, None, None, 1)
    with pytest.raises(ValueError, match="table"):
        sp.sparse_attention(q, q, q, pattern, buckets=sp.relative_buckets(32), **more)


@pytest.mark.parametrize("scale,table,refused", [(2.0 ** -101, 256, True), (1e-39, 256, True), (2.0 ** -100, 256, False), (0.0, 256, False), (1e-39, None, False)])
def test_scales_that_biases_cannot_be_divided_by(scale, table, refused):
    """A bias of 2^27 over 2^-100 is a number of fp32, one of 1 over 1e-39 is not."""
    p, x = _params(scale=scale), _extras(table=table)
    sizes = [sp.load().spion_attn_with_workspace_bytes(ctypes.byref(p), ctypes.byref(x), 10, is_bwd) for is_bwd in (0, 1)]
    assert [n == ctypes.c_size_t(-1).value for n in sizes] == [refused] * 2
    if refused:
        assert all(call(*args) == -5 for call, args in _calls(p, x))
