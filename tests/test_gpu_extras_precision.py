"""Attention with a bias: score scales other than 1 / 8, and what the forward leaves so that the table's gradient is as exact as one in fp32.

u = 2^-8 is half a step of bf16, relative to the value."""
import numpy as np
import pytest
import torch

from test_gpu_extras import RNG, TOL, _formula, _inputs, _kept, _mask, _near, _rng, _run, _table, sp  # noqa: F401  (sp: the module's fixture)
from test_gpu_parity import _pattern_from_mask

pytestmark = pytest.mark.gpu


# Scores as large as elsewhere, so that the tolerances are; 0.3 has no exact inverse (the scale, its inverse and the bias over it are rounded once each:
# 3 u32 of a bias of less than 5, within the 256 u32); at 2^-100 the scores are the biases alone, and dQ and dK 2^-97 of what they are elsewhere.
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("scale", [1.0, 0.3, 2.0 ** -100])
def test_score_scales_with_a_bias(sp, dtype, block, scale):
    nb, B, H = 5, 2, 3
    L = nb * block
    fl = _mask(nb, seed=block + 1, density=0.7)
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, dtype, 80)
    q = (q * min(1.0, 0.125 / scale)).to(dtype)
    table, buckets = _table(32, H, dtype, 81), sp.relative_buckets(L, 32, 64, device="cuda")
    table[16:, 0] = -np.inf   # keys ahead, for one head
    lengths = torch.tensor([L, L - 21], dtype=torch.int32, device="cuda")
    got = _run(sp, q, k, v, do, pat, table, buckets=buckets, lengths=lengths, dropout=0.1, rng=_rng(), scale=scale)
    want, _ = _formula(q, k, v, do, _kept(fl, block), table, buckets.map, lengths, 0.1, RNG, 0, scale=float(np.float32(scale)))
    _near(got, want, TOL[dtype])


def _through_the_c_entries(sp, q, k, v, do, pat, block, table, bucket_of, dropout, rest):
    """O and the gradients, the backward with or without what rounding left of O."""
    B, H, L, _ = q.shape
    shape = dict(B=B, H=H, L=L, d=64, block=block, dtype=sp.SPION_BF16)
    kw = dict(table=table, bucket_of=bucket_of, dropout=dropout, rng=_rng())
    room = [torch.empty(max(sp.spion_attn_with_workspace_bytes(**shape, nnzb=pat.nnzb, is_bwd=b, **kw), 256), dtype=torch.uint8, device="cuda") for b in (False, True)]
    out = {n: torch.empty_like(table if n == "dtable" else q) for n in ("o", "dq", "dk", "dv") + (("dtable",) if table is not None else ())}
    lse = torch.empty((B, H, L), device="cuda")
    sp.spion_attn_fwd_with(q, k, v, out["o"], lse, pat.row_ptr, pat.col_idx, pat.nnzb, **shape, workspace=room[0], o_rest=rest, **kw)
    sp.spion_attn_bwd_with(q, k, v, out["o"], do, lse, out["dq"], out["dk"], out["dv"], out.get("dtable"), pat.row_ptr, pat.col_idx, pat.col_ptr, pat.row_idx,
                           pat.bsr_pos, pat.nnzb, **shape, workspace=room[1], o_rest=rest, **kw)
    return out


# O and o_rest together against the formula.  With a bias: what bf16 leaves of P (u of it) is rounded once more (u^2 = 2^-16 of P), in the product and in the sums,
# and so is what it leaves of O (2^-16 of O): with fp32's 256 * 2^-24 = 2^-16, 4 * 2^-16 of the magnitudes.  Without one P itself is rounded: scores that
# are all 0 give P = 1, which is exact; others are off by about u / sqrt(3) of the root of the sum of the squares of P, some 2^-12 of the magnitudes here.
@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("dropout", [0.0, 0.2])
def test_what_rounding_leaves_of_the_output(sp, block, dropout):
    nb, B, H = 8, 2, 2
    L = nb * block
    fl = _mask(nb, seed=9, density=0.6)
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, torch.bfloat16, 82)
    table, buckets = _table(32, H, torch.float32, 83), sp.relative_buckets(L, device="cuda")

    def off(q, table):   # of O, and of O with o_rest, in magnitudes; largest
        rest = torch.full_like(q, float("nan"))
        o = _through_the_c_entries(sp, q, k, v, do, pat, block, table, None if table is None else buckets.map, dropout, rest)["o"].double()
        exact, mag = _formula(q, k, v, do, _kept(fl, block), table, buckets.map, None, dropout, RNG, 0)[0]["o"]
        return [((got - exact).abs() / mag.clamp_min(2.0 ** -60)).max().item() for got in (o, o + rest.double())]

    for alone, both in (off(q, table), off(torch.zeros_like(q), None)):
        assert both <= 2.0 ** -14 < alone
    assert off(q, None)[1] > 2.0 ** -14


# Two buckets of half the keys each (and one of a single distance).  delta's error e is common to a row, and of the size of u |dO| |O| where O is a rounded one: over a
# bucket with the share f = 1 / 2 of a row it adds up to e f, where the values that cancel leave sqrt(f (1 - f)) of |dO| |O|: about u / 2.5 (the root mean
# square of a rounding's relative error) = 1.6e-3 of the table's gradient for O, and as much for P: 2.3e-3.  With what both left, 2^-8 of that, 9e-6, and fp32's
# noise.  The bounds are a tenth of the first and a dozen times the second, with a factor of two between them.
@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("dropout", [0.0, 0.1])
def test_table_gradient_over_far_buckets(sp, block, dropout):
    L, B, H = 1024, 2, 8
    nb = L // block
    fl = np.ones((nb, nb), dtype=np.uint8)
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, torch.bfloat16, 84)
    table, buckets = _table(4, H, torch.float32, 85), sp.relative_buckets(L, 4, 2, device="cuda")
    want, _ = _formula(q, k, v, do, _kept(fl, block), table, buckets.map, None, dropout, RNG, 0)
    exact = want["dtable"][0]
    off = lambda got: ((got["dtable"].double() - exact).norm() / exact.norm()).item()
    node = _run(sp, q, k, v, do, pat, table, buckets=buckets, dropout=dropout, rng=_rng())
    entries = [_through_the_c_entries(sp, q, k, v, do, pat, block, table, buckets.map, dropout, rest) for rest in (torch.empty_like(q), None)]
    assert off(node) <= 2.0 ** -13 and off(entries[0]) <= 2.0 ** -13
    assert off(entries[1]) > 2.0 ** -12
    for e in (node, *entries):
        _near(e, want, TOL[torch.bfloat16])
