"""Attention with a bias, dropout and lengths, the dense bias, and dropout with the residual, against their formulas in fp64.

Tolerances count roundings, each at most half a step relative to the value (bf16: u = 2^-8, fp32: 2^-24), per element and relative to
the sum of the magnitudes that the element is added up from.  bf16: the probabilities or their gradients as operands, the saved
output inside delta, the result: fewer than 4 u.  fp32: sums of up to 64 products and of a row's terms, an exponential of a
score of magnitude 16 or less: 256 u."""
import numpy as np
import pytest
import torch

import spion_inputs as si
from test_gpu_parity import _pattern_from_mask

pytestmark = pytest.mark.gpu
TOL = {torch.float32: 256 * 2.0 ** -24, torch.bfloat16: 4 * 2.0 ** -8}
M32 = 0xffffffff


@pytest.fixture(scope="module")
def sp():
    import paper_2309_12578_amd as sp
    sp.load()
    sp.binding._native()
    return sp


def _philox(c0, c1, c2, c3, seed):
    """Philox4x32 with 7 rounds on int64 tensors and numbers below 2^32."""
    k0, k1 = seed & M32, (seed >> 32) & M32

    def product(m, c):   # 32 x 32 bits in halves of 16: int64 has no room for all 64
        lo, hi = (c & 0xffff) * m, (c >> 16) * m
        low = lo + ((hi & 0xffff) << 16)
        return (hi >> 16) + (low >> 32), low & M32

    for _ in range(7):
        h0, l0 = product(0xD2511F53, c0)
        h1, l1 = product(0xCD9E8D57, c2)
        c0, c1, c2, c3 = (h1 ^ c1 ^ k0) & M32, l1, (h0 ^ c3 ^ k1) & M32, l0
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return c0, c1, c2, c3


def _threshold(p):
    return int(np.rint(65536 * p))


def _factors(draws, p):
    """c M of 16-bit draws, fp64"""
    t = _threshold(p)
    return (draws >= t).double() * (65536.0 / (65536 - t))


def _score_factors(BH, L, p, rng, stream):
    seed, offset = [int(v) for v in rng]
    dev = "cuda"
    bh, q, k = [torch.arange(n, device=dev) for n in (BH, L, L)]
    bh, q, k = bh[:, None, None], q[None, :, None], k[None, None, :]
    c0 = ((q // 2) << 14 | k // 4).expand(BH, L, L)
    one = torch.ones_like(c0)
    words = torch.stack(_philox(c0, (bh + 2 ** 31) * one, one * (offset & M32), one * stream, seed), -1)
    word = torch.gather(words, -1, (k % 4).expand(BH, L, L)[..., None])[..., 0]
    return _factors(torch.where(q % 2 == 0, word & 0xffff, word >> 16), p)


def _flat_factors(index, p, rng, stream):
    seed, offset = [int(v) for v in rng]
    one = torch.ones_like(index)
    words = torch.stack(_philox(index // 8 & M32, index // 8 >> 32, one * (offset & M32), one * stream, seed), -1)
    word = torch.gather(words, -1, (index // 2 % 4)[..., None])[..., 0]
    return _factors(torch.where(index % 2 == 0, word & 0xffff, word >> 16), p)


def _formula(q, k, v, do, kept, table, bucket_of, lengths, p, rng, stream, scale=0.125):
    """O, LSE, dQ, dK, dV, dtable and the magnitudes that they are sums of; kept: bool [L, L]."""
    B, H, L, _ = q.shape
    pos = torch.arange(L, device="cuda")
    seen = kept.expand(B, H, L, L)
    if lengths is not None:
        valid = pos[None] < lengths[:, None]
        seen = seen & valid[:, None, None, :] & valid[:, None, :, None]
        q, k, v, do = [torch.where(valid[:, None, :, None], t, torch.zeros_like(t)) for t in (q, k, v, do)]
    q, k, v, do = [t.double() for t in (q, k, v, do)]
    s = q @ k.transpose(-1, -2).contiguous() * scale
    if table is not None:
        t = torch.where(table > -1e30, table.double(), torch.full_like(table, -np.inf, dtype=torch.float64))
        bucket = bucket_of[(pos[None, :] - pos[:, None]) + L - 1].long().clamp_max(table.shape[0] - 1)
        s = s + t[bucket].permute(2, 0, 1)
    s = s.masked_fill(~seen, -np.inf)
    lse = torch.logsumexp(s, -1)
    P = torch.where(lse[..., None] > -np.inf, (s - lse[..., None]).exp(), torch.zeros_like(s))
    P = P.masked_fill(~seen, 0.0)
    cM = _score_factors(B * H, L, p, rng, stream).view(B, H, L, L) if _threshold(p) else torch.ones_like(P)
    A = P * cM
    T = lambda m: m.transpose(-1, -2).contiguous()
    o, o_mag = A @ v, A @ v.abs()
    dP, dP_mag = do @ T(v) * cM, do.abs() @ T(v.abs()) * cM
    delta, delta_mag = (do * o).sum(-1, keepdim=True), (do.abs() * o_mag).sum(-1, keepdim=True)
    dS, dS_mag = P * (dP - delta), P * (dP_mag + delta_mag)
    res = {"o": (o, o_mag), "dq": (dS @ k * scale, dS_mag @ k.abs() * scale), "dk": (T(dS) @ q * scale, T(dS_mag) @ q.abs() * scale),
           "dv": (T(A) @ do, T(A) @ do.abs())}
    if table is not None:
        sums = [torch.zeros(table.shape, dtype=torch.float64, device="cuda").index_add_(
            0, bucket.reshape(-1), m.sum(0).permute(1, 2, 0).reshape(-1, H)) for m in (dS, dS_mag)]
        res["dtable"] = tuple(sums)
    return res, lse


def _near(got, want, tol):
    for name, (value, mag) in want.items():
        g = got[name].double()
        assert g.shape == value.shape, name
        bad = ~((g - value).abs() <= tol * mag)
        assert not bad.any(), (name, int(bad.sum()), (g - value).abs()[bad].max().item(), mag[bad].max().item())


def _mask(nb, seed, density=0.5):
    """A pattern with a block row and a block column that keep nothing."""
    fl = si.random_block_mask(nb, density, seed=seed)
    if nb > 2:
        fl[nb // 2, :] = 0
        fl[:, nb // 3] = 0
    return np.ascontiguousarray(fl)


def _inputs(B, H, L, dtype, seed, n=4):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((B, H, L, 64), generator=gen, device="cuda").to(dtype) for _ in range(n)]


def _table(count, H, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((count, H), generator=gen, device="cuda").to(dtype)


def _run(sp, q, k, v, do, pat, table=None, **kw):
    leaves = [t.detach().requires_grad_(True) for t in (q, k, v)]
    t = None if table is None else table.detach().requires_grad_(True)
    o = sp.sparse_attention(*leaves, pat, bias=t, **kw)
    grads = torch.autograd.grad(o, leaves + ([t] if t is not None else []), do)
    return dict(zip(("o", "dq", "dk", "dv", "dtable"), (o.detach(), *grads)))


def _kept(fl, block):
    return torch.from_numpy(np.kron(fl, np.ones((block, block), dtype=np.uint8))).cuda().bool()


RNG = (-0x123456789abcdef, (5 << 32) + 77)   # a seed with all its bits, an offset of which the low 32 count


def _rng(values=RNG):
    return torch.tensor(values, dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("parts", ["lengths", "bias", "dropout", "bias dropout", "bias lengths dropout"])
def test_attention_against_the_formula(sp, dtype, block, parts):
    nb, B, H = 7, 3, 2
    L = nb * block
    fl = _mask(nb, seed=block)
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, dtype, 1)
    kw, table, buckets, lengths, p = {}, None, None, None, 0.0
    if "lengths" in parts:
        lengths = torch.tensor([L - 5, 0, 2 * block + 1], dtype=torch.int32, device="cuda")
        kw["lengths"] = lengths
        for t in (q, k, v, do):   # what lies there enters nothing
            for b, n in enumerate(lengths.tolist()):
                t[b, :, n:] = float("nan")
    if "bias" in parts:
        table, buckets = _table(32, H, dtype, 2), sp.relative_buckets(L, 32, 64, device="cuda")
        kw["buckets"] = buckets
    if "dropout" in parts:
        p = 0.3
        kw.update(dropout=p, rng=_rng(), stream=9)
    got = _run(sp, q, k, v, do, pat, table, **kw)
    want, _ = _formula(q, k, v, do, _kept(fl, block), table, None if buckets is None else buckets.map, lengths, p, RNG, 9)
    _near(got, want, TOL[dtype])
    if lengths is not None:   # exactly nothing from the lengths on
        for b, n in enumerate(lengths.tolist()):
            assert all(not got[name][b, :, n:].any() for name in ("o", "dq", "dk", "dv"))
    again = _run(sp, q, k, v, do, pat, table, **kw)
    assert all(torch.equal(got[n], again[n]) for n in got)


# Rows of one block to more than the 64 that are looked up at once, and rows that are cut into pieces because few heads have them
@pytest.mark.parametrize("dtype,block,nb,B,H", [(torch.bfloat16, 64, 70, 1, 1), (torch.bfloat16, 32, 140, 1, 1), (torch.bfloat16, 32, 67, 2, 2),
                                               (torch.bfloat16, 16, 70, 1, 1), (torch.float32, 16, 70, 1, 2), (torch.float32, 32, 66, 1, 1)])
def test_long_and_short_rows(sp, dtype, block, nb, B, H):
    L = nb * block
    fl = np.eye(nb, dtype=np.uint8)
    fl[1, :] = 1          # all keys, and all queries of one block column
    fl[:, 2] = 1
    fl[nb - 1, ::2] = 1
    fl[5, :] = 0
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, dtype, 3)
    table, buckets = _table(32, H, dtype, 4), sp.relative_buckets(L, device="cuda")
    lengths = torch.tensor([L - 3, L // 2 + 1][:B], dtype=torch.int32, device="cuda")
    got = _run(sp, q, k, v, do, pat, table, buckets=buckets, lengths=lengths, dropout=0.1, rng=_rng())
    want, _ = _formula(q, k, v, do, _kept(fl, block), table, buckets.map, lengths, 0.1, RNG, 0)
    _near(got, want, TOL[dtype])


# More workgroups than run at once: rows and columns in their other orders, 32 rows a workgroup in fp32; heads that divide over the XCDs and not
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("B,H", [(8, 8), (9, 7)])
def test_many_heads(sp, dtype, block, B, H):
    L = 1088
    nb = L // block
    fl = _mask(nb, seed=block + B, density=0.2)
    fl[:, nb - 1] = 1
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, dtype, 50)
    table, buckets = _table(32, H, dtype, 51), sp.relative_buckets(L, device="cuda")
    lengths = torch.tensor([L - 130 * b for b in range(B)], dtype=torch.int32, device="cuda")
    got = _run(sp, q, k, v, do, pat, table, buckets=buckets, lengths=lengths, dropout=0.15, rng=_rng())
    want, _ = _formula(q, k, v, do, _kept(fl, block), table, buckets.map, lengths, 0.15, RNG, 0)
    _near(got, want, TOL[dtype])


def test_calls_on_two_streams_at_once(sp):
    block, nb = 64, 40
    L = nb * block
    pat = _pattern_from_mask(sp, _mask(nb, seed=6, density=0.9), block)   # rows and columns in pieces
    buckets, rng = sp.relative_buckets(L, device="cuda"), _rng()
    sets = [(*_inputs(1, 2, L, torch.bfloat16, 60 + i), _table(32, 2, torch.float32, 62 + i)) for i in range(2)]
    run = lambda s: _run(sp, *s[:4], pat, s[4], buckets=buckets, dropout=0.1, rng=rng)
    want = [run(s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(run(sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g[n], want[i][n]) for g in got[i] for n in want[i])


@pytest.mark.parametrize("dtype,block", [(torch.float32, 16), (torch.bfloat16, 16), (torch.bfloat16, 32), (torch.bfloat16, 64)])
@pytest.mark.parametrize("count", [1, 3, 64, 65, 256])
def test_any_map_and_any_number_of_buckets(sp, dtype, block, count):
    nb, B, H = 4, 2, 3
    L = nb * block
    gen = torch.Generator().manual_seed(count)
    m = torch.randint(0, min(count + 2, 256), (2 * L - 1,), generator=gen, dtype=torch.uint8)   # past the last counts as the last
    m[L - 1:L + block] = 0                                                                      # and a stretch of one bucket
    buckets = sp.RelativeBuckets(L, count, m.cuda())
    table = _table(count, H, dtype, 5)
    fl = _mask(nb, seed=count, density=0.7)
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, dtype, 6)
    want, _ = _formula(q, k, v, do, _kept(fl, block), table, buckets.map, None, 0.0, RNG, 0)
    _near(_run(sp, q, k, v, do, pat, table, buckets=buckets), want, TOL[dtype])


@pytest.mark.parametrize("dtype,block", [(torch.float32, 32), (torch.bfloat16, 16), (torch.bfloat16, 32), (torch.bfloat16, 64)])
@pytest.mark.parametrize("masked", [-np.inf, -3.3e38, -1e30])
def test_biases_that_mask(sp, dtype, block, masked):
    nb, B, H = 5, 1, 2
    L = nb * block
    table = _table(32, H, dtype, 7)
    table[16:, 0] = masked      # keys ahead: one head attends backwards only
    table[:, 1] = masked        # the other to nothing
    if masked == -1e30:
        table[table < -1e29] = -1.01e30   # (-1e30 itself is no bf16 number)
    buckets = sp.relative_buckets(L, 32, 40, device="cuda")
    fl = np.ones((nb, nb), dtype=np.uint8)
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, dtype, 8)
    got = _run(sp, q, k, v, do, pat, table, buckets=buckets, dropout=0.2, rng=_rng())
    want, lse = _formula(q, k, v, do, _kept(fl, block), table, buckets.map, None, 0.2, RNG, 0)
    assert torch.isinf(lse[:, 1]).all()
    _near(got, want, TOL[dtype])
    for name in ("o", "dq", "dk", "dv"):
        assert not got[name][:, 1].any()
    assert not got["dtable"][:, 1].any() and not got["dtable"][17:, 0].any()


@pytest.mark.parametrize("dtype,block", [(torch.float32, 16), (torch.bfloat16, 32), (torch.bfloat16, 64)])
@pytest.mark.parametrize("length", [0, 1, 2])
def test_sequences_of_no_and_one_token(sp, dtype, block, length):
    nb, B, H = 2, 2, 2
    L = nb * block
    fl = np.ones((nb, nb), dtype=np.uint8)
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, dtype, 9)
    lengths = torch.full((B,), length, dtype=torch.int32, device="cuda")
    table, buckets = _table(8, H, dtype, 10), sp.relative_buckets(L, 8, 16, device="cuda")
    want, _ = _formula(q, k, v, do, _kept(fl, block), table, buckets.map, lengths, 0.0, RNG, 0)
    _near(_run(sp, q, k, v, do, pat, table, buckets=buckets, lengths=lengths), want, TOL[dtype])
    # outside 0 .. L they count as the ends
    for n, same in ((-7, 0), (L + 9, L)):
        a, b = [_run(sp, q, k, v, do, pat, table, buckets=buckets, lengths=torch.full((B,), m, dtype=torch.int32, device="cuda")) for m in (n, same)]
        assert all(torch.equal(a[x], b[x]) for x in a)


@pytest.mark.parametrize("dtype,block", [(torch.float32, 16), (torch.bfloat16, 64)])
def test_a_pattern_that_keeps_nothing(sp, dtype, block):
    pat = _pattern_from_mask(sp, np.zeros((3, 3), dtype=np.uint8), block)
    q, k, v, do = _inputs(1, 2, 3 * block, dtype, 11)
    got = _run(sp, q, k, v, do, pat, _table(32, 2, dtype, 1), buckets=sp.relative_buckets(3 * block, device="cuda"), dropout=0.5, rng=_rng())
    assert all(not t.any() for t in got.values())


@pytest.mark.parametrize("dtype,block", [(torch.float32, 32), (torch.bfloat16, 32), (torch.bfloat16, 64)])
@pytest.mark.parametrize("p", [2.0 ** -16, 0.5, 1 - 2.0 ** -16])
def test_probabilities_of_dropout(sp, dtype, block, p):
    nb, B, H = 3, 1, 3
    L = nb * block
    fl = np.ones((nb, nb), dtype=np.uint8)
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, dtype, 12)
    rng = (3, 4)
    got = _run(sp, q, k, v, do, pat, dropout=p, rng=_rng(rng), stream=M32)
    want, _ = _formula(q, k, v, do, _kept(fl, block), None, None, None, p, rng, M32)
    _near(got, want, TOL[dtype])


def test_a_probability_that_rounds_to_none(sp):
    block, L = 32, 96
    pat = _pattern_from_mask(sp, np.ones((3, 3), dtype=np.uint8), block)
    q, k, v, do = _inputs(1, 2, L, torch.bfloat16, 13)
    got, want = [_run(sp, q, k, v, do, pat, lengths=torch.full((1,), L, dtype=torch.int32, device="cuda"), **kw) for kw in (dict(dropout=2.0 ** -18), {})]
    assert all(torch.equal(got[n], want[n]) for n in got)


# The formula's gradient against differences of the kernel's own output in fp32, loss sum(O dO) along a direction: half a step h either way.
# The cubic term of a softmax whose scores move by h |x| is below (h |x|)^2 of the magnitudes, |x| at most 4 for the table and 8 for a score of
# q's (8 h)^2 / 6; a loss is exact to 256 u of its own magnitudes.
@pytest.mark.parametrize("of", ["table", "q", "k", "v"])
def test_gradients_against_differences(sp, of):
    block, nb, B, H = 16, 4, 2, 2
    L = nb * block
    fl = _mask(nb, seed=3)
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, torch.float32, 14)
    table, buckets = _table(16, H, torch.float32, 15), sp.relative_buckets(L, 16, 32, device="cuda")
    kw = dict(buckets=buckets, dropout=0.25, rng=_rng(), lengths=torch.tensor([L, 37], dtype=torch.int32, device="cuda"))
    got = _run(sp, q, k, v, do, pat, table, **kw)
    want, _ = _formula(q, k, v, do, _kept(fl, block), table, buckets.map, kw["lengths"], 0.25, RNG, 0)
    x = dict(table=table, q=q, k=k, v=v)[of]
    gen = torch.Generator(device="cuda").manual_seed(16)
    direction, h = torch.randn(x.shape, generator=gen, device="cuda").clamp(-4, 4), 2.0 ** -6

    def loss(step):
        args = dict(table=table, q=q, k=k, v=v)
        args[of] = x + step * direction
        o = sp.sparse_attention(args["q"], args["k"], args["v"], pat, bias=args["table"], **kw)
        return (o.double() * do.double()).sum().item()

    difference = (loss(h) - loss(-h)) / (2 * h)
    slope = (got["d" + of].double() * direction.double()).sum().item()
    magnitude = (want["d" + of][1] * direction.double().abs()).sum().item()
    loss_magnitude = (want["o"][1] * do.double().abs()).sum().item()
    assert abs(difference - slope) <= (8 * h) ** 2 / 6 * magnitude + TOL[torch.float32] * (magnitude + loss_magnitude / h)


@pytest.mark.parametrize("dtype,block", [(torch.float32, 16), (torch.bfloat16, 32), (torch.bfloat16, 64)])
def test_strides_alignment_and_shared_inputs(sp, dtype, block):
    nb, B, H = 3, 2, 2
    L = nb * block
    fl = _mask(nb, seed=1, density=0.8)
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, dtype, 17)
    table, buckets = _table(32, H, dtype, 18), sp.relative_buckets(2 * L, device="cuda")   # longer than the sequences
    kw = dict(buckets=buckets, dropout=0.1, rng=_rng())
    want = _run(sp, q, k, v, do, pat, table, **kw)
    odd = lambda t: torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)
    beside = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)
    for change in (odd, beside):
        got = _run(sp, change(q), change(k), change(v), change(do), pat, table.t().contiguous().t(), **kw)
        assert all(torch.equal(got[n], want[n]) for n in got)
    # one tensor for all three: its gradient is the sum
    x = q.clone().requires_grad_(True)
    sp.sparse_attention(x, x, x, pat, bias=table, **kw).backward(do)
    apart = _run(sp, q, q, q, do, pat, table, **kw)
    total = sum(apart[n].double() for n in ("dq", "dk", "dv"))
    mag = sum(apart[n].double().abs() for n in ("dq", "dk", "dv"))
    assert ((x.grad.double() - total).abs() <= 2 * torch.finfo(dtype).eps / 2 * mag).all()
    # a gradient that is the same number everywhere has strides of 0
    ones, expanded = [_run(sp, q, k, v, g, pat, table, **kw) for g in (torch.ones_like(do), torch.ones((), device="cuda", dtype=dtype).expand_as(do))]
    assert all(torch.equal(ones[n], expanded[n]) for n in ones)


def test_only_what_is_asked_for(sp):
    """A frozen table, frozen inputs, no gradients at all."""
    block, nb, H = 32, 3, 2
    L = nb * block
    pat = _pattern_from_mask(sp, np.ones((nb, nb), dtype=np.uint8), block)
    q, k, v, do = _inputs(2, H, L, torch.bfloat16, 19)
    table, buckets = _table(32, H, torch.float32, 20), sp.relative_buckets(L, device="cuda")   # a table of another type than the tensors
    kw = dict(buckets=buckets, dropout=0.1, rng=_rng())
    want = _run(sp, q, k, v, do, pat, table, **kw)
    assert want["dtable"].dtype == torch.float32
    # without gradients the probabilities are rounded to bf16, as summands (u = 2^-8 of each) and in their sum (u), with
    # gradients not, and either output is rounded (2 u): within 4 u of the magnitudes
    with torch.no_grad():
        o = sp.sparse_attention(q, k, v, pat, bias=table, **kw)
    exact, _ = _formula(q, k, v, do, torch.ones((L, L), dtype=torch.bool, device="cuda"), table, buckets.map, None, 0.1, RNG, 0)
    assert ((o.double() - want["o"].double()).abs() <= 4 * 2.0 ** -8 * exact["o"][1]).all()
    a = q.clone().requires_grad_(True)
    o = sp.sparse_attention(a, k, v, pat, bias=table, **kw)
    assert torch.equal(torch.autograd.grad(o, a, do)[0], want["dq"])
    t = table.clone().requires_grad_(True)
    o = sp.sparse_attention(q, k, v, pat, bias=t, **kw)
    assert torch.equal(torch.autograd.grad(o, t, do, retain_graph=True)[0], want["dtable"])
    assert torch.equal(torch.autograd.grad(o, t, do)[0], want["dtable"])
    with pytest.raises(RuntimeError):   # what was saved is gone
        torch.autograd.grad(o, t, do)


def test_rng_is_read_when_the_kernels_run(sp):
    """The backward pass has the values of its forward pass, whatever the program writes in between."""
    block, nb, H = 64, 2, 2
    L = nb * block
    pat = _pattern_from_mask(sp, np.ones((nb, nb), dtype=np.uint8), block)
    q, k, v, do = _inputs(1, H, L, torch.bfloat16, 21)
    rng = _rng((1, 2))
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
    x = q.clone().requires_grad_(True)
    o, y = sp.sparse_attention(*leaves, pat, dropout=0.5, rng=rng), sp.dropout_add(x, None, 0.5, rng)
    rng.copy_(_rng((8, 9)))
    grads, dx = torch.autograd.grad(o, leaves, do), torch.autograd.grad(y, x, do)[0]
    want = _run(sp, q, k, v, do, pat, dropout=0.5, rng=_rng((1, 2)))
    assert all(torch.equal(a, b) for a, b in zip((o, *grads), want.values()))
    assert torch.equal(dx, sp.dropout_add(do, None, 0.5, _rng((1, 2))))
    assert not torch.equal(_run(sp, q, k, v, do, pat, dropout=0.5, rng=rng)["o"], o)


@pytest.mark.parametrize("dtype,block", [(torch.float32, 16), (torch.bfloat16, 32), (torch.bfloat16, 64)])
def test_graphs_and_another_stream(sp, dtype, block):
    """Two captured steps replayed in turn, eager work between them, each replay against the eager result of its rng."""
    nb, B, H = 40, 1, 1   # rows that are cut: forward and backward have workspaces
    L = nb * block
    fl = _mask(nb, seed=2, density=0.9)
    pat = _pattern_from_mask(sp, fl, block)
    table, buckets = _table(32, H, dtype, 22), sp.relative_buckets(L, device="cuda")
    sets = [_inputs(B, H, L, dtype, 23 + i) for i in range(2)]
    rng = _rng((1, 0))
    step = lambda s: _run(sp, *s, pat, table, buckets=buckets, dropout=0.2, rng=rng)
    for s in sets:
        step(s)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step(s)
        graphs.append(g)
        outs.append(out)
    for i in range(4):
        rng.copy_(_rng((1, i)))
        for g, out, s in zip(graphs, outs, sets):
            want = step(s)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(out[n], want[n]) for n in want), i
        for g in graphs:   # both without anything between
            g.replay()
        for out, s in zip(outs, sets):
            want = step(s)
            assert all(torch.equal(out[n], want[n]) for n in want), i
    side = torch.cuda.Stream()
    want = step(sets[0])
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(sets[0])
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_rows_whose_addresses_pass_32_bits(sp):
    """As many heads as have their last rows beyond 2^32 bytes, each sequence of the longest length."""
    block, L, H, dtype = 64, 65536, 520, torch.bfloat16
    nb = L // block
    fl = np.eye(nb, dtype=np.uint8)
    fl[-1, :8] = 1
    pat = _pattern_from_mask(sp, fl, block)
    gen = torch.Generator(device="cuda").manual_seed(25)
    q, k, v, do = [torch.empty((1, H, L, 64), device="cuda", dtype=dtype).normal_(generator=gen) for _ in range(4)]
    table, buckets = _table(32, H, dtype, 26), sp.relative_buckets(L, device="cuda")
    lengths = torch.full((1,), L - 1, dtype=torch.int32, device="cuda")
    got = _run(sp, q, k, v, do, pat, table, buckets=buckets, lengths=lengths)
    last = [t[:, -1:].contiguous() for t in (q, k, v, do)]
    del q, k, v, do
    want = _run(sp, *last, pat, table[:, -1:].contiguous(), buckets=buckets, lengths=lengths)
    for n in ("o", "dq", "dk", "dv"):   # the few long rows may be cut differently: sums in another order, then rounded
        a, b = got[n][:, -1:].double(), want[n].double()
        assert (a - b).norm() <= 2.0 ** -8 * b.norm(), n
    a, b = got["dtable"][:, -1:].double(), want["dtable"].double()
    assert (a - b).norm() <= 2.0 ** -7 * b.norm()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,q_len,k_len,q_start", [(1, 1, 1, 0), (3, 1, 7, 5), (8, 1, 1000, 999), (5, 300, 1, 0), (2, 17, 8, 100), (3, 257, 511, 0),
                                                   (1, 129, 2049, 4), (2, 1000, 77, 3), (600, 3, 5, 0), (2, 700, 520, 0)])
def test_dense_bias(sp, dtype, H, q_len, k_len, q_start):
    b = sp.relative_buckets(max(q_start + q_len, k_len) + 2, 32, 300, device="cuda")
    table = _table(32, H, dtype, 27).requires_grad_(True)
    out = sp.relative_bias(table, b, q_len, k_len, q_start)
    i, j = torch.arange(q_len, device="cuda")[:, None] + q_start, torch.arange(k_len, device="cuda")[None]
    of = b.map[j - i + b.length - 1].long()
    assert torch.equal(out, table.detach()[of].permute(2, 0, 1))
    gen = torch.Generator(device="cuda").manual_seed(28)
    for g in (torch.randn(out.shape, generator=gen, device="cuda").to(dtype), torch.ones((), device="cuda", dtype=dtype).expand_as(out),
              torch.cat([out.new_ones(1), torch.randn(out.shape, generator=gen, device="cuda").to(dtype).flatten()])[1:].view(out.shape)):
        got, = torch.autograd.grad(out, table, g, retain_graph=True)
        sums = [torch.zeros(table.shape, dtype=torch.float64, device="cuda").index_add_(0, of.reshape(-1), m.permute(1, 2, 0).reshape(-1, H))
                for m in (g.double(), g.double().abs())]
        # sums of up to a million fp32 terms in pieces, then one rounding
        assert ((got.double() - sums[0]).abs() <= torch.finfo(dtype).eps / 2 * sums[0].abs() + 2.0 ** -16 * sums[1]).all()
        assert torch.equal(got, torch.autograd.grad(out, table, g, retain_graph=True)[0])


@pytest.mark.parametrize("count", [1, 65, 256])
def test_dense_bias_of_any_map(sp, count):
    gen = torch.Generator().manual_seed(count)
    b = sp.RelativeBuckets(90, count, torch.randint(0, min(count + 2, 256), (179,), generator=gen, dtype=torch.uint8).cuda())
    table = _table(count, 2, torch.float32, 29).requires_grad_(True)
    out = sp.relative_bias(table, b, 90, 90)
    i = torch.arange(90, device="cuda")
    of = b.map[i[None] - i[:, None] + 89].long().clamp_max(count - 1)
    assert torch.equal(out, table.detach()[of].permute(2, 0, 1))
    g = torch.randn(out.shape, device="cuda")
    got, = torch.autograd.grad(out, table, g)
    want, mag = [torch.zeros(table.shape, dtype=torch.float64, device="cuda").index_add_(0, of.reshape(-1), m.permute(1, 2, 0).reshape(-1, 2))
                 for m in (g.double(), g.double().abs())]
    assert ((got.double() - want).abs() <= 2.0 ** -16 * mag).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 1023, 5000, 100003])
@pytest.mark.parametrize("p,residual,odd", [(0.1, True, False), (0.5, False, False), (0.0, True, True), (1 - 2.0 ** -16, True, True), (0.1, True, True)])
def test_dropout_add(sp, dtype, n, p, residual, odd):
    gen = torch.Generator(device="cuda").manual_seed(n)
    x, r, dy = [torch.randn(n + 1, generator=gen, device="cuda").to(dtype)[1 if odd else 0:][:n].detach() for _ in range(3)]
    x.requires_grad_(True)
    r.requires_grad_(True)
    y = sp.dropout_add(x, r if residual else None, p, _rng(), 3)
    f = _flat_factors(torch.arange(n, device="cuda"), p, RNG, 3)
    exact = x.detach().double() * f + (r.detach().double() if residual else 0)
    mag = (x.detach().double() * f).abs() + r.detach().double().abs()
    u = torch.finfo(dtype).eps / 2
    assert ((y.double() - exact).abs() <= u * exact.abs() + 2.0 ** -22 * mag).all()
    grads = torch.autograd.grad(y, [x, r] if residual else [x], dy)
    exact = dy.double() * f
    assert ((grads[0].double() - exact).abs() <= (u + 2.0 ** -22) * exact.abs()).all()
    if residual:
        assert torch.equal(grads[1], dy)
    # not finite where nothing is kept, or kept
    bad = x.detach().clone()
    bad[0] = float("inf")
    y = sp.dropout_add(bad, None, p, _rng(), 3)
    assert torch.isinf(y[0]) if f[0] > 0 else y[0] == 0


def test_dropout_add_of_nothing_and_of_views(sp):
    x = torch.zeros((0, 5), device="cuda", requires_grad=True)
    y = sp.dropout_add(x, x, 0.5, _rng())
    assert y.shape == x.shape and torch.autograd.grad(y.sum(), x)[0].shape == x.shape
    a, b = torch.randn((2, 33, 17), device="cuda")
    assert torch.equal(sp.dropout_add(a.t(), b.t(), 0.3, _rng()), sp.dropout_add(a.t().contiguous(), b.t().contiguous(), 0.3, _rng()))
    leaf = torch.randn(40, device="cuda", requires_grad=True)   # the same tensor twice
    g, = torch.autograd.grad(sp.dropout_add(leaf, leaf, 0.5, _rng()), leaf, torch.ones(40, device="cuda"))
    assert torch.equal(g, (1 + _flat_factors(torch.arange(40, device="cuda"), 0.5, RNG, 0)).float())


def test_dropout_add_past_32_bits(sp):
    n = 2 ** 32 + 2 ** 10 + 5
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    y = sp.dropout_add(x, x, 0.5, _rng())
    for at in (0, 2 ** 31 - 100, 2 ** 32 - 100, n - 200):
        f = _flat_factors(torch.arange(at, at + 200, device="cuda"), 0.5, RNG, 0)
        assert torch.equal(y[at:at + 200].double(), 1 + f)


@pytest.mark.parametrize("dtype,block", [(torch.float32, 32), (torch.bfloat16, 16), (torch.bfloat16, 64)])
def test_entries_of_the_c_abi(sp, dtype, block):
    """The calls themselves, with workspaces of their sizes that hold anything: the same bits as the nodes; and without o_rest."""
    nb, B, H = 34, 1, 2
    L = nb * block
    fl = _mask(nb, seed=8, density=0.8)
    pat = _pattern_from_mask(sp, fl, block)
    q, k, v, do = _inputs(B, H, L, dtype, 70)
    table, buckets, rng = _table(32, H, dtype, 71), sp.relative_buckets(L, device="cuda"), _rng()
    lengths = torch.full((B,), L - 9, dtype=torch.int32, device="cuda")
    want = _run(sp, q, k, v, do, pat, table, buckets=buckets, lengths=lengths, dropout=0.1, rng=rng, stream=3)
    formula, _ = _formula(q, k, v, do, _kept(fl, block), table, buckets.map, lengths, 0.1, RNG, 3)
    code = sp.SPION_F32 if dtype == torch.float32 else sp.SPION_BF16
    shape = dict(B=B, H=H, L=L, d=64, block=block, dtype=code)
    room = lambda n: torch.full((max(n, 256),), 0xa5, dtype=torch.uint8, device="cuda")
    for rest in (torch.empty_like(q), None):
        kw = dict(table=table, bucket_of=buckets.map, lengths=lengths, dropout=0.1)
        sizes = [sp.spion_attn_with_workspace_bytes(**shape, nnzb=pat.nnzb, is_bwd=b, rng=rng, **kw) for b in (False, True)]
        got = {n: torch.full_like(table if n == "dtable" else q, float("nan")) for n in ("o", "dq", "dk", "dv", "dtable")}
        lse, used = torch.empty((B, H, L), device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
        sp.spion_attn_fwd_with(q, k, v, got["o"], lse, pat.row_ptr, pat.col_idx, pat.nnzb, **shape, rng=rng, rng_used=used, dropout_stream=3,
                               workspace=room(sizes[0]), o_rest=rest, **kw)
        assert torch.equal(used, rng)
        sp.spion_attn_bwd_with(q, k, v, got["o"], do, lse, got["dq"], got["dk"], got["dv"], got["dtable"], pat.row_ptr, pat.col_idx, pat.col_ptr,
                               pat.row_idx, pat.bsr_pos, pat.nnzb, **shape, rng=used, dropout_stream=3, workspace=room(sizes[1]), o_rest=rest, **kw)
        if rest is not None:
            assert all(torch.equal(got[n], want[n]) for n in want)
        _near(got, formula, TOL[dtype])
    bias = torch.empty((H, 70, L), dtype=dtype, device="cuda")
    sp.spion_relative_bias(table, buckets.map, bias, L, 32, H, 70, L, 5, code)
    t = table.clone().requires_grad_(True)
    node = sp.relative_bias(t, buckets, 70, L, 5)
    g, dtable = torch.randn_like(bias), torch.empty_like(table)
    sp.spion_relative_bias_grad(g, buckets.map, dtable, L, 32, H, 70, L, 5, code, room(sp.spion_relative_bias_workspace_bytes(32, H, 70, L)))
    assert torch.equal(bias, node) and torch.equal(dtable, torch.autograd.grad(node, t, g)[0])
    y, used = torch.empty_like(q), torch.zeros(2, dtype=torch.int64, device="cuda")
    sp.spion_dropout_add(q, k, y, q.numel(), code, 0.2, rng, used, 7)
    assert torch.equal(y, sp.dropout_add(q, k, 0.2, rng, 7)) and torch.equal(used, rng)


def test_calls_that_are_refused(sp):
    block, nb, H = 32, 2, 2
    L = nb * block
    pat = _pattern_from_mask(sp, np.ones((nb, nb), dtype=np.uint8), block)
    q, k, v, do = _inputs(2, H, L, torch.bfloat16, 30)
    table, buckets, rng = _table(32, H, torch.bfloat16, 31), sp.relative_buckets(L, device="cuda"), _rng()
    lengths = torch.full((2,), L, dtype=torch.int32, device="cuda")
    call = lambda *a, **kw: (lambda: sp.sparse_attention(*(a or (q, k, v)), pat, **kw))
    for f in (call(bias=table), call(bias=table[:31], buckets=buckets), call(bias=table[:, :1], buckets=buckets), call(bias=table.half(), buckets=buckets),
              call(bias=table, buckets=sp.relative_buckets(L - 1, device="cuda")), call(bias=table, buckets=sp.relative_buckets(L)),
              call(lengths=lengths.long()), call(lengths=lengths[:1]), call(lengths=lengths.cpu()), call(dropout=0.1), call(dropout=1.0, rng=rng),
              call(dropout=-0.5, rng=rng), call(dropout=float("nan"), rng=rng), call(dropout=0.1, rng=rng.int()), call(dropout=0.1, rng=rng[:1]),
              call(dropout=0.1, rng=rng.cpu()), call(dropout=0.1, rng=rng, stream=-1), call(dropout=0.1, rng=rng, stream=2 ** 32),
              call(lengths=lengths, flags=sp.SPION_ATTN_PAPER_DENOM), call(q, k[:1], v, lengths=lengths), call(q, k, v.float(), lengths=lengths),
              call(q.half(), k.half(), v.half(), lengths=lengths), call(q[0], k[0], v[0], lengths=lengths),
              lambda: sp.relative_bias(table, buckets, L + 1, L), lambda: sp.relative_bias(table, buckets, L, L, 1), lambda: sp.relative_bias(table, buckets, 0, L),
              lambda: sp.relative_bias(table, buckets, 1, L, -1), lambda: sp.relative_bias(table[0], buckets, L, L), lambda: sp.relative_bias(table.half(), buckets, L, L),
              lambda: sp.dropout_add(q, k[:1], 0.1, rng), lambda: sp.dropout_add(q, k.float(), 0.1, rng), lambda: sp.dropout_add(q.half(), None, 0.1, rng),
              lambda: sp.dropout_add(q, None, 1.0, rng), lambda: sp.dropout_add(q, None, 0.1, None), lambda: sp.dropout_add(q, None, 0.1, rng, 2 ** 32)):
        with pytest.raises(ValueError):
            f()
    longer = _inputs(2, H, L + block, torch.bfloat16, 40, 3)   # than the pattern
    uncounted = sp.Pattern(**{**vars(pat), "nnzb": -1})
    for a, p in ((longer, pat), ((q[:, :, :block], k[:, :, :block], v[:, :, :block]), pat), ((q, k, v), uncounted)):
        with pytest.raises(ValueError):
            sp.sparse_attention(*a, p, lengths=lengths)
    mha = sp.SparseMHA(64 * H, H, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        mha(torch.zeros(2, L + block, 64 * H, device="cuda", dtype=torch.bfloat16), pat, lengths=lengths)
    with pytest.raises(sp.SpionError):
        sp.sparse_attention(q[..., :32], k[..., :32], v[..., :32], pat, lengths=lengths)
    leaf = q.float().requires_grad_(True)
    for f in (lambda x: sp.sparse_attention(x, k.float(), v.float(), pat, lengths=lengths), lambda x: sp.dropout_add(x, None, 0.1, rng)):
        g, = torch.autograd.grad(f(leaf).square().sum(), leaf)
        with pytest.raises(NotImplementedError):
            torch.autograd.grad(f(leaf).square().sum(), leaf, create_graph=True)
        with pytest.raises(NotImplementedError):
            torch.func.vmap(f)(leaf[None])
        with pytest.raises(NotImplementedError), torch.autograd.forward_ad.dual_level():
            f(torch.autograd.forward_ad.make_dual(leaf.detach(), leaf.detach()))
        with pytest.raises(NotImplementedError):
            torch.jit.trace(f, leaf, check_trace=False)


def test_saved_tensors_are_looked_at(sp):
    block, nb, H = 32, 2, 2
    L = nb * block
    pat = _pattern_from_mask(sp, np.ones((nb, nb), dtype=np.uint8), block)
    q, k, v, do = _inputs(2, H, L, torch.bfloat16, 32)
    table, buckets = _table(32, H, torch.bfloat16, 33), sp.relative_buckets(L, device="cuda")
    kw = dict(buckets=buckets, lengths=torch.full((2,), L, dtype=torch.int32, device="cuda"), dropout=0.1, rng=_rng())
    shapes = set()
    with torch.autograd.graph.saved_tensors_hooks(lambda t: shapes.add(t.shape) or t, lambda t: t):
        sp.sparse_attention(*[t.clone().requires_grad_(True) for t in (q, k, v)], pat, bias=table.clone().requires_grad_(True), **kw)
    assert {q.shape, table.shape, kw["lengths"].shape} < shapes
    for shape in shapes:   # each kind once: less of it than was saved
        leaves = [t.clone().requires_grad_(True) for t in (q, k, v, table)]
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t[:1] if t.shape == shape else t):
            o = sp.sparse_attention(*leaves[:3], pat, bias=leaves[3], **kw)
            with pytest.raises(ValueError):
                torch.autograd.grad(o, leaves, do)
    for i in range(4):     # and changed in place
        leaves = [t.clone().requires_grad_(True) for t in (q, k, v, table)]
        moved = [t * 1 for t in leaves]
        o = sp.sparse_attention(*moved[:3], pat, bias=moved[3], **kw)
        with torch.no_grad():
            moved[i].add_(1)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(o, leaves, do)


def _sub_layer(mha, E, kept, buckets, lengths, rng, stream, dtype):
    """Algorithm 5 with everything, in torch's operators; probabilities and products in fp64."""
    B, L, D = E.shape
    H = mha.heads
    X = torch.nn.functional.layer_norm(E, (D,), mha.norm.weight, mha.norm.bias, mha.norm.eps)
    qkv = torch.nn.functional.linear(X, mha.w_qkv.weight).view(B, L, 3, H, 64)
    q, k, v = [qkv[:, :, i].transpose(1, 2).double().contiguous() for i in range(3)]
    s = q @ k.transpose(-1, -2).contiguous() / 8.0
    pos = torch.arange(L, device="cuda")
    s = s + mha.bias_table.double()[buckets.map[pos[None] - pos[:, None] + buckets.length - 1].long()].permute(2, 0, 1)
    valid = pos[None] < lengths[:, None]
    seen = kept & valid[:, None, None, :] & valid[:, None, :, None]
    s = s.masked_fill(~seen, -1e300)
    P = torch.softmax(s, -1) * seen
    if mha.training and mha.attn_dropout:
        P = P * _score_factors(B * H, L, mha.attn_dropout, rng, stream).view(P.shape)
    S = (P @ v).to(dtype).transpose(1, 2).reshape(B, L, D)
    y = torch.nn.functional.linear(S, mha.w_o.weight)
    if mha.training and mha.drop.p:
        y = (y.double() * _flat_factors(torch.arange(y.numel(), device="cuda"), mha.drop.p, rng, stream).view(y.shape)).to(dtype)
    return y + E


# bf16 and blocks of 32 and 64: on the heads where the projection has them; the others after a split
@pytest.mark.parametrize("dtype,block", [(torch.float32, 16), (torch.bfloat16, 16), (torch.bfloat16, 32), (torch.bfloat16, 64)])
@pytest.mark.parametrize("training", [True, False])
def test_all_of_them_in_the_sub_layer(sp, dtype, block, training):
    nb, B, H, stream = 4, 2, 3, 6
    L = nb * block
    fl = _mask(nb, seed=4, density=0.8)
    pat = _pattern_from_mask(sp, fl, block)
    buckets = sp.relative_buckets(L + 10, device="cuda")
    torch.manual_seed(34)
    mha = sp.SparseMHA(64 * H, H, dropout=0.2, device="cuda", dtype=dtype, buckets=buckets, attn_dropout=0.1).train(training)
    with torch.no_grad():
        mha.bias_table.normal_()
    E = torch.randn(B, L, 64 * H, device="cuda", dtype=dtype, requires_grad=True)
    dO = torch.randn_like(E)
    lengths = torch.tensor([L - 7, block + 1], dtype=torch.int32, device="cuda")
    leaves = [E, *mha.parameters()]
    assert len(leaves) == 6
    rng = _rng()
    out = mha(E, pat, lengths=lengths, rng=rng, stream=stream)
    got = [out, *torch.autograd.grad(out, leaves, dO)]
    ref = _sub_layer(mha, E, _kept(fl, block), buckets, lengths, RNG, stream, dtype)
    want = [ref, *torch.autograd.grad(ref, leaves, dO)]
    tol = 1e-4 if dtype == torch.float32 else 3e-2   # as for the sub-layer without any of them
    for a, b in zip(got, want):
        assert torch.isfinite(a).all() and (a - b).double().norm() < tol * b.double().norm()
    assert torch.equal(out, mha(E, pat, lengths=lengths, rng=rng, stream=stream))
    assert torch.equal(out, mha(E, pat, lengths=lengths, rng=_rng((RNG[0], RNG[1] + 1)), stream=stream)) == (not training)


def test_sub_layer_without_the_state_to_draw_from(sp):
    pat = _pattern_from_mask(sp, np.ones((2, 2), dtype=np.uint8), 32)
    mha = sp.SparseMHA(128, 2, dropout=0.5, device="cuda", dtype=torch.bfloat16, attn_dropout=0.1)
    E = torch.randn(1, 64, 128, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        mha(E, pat)
    mha.attn_dropout = 0.0
    assert mha(E, pat).shape == E.shape   # torch's dropout, as before
    mha.eval()
    mha.attn_dropout = 0.1
    plain = sp.SparseMHA(128, 2, device="cuda", dtype=torch.bfloat16)
    plain.load_state_dict(mha.state_dict())
    assert torch.equal(mha(E, pat), plain(E, pat))


def test_sub_layer_under_autocast(sp):
    """fp32 weights, products in bf16: the attention's heads in bf16, the residual in fp32."""
    pat = _pattern_from_mask(sp, np.ones((2, 2), dtype=np.uint8), 32)
    mha = sp.SparseMHA(128, 2, dropout=0.3, device="cuda", buckets=sp.relative_buckets(64, device="cuda"), attn_dropout=0.1)
    E = torch.randn(2, 64, 128, device="cuda", requires_grad=True)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        out = mha(E, pat, rng=_rng())
    whole = mha(E, pat, rng=_rng())
    assert out.dtype == torch.float32
    assert (out - whole).norm() <= 16 * 2.0 ** -8 * whole.norm()   # X, qkv, P, S, the products and their weights: fewer than 16 roundings
    assert all(torch.isfinite(g).all() for g in torch.autograd.grad(out.square().sum(), [E, *mha.parameters()]))


def test_sub_layer_whose_projection_is_watched(sp):
    """A hook that changes the projections' tensors in place, after the attention has saved them."""
    pat = _pattern_from_mask(sp, np.ones((2, 2), dtype=np.uint8), 64)
    mha = sp.SparseMHA(128, 2, device="cuda", dtype=torch.bfloat16, buckets=sp.relative_buckets(128, device="cuda"))
    E = torch.randn(1, 128, 128, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    dO = torch.randn_like(E)
    want = torch.autograd.grad(mha(E, pat), [E, *mha.parameters()], dO)
    handle = mha.w_o.register_forward_pre_hook(lambda m, a: None)
    got = torch.autograd.grad(mha(E, pat), [E, *mha.parameters()], dO)
    handle.remove()
    for a, b in zip(got, want):
        assert (a - b).float().norm() <= 2.0 ** -7 * b.float().norm()


def test_sub_layer_step_in_a_graph(sp):
    """A training step, dropout's offset moved on inside it: every replay draws anew, as the eager step of that offset does."""
    block, nb, B, H = 32, 4, 2, 2
    L = nb * block
    pat = _pattern_from_mask(sp, _mask(nb, seed=5, density=0.8), block)
    torch.manual_seed(35)
    mha = sp.SparseMHA(64 * H, H, dropout=0.2, device="cuda", dtype=torch.bfloat16, buckets=sp.relative_buckets(L, device="cuda"), attn_dropout=0.1)
    E, dO = torch.randn(2, B, L, 64 * H, device="cuda", dtype=torch.bfloat16)
    lengths = torch.tensor([L, L - 9], dtype=torch.int32, device="cuda")
    rng, one = _rng((5, 0)), torch.tensor([0, 1], dtype=torch.int64, device="cuda")

    def step():
        rng.add_(one)
        out = mha(E, pat, lengths=lengths, rng=rng, stream=1)
        return (out.detach(), *torch.autograd.grad(out, list(mha.parameters()), dO))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = step()
    seen = []
    for i in range(4):
        rng.copy_(_rng((5, 10 + i)))
        want = step()
        rng.copy_(_rng((5, 10 + i)))
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, want):   # (a library's product may be another one under capture)
            assert (a - b).float().norm() <= 2.0 ** -7 * b.float().norm()
        seen.append(want[0])
    assert not torch.equal(seen[0], seen[1])


def test_dense_phase_and_sparse_phase_agree(sp):
    """The dense attention that precedes a pattern, with the dense bias, and the sparse one on a pattern that keeps everything:
    outputs, and one table's gradient through both."""
    block, nb, B, H = 32, 5, 2, 2
    L = nb * block
    pat = _pattern_from_mask(sp, np.ones((nb, nb), dtype=np.uint8), block)
    q, k, v, do = _inputs(B, H, L, torch.float32, 36)
    buckets = sp.relative_buckets(L, device="cuda")
    table = _table(32, H, torch.float32, 37).requires_grad_(True)
    dense = torch.softmax(q @ k.transpose(-1, -2).contiguous() / 8.0 + sp.relative_bias(table, buckets, L, L), -1) @ v
    sparse = sp.sparse_attention(q, k, v, pat, bias=table, buckets=buckets)
    want, _ = _formula(q, k, v, do, torch.ones((L, L), dtype=torch.bool, device="cuda"), table.detach(), buckets.map, None, 0.0, RNG, 0)
    for o in (dense, sparse):
        _near({"o": o.detach(), "dtable": torch.autograd.grad(o, table, do)[0]}, {n: want[n] for n in ("o", "dtable")}, TOL[torch.float32])
    # a single query of it, as it is asked for when tokens come one by one
    row = sp.relative_bias(table, buckets, 1, L, L - 1)
    one = torch.softmax(q[:, :, -1:] @ k.transpose(-1, -2).contiguous() / 8.0 + row, -1) @ v
    _near({"o": one.detach()}, {"o": tuple(t[:, :, -1:] for t in want["o"])}, TOL[torch.float32])
