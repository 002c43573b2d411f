"""Operators of the attention sub-layer beside its plain sparse attention, as named cases with inputs, one pass, its
outputs and what they should be.

Three kinds of case:
  attn     block-sparse attention with a learned relative position bias (by buckets of key - query), dropout of the
           probabilities and sequences shorter than the batch's length: a training step (forward, and the gradients of Q, K, V
           and of the bias table) or a forward pass alone
  bias     the same bias as a dense [H, Lq, Lk] tensor, for the dense-attention phase that precedes a pattern and for single
           query rows: forward, or forward and the table's gradient
  dropout  the end of the sub-layer: residual + dropout(x), forward and backward

Dropout: the 16-bit draw of an element is a function of seed, offset, stream and the element's place alone (Philox4x32
with 7 rounds), and an element is dropped if its draw is below rint(65536 p).

Sizes are those of the configurations of `spion_inputs.py`, of the tests, and in between; `draw` spreads over the same ranges.
"""
import math

import numpy as np
import torch

own = False

HEAD_DIM = 64
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _attn(name, dtype, B, H, L, block, density, bias=True, buckets=32, max_distance=128, both_sides=True, dropout=0.1,
          ragged=False, backward=True):
    return dict(name=name, kind="attn", dtype=dtype, B=B, H=H, L=L, block=block, density=density, bias=bias,
                buckets=buckets, max_distance=max_distance, both_sides=both_sides, dropout=dropout, ragged=ragged,
                backward=backward)


def _bias(name, dtype, H, q_len, k_len, q_start, buckets=32, max_distance=128, both_sides=True, backward=True):
    return dict(name=name, kind="bias", dtype=dtype, H=H, q_len=q_len, k_len=k_len, q_start=q_start, buckets=buckets,
                max_distance=max_distance, both_sides=both_sides, backward=backward)


def _dropout(name, dtype, B, L, D, dropout=0.1, residual=True, backward=True):
    return dict(name=name, kind="dropout", dtype=dtype, B=B, L=L, D=D, dropout=dropout, residual=residual, backward=backward)


def listed():
    return [
        # configuration 1: one small fp32 head, everything at once; call overhead and launches
        _attn("attn_tiny_f32_step", "f32", 1, 1, 256, 16, 0.074),
        # configuration 2: many short sequences of different lengths, the bias alone
        _attn("attn_cfg2_step", "bf16", 16, 4, 1024, 32, 0.15, dropout=0.0, ragged=True),
        # configuration 4, the one the benchmark quotes: bias and dropout
        _attn("attn_cfg4_step", "bf16", 4, 4, 4096, 64, 0.08),
        # configuration 5, the densest of its four layers, padded
        _attn("attn_cfg5_dense_step", "bf16", 4, 8, 4096, 64, 0.208, ragged=True),
        # full-precision training at the shape of configuration 3, more and wider buckets
        _attn("attn_f32_step", "f32", 2, 4, 2048, 32, 0.10, buckets=64, max_distance=512),
        # fine blocks, odd batch, head and block counts: dropout without a bias, padded
        _attn("attn_b16_step", "bf16", 3, 3, 1936, 16, 0.08, bias=False, dropout=0.2, ragged=True),
        # inference on long documents: forward only, 255 block rows
        _attn("attn_long_fwd", "bf16", 2, 8, 16320, 64, 0.05, dropout=0.0, ragged=True, backward=False),
        # the bias of one query row against a long context
        _bias("bias_row_fwd", "bf16", 8, 1, 4097, 4096, both_sides=False, backward=False),
        # the dense phase of configuration 5: the bias of eight heads and its table's gradient
        _bias("bias_dense_step", "bf16", 8, 4096, 4096, 0),
        # the dropout at the end of a small fp32 sub-layer, an odd number of elements
        _dropout("dropout_small_step", "f32", 1, 255, 63),
        # the end of the sub-layer at the shape of configuration 3
        _dropout("dropout_cfg3_step", "bf16", 8, 2048, 256),
        # the same for a large batch of long sequences
        _dropout("dropout_large_step", "bf16", 16, 16384, 512),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _draw_buckets(rng):
    both = rng.random() < 0.7
    buckets = 2 * int(round(_log_uniform(rng, 4, 128)))
    exact = (buckets // 2 if both else buckets) // 2
    return dict(buckets=buckets, max_distance=exact + int(round(_log_uniform(rng, 1, 1024))), both_sides=both)


def draw(rng):
    kind = rng.choices(("attn", "bias", "dropout"), (4, 1, 1))[0]
    dtype = rng.choices(("bf16", "f32"), (3, 1))[0]
    if kind == "attn":
        block = rng.choice((16, 32, 32, 64, 64, 64))
        backward = rng.random() < 0.75
        # the products of the densest listed step; fp32 and block 16 have a slower path
        flops_max = 1.4e11 if dtype == "bf16" and block > 16 else 4e9
        while True:
            nb = int(round(_log_uniform(rng, 1, 256)))
            B = int(round(_log_uniform(rng, 1, 16)))
            H = rng.randint(1, 8)
            density = round(min(1.0, max(_log_uniform(rng, 0.03, 0.30), 1.0 / nb)), 4)
            dense = B * H * (nb * block) ** 2
            if density * dense * HEAD_DIM * (14 if backward else 4) <= flops_max and dense <= (5.5e8 if backward else 4.2e9):
                break
        bias = rng.random() < 0.75
        return dict(kind="attn", dtype=dtype, B=B, H=H, L=nb * block, block=block, density=density, bias=bias,
                    dropout=round(rng.uniform(0.01, 0.5), 4) if not bias or rng.random() < 0.6 else 0.0,
                    ragged=rng.random() < 0.5, backward=backward, **_draw_buckets(rng))
    if kind == "bias":
        while True:
            k_len = int(round(_log_uniform(rng, 1, 8192)))
            q_len = int(round(_log_uniform(rng, 1, 8192))) if rng.random() < 0.7 else 1
            H = rng.randint(1, 16)
            if H * q_len * k_len <= 2 ** 27:
                break
        return dict(kind="bias", dtype=dtype, H=H, q_len=q_len, k_len=k_len, q_start=rng.randint(0, 4096),
                    backward=rng.random() < 0.7, **_draw_buckets(rng))
    while True:
        B, L = int(round(_log_uniform(rng, 1, 16))), int(round(_log_uniform(rng, 1, 16384)))
        D = rng.choice((64 * rng.randint(1, 16), rng.randint(1, 1024)))
        if B * L * D <= 2 ** 26:
            break
    return dict(kind="dropout", dtype=dtype, B=B, L=L, D=D, dropout=round(rng.uniform(0.01, 0.6), 4),
                residual=rng.random() < 0.75, backward=rng.random() < 0.75)


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _kept(case):
    nb = case["L"] // case["block"]
    return min(nb * nb, max(nb, int(round(case["density"] * nb * nb))))


def _block_mask(nb, kept, seed):
    """A layer's block pattern with exactly `kept` blocks: the diagonal, part of a narrow band beside it, some columns
    kept over long runs of rows (vertical stripes), a row or two far longer than the rest, a little that is scattered."""
    rng = np.random.default_rng(seed)
    score = rng.random((nb, nb)) * 0.5
    i = np.arange(nb)
    for off in (-1, 1):
        near = i[(i + off >= 0) & (i + off < nb)]
        score[near, near + off] += 0.6 * rng.random(near.size)
    for col in rng.permutation(nb)[:max(1, nb // 8)]:
        start = int(rng.integers(0, nb))
        score[start:start + max(1, nb // 2), col] += 0.45
    for row in rng.permutation(nb)[:2]:
        score[row, rng.random(nb) < 0.5] += 0.4
    score[i, i] = 2.0
    mask = np.zeros(nb * nb, bool)
    mask[np.argsort(-score, axis=None, kind="stable")[:kept]] = True
    return mask.reshape(nb, nb)


def _bucket_starts(n, max_distance):
    """First distance of each of n buckets: the first half have one each, from `exact` on they grow geometrically up to
    max_distance (bucket exact + j starts at the smallest d with d >= exact (max_distance / exact)^(j / wide), found in
    integers); the last has everything beyond."""
    exact = n // 2
    wide = n - exact
    starts = list(range(exact))
    for j in range(wide):
        lo, hi = exact, max_distance
        while lo < hi:
            d = (lo + hi) // 2
            if d ** wide * exact ** j >= max_distance ** j * exact ** wide:
                hi = d
            else:
                lo = d + 1
        starts.append(lo)
    return starts


def _bucket_map(L, buckets, max_distance, both_sides):
    """Bucket of key - query for the distances -(L - 1) .. L - 1.  both_sides: keys behind and ahead of the query have half of
    the buckets each, else a key ahead of the query shares bucket 0 with its own position."""
    n = buckets // 2 if both_sides else buckets
    d = np.arange(-(L - 1), L)
    far = np.abs(d) if both_sides else np.maximum(-d, 0)
    bucket = np.searchsorted(np.asarray(_bucket_starts(n, max_distance)), far, side="right") - 1
    if both_sides:
        bucket = bucket + n * (d > 0)
    return torch.from_numpy(bucket.astype(np.int64))


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def prepare(case, seed):
    gen = _generator(seed)
    dtype = DTYPES[case["dtype"]]
    rng = torch.tensor([seed * 7919 + 13, seed % 1000], dtype=torch.int64, device="cuda")   # seed, offset
    st = {"case": case, "rng": rng}
    if case["kind"] == "dropout":
        shape = (case["B"], case["L"], case["D"])
        st["x"] = _randn(shape, dtype, gen)
        st["residual"] = _randn(shape, dtype, gen) if case["residual"] else None
        st["dy"] = _randn(shape, dtype, gen) if case["backward"] else None
        if own and case["backward"]:
            st["x"].requires_grad_()
            if case["residual"]:
                st["residual"].requires_grad_()
        return st
    # a trained table: biases of about one
    st["table"] = _randn((case["buckets"], case["H"]), dtype, gen) if case.get("bias", True) else None
    if case["kind"] == "bias":
        reach = max(case["q_start"] + case["q_len"], case["k_len"])
        st["dbias"] = _randn((case["H"], case["q_len"], case["k_len"]), dtype, gen) if case["backward"] else None
        if own:
            import paper_2309_12578_amd as sp
            st["plan"] = sp.relative_buckets(reach, case["buckets"], case["max_distance"], case["both_sides"], device="cuda")
            st["table"].requires_grad_(case["backward"])
        else:
            st["reach"] = reach
            st["bucket_of"] = _bucket_map(reach, case["buckets"], case["max_distance"], case["both_sides"]).cuda()
        return st
    B, H, L, block = case["B"], case["H"], case["L"], case["block"]
    nb = L // block
    shape = (B, H, L, HEAD_DIM)
    st["q"], st["k"], st["v"] = [_randn(shape, dtype, gen) for _ in range(3)]
    st["do"] = _randn(shape, dtype, gen) if case["backward"] else None
    st["lengths"] = None
    if case["ragged"]:   # the batch is padded to its longest sequence, which need not end with a block
        lengths = np.random.default_rng(seed).integers((L + 1) // 2, L + 1, size=B)
        lengths[seed % B] = L - seed % min(block, L)
        st["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    mask = _block_mask(nb, _kept(case), seed)
    if not own:
        st["mask"] = torch.from_numpy(mask).cuda()
        st["bucket_of"] = _bucket_map(L, case["buckets"], case["max_distance"], case["both_sides"]).cuda()
        return st
    import paper_2309_12578_amd as sp
    rows, cols = np.nonzero(mask)
    order = np.lexsort((rows, cols))   # by column, rows ascending
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    ptr = lambda a: ints(np.concatenate([[0], np.cumsum(np.bincount(a, minlength=nb))]))
    st["pattern"] = sp.Pattern(L, block, torch.from_numpy(mask.astype(np.uint8)).cuda(), ptr(rows), ints(cols), ptr(cols),
                               ints(rows[order]), ints(order), ints([rows.size]), torch.zeros((nb, nb), dtype=torch.int64,
                                                                                              device="cuda"), int(rows.size))
    st["plan"] = sp.relative_buckets(L, case["buckets"], case["max_distance"], case["both_sides"], device="cuda") \
        if case["bias"] else None
    if case["backward"]:
        st["inputs"] = [t.requires_grad_() for t in (st["q"], st["k"], st["v"], st["table"]) if t is not None]
    return st


# ------------------------------------------------------------------------------------------------
# the plain form
# ------------------------------------------------------------------------------------------------
M32 = 0xffffffff


def _philox(c0, c1, c2, c3, key):
    """Philox4x32, 7 rounds (Salmon, Moraes, Dror and Shaw, 2011): 32-bit words in int64 tensors (or numbers)."""
    k0, k1 = key & M32, (key >> 32) & M32
    for _ in range(7):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & M32) ^ c1 ^ k0, p1 & M32, ((p0 >> 32) & M32) ^ c3 ^ k1, p0 & M32
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return c0, c1, c2, c3


def _threshold(p):
    return int(round(65536 * p))


def _keep_flat(n, p, rng, stream=0):
    """bool [n]: element i has half i % 2 of word i / 2 % 4 of call i / 8."""
    c = torch.arange((n + 7) // 8, device=rng.device, dtype=torch.int64)
    zero = torch.zeros_like(c)
    words = _philox(c & M32, c >> 32, zero + (rng[1] & M32), zero + stream, rng[0])
    draws = torch.stack([h for w in words for h in (w & 0xffff, w >> 16)], dim=1).reshape(-1)[:n]
    return draws >= _threshold(p)


def _keep_scores(heads, L, p, rng, stream=0):
    """bool [heads, L, L]: query q and key k of head bh have half q % 2 of word k % 4 of call (q / 2, k / 4)."""
    dev = rng.device
    q = torch.arange(L // 2, device=dev, dtype=torch.int64)[:, None]
    k = torch.arange(L // 4, device=dev, dtype=torch.int64)[None, :]
    keep = torch.empty((len(heads), L // 2, 2, L // 4, 4), dtype=torch.bool, device=dev)
    for i, bh in enumerate(heads):
        c0 = q << 14 | k
        zero = torch.zeros_like(c0)
        words = _philox(c0, zero + (bh | 1 << 31), zero + (rng[1] & M32), zero + stream, rng[0])
        for w in range(4):
            keep[i, :, 0, :, w] = (words[w] & 0xffff) >= _threshold(p)
            keep[i, :, 1, :, w] = (words[w] >> 16) >= _threshold(p)
    return keep.view(len(heads), L, L)


def _by_distance(g):
    """Sums of g [n, m] over each distance j - i, from -(n - 1) on: rows upside down, each moved one column on from the
    one before."""
    n, m = g.shape
    moved = torch.nn.functional.pad(g.flip(0), (0, n)).flatten()[:n * (m + n - 1)].view(n, m + n - 1)
    return moved.sum(dim=0, dtype=torch.float64)


def _plain_attn(st):
    case = st["case"]
    B, H, L, block, p = case["B"], case["H"], case["L"], case["block"], case["dropout"]
    dtype = DTYPES[case["dtype"]]
    scale = 1.0 / math.sqrt(HEAD_DIM)
    c = 65536.0 / (65536 - _threshold(p))
    kept = st["mask"].repeat_interleave(block, 0).repeat_interleave(block, 1)
    pos = torch.arange(L, device="cuda")
    bucket = st["bucket_of"][pos[None, :] - pos[:, None] + L - 1] if case["bias"] else None
    out = {n: torch.zeros((B * H, L, HEAD_DIM), dtype=torch.float32, device="cuda") for n in ("o", "dq", "dk", "dv")}
    dtable = torch.zeros((case["buckets"], H), dtype=torch.float64, device="cuda")
    q, k, v = [st[n].view(B * H, L, HEAD_DIM) for n in ("q", "k", "v")]
    do = st["do"].view(B * H, L, HEAD_DIM) if case["backward"] else None
    for bh in range(B * H):
        seen = kept
        length = None
        if st["lengths"] is not None:
            length = st["lengths"][bh // H]
            seen = kept & (pos < length)[None, :] & (pos < length)[:, None]
        Q, K, V = q[bh].float(), k[bh].float(), v[bh].float()
        s = torch.matmul(Q, K.t()) * scale
        if case["bias"]:
            s += st["table"][:, bh % H].float()[bucket]
        s.masked_fill_(~seen, -math.inf)
        m = s.amax(dim=1, keepdim=True)
        m = torch.where(m == -math.inf, torch.zeros_like(m), m)
        s = torch.exp_(s.sub_(m))
        total = s.sum(dim=1, keepdim=True)
        P = s.div_(torch.where(total > 0, total, torch.ones_like(total)))
        keep = _keep_scores([bh], L, p, st["rng"])[0] if p > 0 else None
        A = P * keep * c if p > 0 else P
        O = torch.matmul(A, V)
        out["o"][bh] = O
        if not case["backward"]:
            continue
        G = do[bh].float()
        if length is not None:
            G = torch.where((pos < length)[:, None], G, torch.zeros_like(G))
        out["dv"][bh] = torch.matmul(A.t(), G)
        dP = torch.matmul(G, V.t())
        if p > 0:
            dP = dP * keep * c
        dS = dP.sub_((G * O).sum(dim=1, keepdim=True)).mul_(P)
        out["dq"][bh] = torch.matmul(dS, K) * scale
        out["dk"][bh] = torch.matmul(dS.t(), Q) * scale
        if case["bias"]:
            dtable[:, bh % H].index_add_(0, st["bucket_of"], _by_distance(dS))
    shape = (B, H, L, HEAD_DIM)
    res = {n: out[n].view(shape).to(dtype) for n in (("o", "dq", "dk", "dv") if case["backward"] else ("o",))}
    if case["backward"] and case["bias"]:
        res["dtable"] = dtable.to(dtype)
    return res


def _plain_bias(st):
    case = st["case"]
    dtype = DTYPES[case["dtype"]]
    i = torch.arange(case["q_len"], device="cuda")[:, None] + case["q_start"]
    j = torch.arange(case["k_len"], device="cuda")[None, :]
    bucket = st["bucket_of"][j - i + st["reach"] - 1]
    res = {"bias": st["table"].float().t()[:, bucket].to(dtype)}
    if case["backward"]:
        first = st["reach"] - case["q_start"] - case["q_len"]   # of distance -(q_start + q_len - 1)
        of = st["bucket_of"][first:first + case["q_len"] + case["k_len"] - 1]
        d = torch.zeros((case["buckets"], case["H"]), dtype=torch.float64, device="cuda")
        for h, g in enumerate(st["dbias"]):
            d[:, h].index_add_(0, of, _by_distance(g.float()))
        res["dtable"] = d.to(dtype)
    return res


def _plain_dropout(st):
    case = st["case"]
    dtype = DTYPES[case["dtype"]]
    x, p = st["x"], case["dropout"]
    keep = _keep_flat(x.numel(), p, st["rng"]).view(x.shape)
    c = 65536.0 / (65536 - _threshold(p))
    y = x.float() * keep * c
    if case["residual"]:
        y = st["residual"].float() + y
    res = {"y": y.to(dtype)}
    if case["backward"]:
        res["dx"] = (st["dy"].float() * keep * c).to(dtype)
        if case["residual"]:
            res["dresidual"] = st["dy"]
    return res


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(st):
    case = st["case"]
    if not own:
        return {"attn": _plain_attn, "bias": _plain_bias, "dropout": _plain_dropout}[case["kind"]](st)
    import paper_2309_12578_amd as sp
    with torch.set_grad_enabled(case["backward"]):
        if case["kind"] == "attn":
            o = sp.sparse_attention(st["q"], st["k"], st["v"], st["pattern"], bias=st["table"], buckets=st["plan"],
                                    lengths=st["lengths"], dropout=case["dropout"], rng=st["rng"])
            if not case["backward"]:
                return {"o": o}
            grads = torch.autograd.grad(o, st["inputs"], st["do"])
            return dict(zip(("o", "dq", "dk", "dv", "dtable"), (o.detach(), *grads)))
        if case["kind"] == "bias":
            bias = sp.relative_bias(st["table"], st["plan"], case["q_len"], case["k_len"], case["q_start"])
            if not case["backward"]:
                return {"bias": bias}
            return {"bias": bias.detach(), "dtable": torch.autograd.grad(bias, st["table"], st["dbias"])[0]}
        y = sp.dropout_add(st["x"], st["residual"], case["dropout"], st["rng"])
        if not case["backward"]:
            return {"y": y}
        inputs = [st["x"]] + ([st["residual"]] if case["residual"] else [])
        return dict(zip(("y", "dx", "dresidual"), (y.detach(), *torch.autograd.grad(y, inputs, st["dy"]))))


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "dropout":
        n = case["B"] * case["L"] * case["D"]
        tensors = 2 + case["residual"] + 2 * case["backward"]
        return {"bytes": n * size * tensors, "flops": 2 * n * (1 + case["backward"])}
    if case["kind"] == "bias":
        n = case["H"] * case["q_len"] * case["k_len"]
        return {"bytes": n * size * (1 + case["backward"]), "flops": n * case["backward"]}
    n = case["B"] * case["H"] * case["L"] * HEAD_DIM
    # what a ragged batch keeps: lengths of three quarters of L on average, in both directions
    share = 0.6 if case["ragged"] else 1.0
    flops = share * case["B"] * case["H"] * _kept(case) * case["block"] ** 2 * HEAD_DIM * (14 if case["backward"] else 4)
    return {"bytes": n * size * (8 if case["backward"] else 4) + 4 * case["B"] * case["H"] * case["L"], "flops": flops}


# ------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------------
def _halves(words, half):
    return torch.where(half, torch.bitwise_right_shift(words, 16), words) % 65536


def _draws(call, c1, half, word, rng):
    """16-bit draws: of Philox calls with counter (call, c1, offset, 0), word `word`, half `half` (tensors of one shape)."""
    seed, offset = int(rng[0]), int(rng[1])
    state = [call, c1.expand_as(call), torch.full_like(call, offset % 2 ** 32), torch.zeros_like(call)]
    for r in range(7):
        keys = [(seed % 2 ** 32 + r * 2654435769) % 2 ** 32, (seed // 2 ** 32 % 2 ** 32 + r * 3144134277) % 2 ** 32]
        hi, lo = [], []
        for x, mul in ((state[0], 3528531795), (state[2], 3449720151)):
            # 32 x 32 bits by halves of the first factor, so that no product passes 48 bits
            low, high = (x % 65536) * mul, (x // 65536) * mul
            both = low // 65536 + high
            lo.append(both % 65536 * 65536 + low % 65536)
            hi.append(both // 65536)
        state = [hi[1] ^ state[1] ^ keys[0], lo[1], hi[0] ^ state[3] ^ keys[1], lo[0]]
    picked = state[0]
    for w in (1, 2, 3):
        picked = torch.where(word == w, state[w], picked)
    return _halves(picked, half)


def _exact_attn(case, st):
    B, H, L, block, p = case["B"], case["H"], case["L"], case["block"], case["dropout"]
    f64 = dict(dtype=torch.float64, device="cuda")
    q, k, v = [st[n].double().view(B * H, L, HEAD_DIM) for n in ("q", "k", "v")]
    g = st["do"].double().view(B * H, L, HEAD_DIM) if case["backward"] else None
    lengths = torch.full((B,), L, device="cuda") if st["lengths"] is None else st["lengths"].long()
    length = lengths.repeat_interleave(H)
    o = torch.zeros((B * H, L, HEAD_DIM), **f64)
    dq, dk, dv = [torch.zeros_like(o) for _ in range(3)]
    dtable = torch.zeros((H, case["buckets"]), **f64)
    inside = torch.arange(block, device="cuda")
    heads = torch.arange(B * H, device="cuda")
    drop = round(p * 65536)
    mask = st["mask"].cpu().numpy()
    for row in range(L // block):
        i = row * block + inside
        j = (torch.from_numpy(np.flatnonzero(mask[row])).cuda()[:, None] * block + inside).flatten()
        if j.numel() == 0:
            continue
        # heads at a time, for the memory of a long row
        step = max(1, int(2 ** 25 // (block * j.numel())))
        for h0 in range(0, B * H, step):
            hs = heads[h0:h0 + step]
            valid = (i[None, :, None] < length[hs][:, None, None]) & (j[None, None, :] < length[hs][:, None, None])
            kj, vj = k[hs][:, j], v[hs][:, j]
            x = torch.matmul(q[hs][:, i], kj.transpose(1, 2).contiguous()) / 8.0
            which = st["bucket_of"][(j[None, :] - i[:, None]) + (L - 1)]
            if case["bias"]:
                x = x + st["table"].double().t()[hs % H][:, which]
            top = torch.where(valid, x, torch.full_like(x, -1e300)).max(dim=2, keepdim=True).values
            e = torch.where(valid, torch.exp(x - top), torch.zeros_like(x))
            z = e.sum(2, keepdim=True)
            prob = e / torch.where(z == 0, torch.ones_like(z), z)
            factor = torch.ones_like(prob)
            if drop > 0:
                call = ((i // 2)[:, None] * 16384 + (j // 4)[None, :]).expand(hs.numel(), -1, -1)
                d = _draws(call, (hs + 2 ** 31)[:, None, None], (i % 2 == 1)[None, :, None], (j % 4)[None, None, :], st["rng"])
                factor = (d >= drop).double() / (1 - drop / 65536)
            w = prob * factor
            o[h0:h0 + step, i] = torch.matmul(w, vj)
            if not case["backward"]:
                continue
            gi = torch.where((i[None, :] < length[hs][:, None])[:, :, None], g[hs][:, i], torch.zeros((), **f64))
            dv[h0:h0 + step, j] += torch.matmul(w.transpose(1, 2), gi)
            dw = torch.matmul(gi, vj.transpose(1, 2).contiguous()) * factor
            ds = prob * (dw - (prob * dw).sum(2, keepdim=True))
            dq[h0:h0 + step, i] = torch.matmul(ds, kj) / 8.0
            dk[h0:h0 + step, j] += torch.matmul(ds.transpose(1, 2), q[hs][:, i]) / 8.0
            if case["bias"]:
                flat = (hs % H)[:, None] * case["buckets"] + which.reshape(1, -1)
                dtable.view(-1).scatter_add_(0, flat.flatten(), ds.flatten())
    shape = (B, H, L, HEAD_DIM)
    res = {"o": o.view(shape)}
    if case["backward"]:
        res.update(dq=dq.view(shape), dk=dk.view(shape), dv=dv.view(shape))
        if case["bias"]:
            res["dtable"] = dtable.t().contiguous()
    return res


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "attn":
        return _exact_attn(case, st)
    if case["kind"] == "bias":
        n, m = case["q_len"], case["k_len"]
        first = st["reach"] - 1 - case["q_start"]
        rows = [st["bucket_of"][first - i:first - i + m] for i in range(n)]
        table = st["table"].double()
        res = {"bias": torch.stack([table[r] for r in rows], dim=0).permute(2, 0, 1).contiguous()}
        if case["backward"]:
            d = torch.zeros((case["buckets"], case["H"]), dtype=torch.float64, device="cuda")
            for i, r in enumerate(rows):
                d.index_add_(0, r, st["dbias"][:, i].double().t().contiguous())
            res["dtable"] = d
        return res
    x, drop = st["x"].double(), round(case["dropout"] * 65536)
    n = torch.arange(x.numel(), device="cuda")
    d = torch.cat([_draws(c // 8, torch.zeros((), dtype=torch.int64, device="cuda"), c % 2 == 1, c // 2 % 4, st["rng"])
                   for c in n.split(2 ** 25)]).view(x.shape)
    scale = 65536 / (65536 - drop)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    res = {"y": torch.where(d < drop, zero, x * scale)}
    if case["residual"]:
        res["y"] = res["y"] + st["residual"].double()
    if case["backward"]:
        res["dx"] = torch.where(d < drop, zero, st["dy"].double() * scale)
        if case["residual"]:
            res["dresidual"] = st["dy"].double()
    return res
