"""Rows of logits as categorical distributions (xrl_logprob, xrl_logprob_grad) against their definition in 64 bits.

Tolerances.  An exponential is off by 2 units in its last place (2^-22) and by what its argument is: (x - m) c is rounded twice,
and weighted by the probabilities |argument| is at most the entropy.  A thread adds ceil(vocab / threads) terms one after the
other and some ten partial sums are joined, each step 2^-24.  That is the relative error of a row's sum, `sum_error`; logarithms,
products and the result's own rounding are 2^-23 of what they round."""
import math

import pytest
import torch

import paper_2304_14698_b200 as xrl

pytestmark = pytest.mark.gpu
INF = math.inf
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
OUTS = ("logp", "entropy", "norm", "top_token", "top_logp")


def sum_error(vocab):
    return (math.ceil(vocab / 128) + 80) * 2.0 ** -24


def define(x, token, mask, scale, top):
    """The definition, row for row, in 64 bits."""
    z = x.double()
    if mask is not None:
        z = z.masked_fill(mask.expand(z.shape) == 0, -INF)
    m = z.max(1).values
    empty = m == -INF
    d = scale * (z - m.masked_fill(empty, 0)[:, None])
    l = torch.log(torch.exp(d).sum(1))
    lp = d - l[:, None]
    p = torch.exp(lp)
    h = -torch.where(p == 0, torch.zeros_like(p), p * lp).sum(1)
    o = {"norm": torch.stack((m, l), 1), "entropy": h.masked_fill(empty, 0), "lp": lp, "p": p, "z": z}
    if token is not None:
        t = token.long()
        logp = lp.gather(1, t.clamp(0, x.shape[1] - 1)[:, None])[:, 0]
        logp = logp.masked_fill(z.gather(1, t.clamp(0, x.shape[1] - 1)[:, None])[:, 0] == -INF, -INF)
        logp[t == -1] = 0
        logp[(t < -1) | (t >= x.shape[1])] = math.nan
        o["logp"] = logp
    if top:
        v, i = torch.sort(z, dim=1, descending=True, stable=True)
        v, i = v[:, :top], i[:, :top]
        o["top_token"] = i.masked_fill(v == -INF, -1).int()
        o["top_logp"] = lp.gather(1, i).masked_fill(v == -INF, -INF)
    return o


def near(got, want, tol, what):
    got, want, tol = got.double(), want.double(), torch.as_tensor(tol, dtype=torch.float64, device=got.device)
    assert got.shape == want.shape, what
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    same = fine | torch.isnan(want) | (got == want)
    assert bool(same.all()), (what, got[~same][:4], want[~same][:4])
    off = ((got - want).abs() - tol)[fine] if tol.dim() else (got - want).abs()[fine] - tol
    assert off.numel() == 0 or float(off.max()) <= 0, (what, float(off.max()))


def check_scores(o, x, token, mask, scale, top):
    want, e = define(x, token, mask, scale, top), sum_error(x.shape[1])
    m, l = want["norm"].T
    near(o["norm"][:, 0], m, 0.0, "largest")
    near(o["norm"][:, 1], l, e + 2.0 ** -23 * l.abs(), "l")
    near(o["entropy"], want["entropy"], 4 * e * (1 + want["entropy"]), "entropy")
    if token is not None:
        near(o["logp"], want["logp"], e + 2.0 ** -22 * (want["logp"].abs() + l.abs()), "logp")
    if top:
        assert torch.equal(o["top_token"], want["top_token"]), "alternatives"
        near(o["top_logp"], want["top_logp"], e + 2.0 ** -22 * (want["top_logp"].abs() + l.abs()[:, None]), "top_logp")
    return want


def make(dtype, rows, vocab, seed, pad=0, shift=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (3 * torch.randn(rows, vocab + pad + shift, device="cuda", generator=g)).to(DTYPES[dtype])[:, shift:shift + vocab]
    token = torch.randint(-1, vocab, (rows,), device="cuda", generator=g, dtype=torch.int32)
    mask = (torch.rand(rows, vocab, device="cuda", generator=g) < 0.5).to(torch.uint8)
    return x, token, mask, g


SIZES = [(5, 1), (3, 2), (9, 7), (64, 33), (7, 128), (64, 129), (6, 256), (3, 257), (5, 512), (4, 1000), (3, 1024), (2, 1025),
         (5, 1031), (300, 1100), (2, 4099), (1, 8192), (3, 16391), (40, 33000), (150, 9001), (2, 50001), (1, 131072), (17, 131071)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("masked", ["none", "one", "rows"])
def test_scores_of_every_size(dtype, rows, vocab, masked):
    x, token, mask, _ = make(dtype, rows, vocab, rows + vocab, pad=vocab % 5, shift=rows % 3)
    mask = None if masked == "none" else mask[:1] if masked == "one" else mask
    for top, scale in ((0, 1.0), (min(5, vocab), 0.7), (min(32, vocab), 1.5)):
        check_scores(xrl.xrl_logprob(x, token, mask=mask, scale=scale, top=top), x, token, mask, scale, top)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [9, 700, 1500, 40000])
def test_rows_at_the_edges_of_the_range(dtype, vocab):
    """Rows without support, of the type's lowest value, with infinities and numbers that are none, ties, few valid entries."""
    x, token, mask, g = make(dtype, 16, vocab, 3)
    x, low = x.clone(), torch.finfo(DTYPES[dtype]).min
    mask[:] = 1
    token[:] = vocab // 2
    mask[0] = 0                                                      # nothing valid
    x[1] = -INF                                                      # nothing above -infinity
    x[2] = low                                                       # all at the lowest value: uniform
    x[3, :] = -INF
    x[3, vocab // 2] = 1.0                                           # one entry
    x[4] = low
    x[4, 3] = 2.0                                                    # masked by the lowest value
    x[5, ::2], mask[5] = math.nan, 1
    mask[5, ::2] = 0                                                 # no number where the mask looks away
    x[6, 5] = math.nan
    x[7, 1] = INF
    x[8] = 1.25                                                      # all equal
    x[9] = torch.arange(vocab, device="cuda", dtype=torch.float32).to(x.dtype)      # rising
    x[10] = -x[9]
    mask[11] = 0
    mask[11, [0, vocab // 2, vocab - 1]] = 1
    x[12], mask[12] = INF, 0
    mask[12, 2] = 1
    x[12, 2] = -3.0
    x[13] = 1e4 if dtype == "fp32" else 1e4
    x[13, :: 3] += 64
    x[14] = torch.where(torch.arange(vocab, device="cuda") % 2 == 0, 0.0, -0.0).to(x.dtype)    # equal zeros
    x[15, : vocab // 2 + 1] = low
    x[15, vocab // 2 + 1:] = -INF
    for top in (0, 4, min(vocab, 32)):
        o = xrl.xrl_logprob(x, token, mask=mask, top=top)
        keep = [i for i in range(16) if i not in (6, 7)]
        w = torch.tensor(keep, device="cuda")
        check_scores({k: v[w] for k, v in o.items()}, x[w], token[w], mask[w], 1.0, top)
        assert torch.isnan(o["logp"][6:8]).all() and torch.isnan(o["entropy"][6:8]).all() and torch.isnan(o["norm"][6:8, 1]).all()
        if top:
            # the one number that is none is no alternative: a list of all entries ends without it
            assert o["top_token"][7, 0] == 1 and torch.equal(torch.isnan(o["top_logp"][6:8]), o["top_token"][6:8] >= 0)
            rest = x[6].float().clone()
            rest[5] = -INF
            v, i = torch.sort(rest, descending=True, stable=True)
            assert torch.equal(o["top_token"][6], i.masked_fill(v == -INF, -1)[:top].int())


def test_tokens_out_of_range_and_outputs_left_out():
    x, token, mask, _ = make("fp32", 6, 2000, 5)
    token[:] = torch.tensor([-1, -2, 2000, 1999, 0, 2 ** 31 - 1], dtype=torch.int32)
    o = xrl.xrl_logprob(x, token)
    check_scores(o, x, token, None, 1.0, 0)
    again = xrl.xrl_logprob(x, None)
    assert set(again) == {"entropy", "norm"} and torch.equal(again["entropy"], o["entropy"])
    only = {"logp": torch.empty(6, device="cuda")}
    assert xrl.xrl_logprob(x, token, out=only) is only
    assert torch.equal(only["logp"].nan_to_num(7.0), o["logp"].nan_to_num(7.0))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [100, 1500, 70001])
@pytest.mark.parametrize("scale", [1e-6, 1e-3, 0.37, 1.0, 3.3, 1e3, 1e6])
def test_logits_of_every_size_and_scale(dtype, vocab, scale):
    """Logits far from 0, and masks by large negative numbers of every size: the scaled ones are off by 2^-23 of themselves, an
    exponential's argument by as much of what it is multiplied from."""
    x, token, _, g = make(dtype, 24, vocab, 15)
    x = x.float() / scale
    for i, far in enumerate((1e3, 1e5, 1e7, 1e8, 1e9, 1e10, 1e12, 1e20, 1e30, 3e38)):
        x[2 * i, torch.rand(vocab, device="cuda", generator=g) < 0.9] = -far
        x[2 * i + 1] -= min(far / scale, 3e38)
    x[20] += 1e3 / scale
    x[21] += 1e9 / scale
    x[22] += 1e30
    x = x.clamp(-3e38, 3e38).to(DTYPES[dtype])
    o, want = xrl.xrl_logprob(x, token, scale=scale, top=5), define(x, token, None, scale, 5)
    e, l = sum_error(vocab), want["norm"][:, 1]
    near(o["norm"][:, 0], want["norm"][:, 0], 0.0, "largest")
    near(o["norm"][:, 1], l, e + 2.0 ** -23 * l.abs(), "l")
    near(o["entropy"], want["entropy"], 4 * e * (1 + want["entropy"]), "entropy")
    assert torch.equal(o["top_token"], want["top_token"])
    fits = want["logp"].abs() < 3e38
    near(o["logp"][fits], want["logp"][fits], (e + 2.0 ** -22 * (want["logp"].abs() + l.abs()))[fits], "logp")


@pytest.mark.parametrize("dtype", DTYPES)
def test_the_same_bits_every_time_and_rows_alone(dtype):
    x, token, mask, _ = make(dtype, 33, 20011, 6)
    a = xrl.xrl_logprob(x, token, mask=mask, top=20)
    for _ in range(5):
        b = xrl.xrl_logprob(x, token, mask=mask, top=20)
        assert all(torch.equal(a[k], b[k]) for k in a)
    r = 7                                                            # one row alone, split over more CTAs
    check_scores(xrl.xrl_logprob(x[r:r + 1], token[r:r + 1], mask=mask[r:r + 1], top=20), x[r:r + 1], token[r:r + 1],
                 mask[r:r + 1], 1.0, 20)


def reference_grad(x, token, mask, scale, norm, entropy, dlogp, dentropy):
    """The formula in 64 bits from the same fp32 inputs, and a bound on a kernel's distance to it."""
    z = x.double()
    if mask is not None:
        z = z.masked_fill(mask.expand(z.shape) == 0, -INF)
    rows, vocab = z.shape
    m, l = norm.double().T
    lp = torch.where(z == -INF, torch.zeros_like(z), scale * (z - m[:, None]) - l[:, None])
    p = torch.exp(lp)
    there = torch.zeros_like(z)
    if token is not None:
        ok = (token >= 0) & (token < vocab)
        there[ok, token[ok].long()] = 1
    zero = torch.zeros(rows, dtype=torch.float64, device=z.device)
    dl = zero if dlogp is None else torch.where(token == -1, zero, dlogp.double())
    if dlogp is not None:
        dl = torch.where((token < -1) | (token >= vocab), math.nan, dl)
    dh = zero if dentropy is None else dentropy.double()
    h = zero if entropy is None or dentropy is None else entropy.double()
    dl, dh, h = dl[:, None], dh[:, None], h[:, None]
    g = scale * (dl * (there - p) - dh * p * (lp + h))
    # the argument of the exponential: three roundings of values up to |lp| + 2 |l|
    arg = 2.0 ** -22 * (lp.abs() + 2 * l.abs()[:, None] + 1)
    rel = arg + 2.0 ** -22
    tol = scale * (dl.abs() * (p * rel + 2.0 ** -23 * (there - p).abs()) + dh.abs() * p * ((lp.abs() + h.abs()) * (rel + 2.0 ** -22) + arg))
    out = z == -INF
    tol = tol + torch.finfo(x.dtype).eps / 2 * (g.abs() + tol) + 2.0 ** -126 * scale
    return g.masked_fill(out, 0.0), tol.masked_fill(out, 0.0).nan_to_num(0.0)


def fp32_norm(x, mask, scale):
    w = define(x, None, mask, scale, 0)
    return w["norm"].float().contiguous(), w["entropy"].float().contiguous()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_gradient_of_every_size(dtype, rows, vocab):
    x, token, mask, g = make(dtype, rows, vocab, rows + 2 * vocab, pad=vocab % 3, shift=vocab % 7)
    dlogp = torch.randn(rows, device="cuda", generator=g)
    dent = torch.randn(rows, device="cuda", generator=g)
    for m, scale, a, b in ((None, 1.0, dlogp, dent), (mask, 0.7, dlogp, dent), (mask[:1], 1.3, dlogp, None), (None, 1.0, None, dent)):
        norm, ent = fp32_norm(x, m, scale)
        got = xrl.xrl_logprob_grad(x, norm, token if a is not None else None, a, ent if b is not None else None, b, mask=m, scale=scale)
        assert got.is_contiguous() and got.dtype == x.dtype
        near(got, *reference_grad(x, token, m, scale, norm, ent, a, b), "gradient")
        # into rows of a wider buffer whose columns outside stay as they are; and over the logits
        wide = torch.full((rows, vocab + 11), 7.0, device="cuda", dtype=x.dtype)
        xrl.xrl_logprob_grad(x, norm, token, a, ent, b, mask=m, scale=scale, grad=wide[:, 5:5 + vocab])
        assert torch.equal(wide[:, 5:5 + vocab], got) and bool((wide[:, :5] == 7).all()) and bool((wide[:, 5 + vocab:] == 7).all())
        over = torch.empty(rows, vocab + 9, device="cuda", dtype=x.dtype)[:, 2:2 + vocab]
        over.copy_(x)
        xrl.xrl_logprob_grad(over, norm, token, a, ent, b, mask=m, scale=scale, grad=over)
        assert torch.equal(over, got)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [12, 3000])
def test_gradient_at_the_edges_of_the_range(dtype, vocab):
    x, token, mask, g = make(dtype, 8, vocab, 4)
    x, mask[:] = x.clone(), 1
    token[:] = torch.tensor([3, 3, 3, -1, vocab, -2, 2, 2], dtype=torch.int32)
    mask[0] = 0
    x[1, 4:] = -INF
    x[2] = torch.finfo(x.dtype).min
    x[6, 1], mask[6, 1] = math.nan, 0
    mask[7, 2] = 0                                                    # the token itself is masked
    dlogp, dent = torch.randn(8, device="cuda", generator=g), torch.randn(8, device="cuda", generator=g)
    o = xrl.xrl_logprob(x, token, mask=mask)
    norm, ent = o["norm"], o["entropy"]
    got = xrl.xrl_logprob_grad(x, norm, token, dlogp, ent, dent, mask=mask)
    near(got, *reference_grad(x, token, mask, 1.0, norm, ent, dlogp, dent), "gradient")
    assert bool((got[0] == 0).all()) and bool(torch.isnan(got[4:6]).all()) and float(got[7, 2]) == 0 and float(got[6, 1]) == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradient_of_extreme_scales_and_gradients(dtype):
    x, token, mask, g = make(dtype, 6, 1000, 14)
    mask.scatter_(1, token.clamp(min=0).long()[:, None], 1)
    x = x.clone()
    x[:, 7] = -INF
    for scale, big in ((1e6, 1e30), (1e-6, 1e30), (1e6, 1e-30)):
        d, e = torch.randn(6, device="cuda", generator=g), big * torch.randn(6, device="cuda", generator=g)
        norm, ent = fp32_norm(x, mask, scale)
        got = xrl.xrl_logprob_grad(x, norm, token, d, ent, e, mask=mask, scale=scale)
        assert bool((got[:, 7] == 0).all()) and bool((got[mask == 0] == 0).all()) and not bool(torch.isnan(got).any())
        want, tol = reference_grad(x, token, mask, scale, norm, ent, d, e)
        fits = want.abs() < torch.finfo(x.dtype).max / 2
        near(got[fits], want[fits], tol[fits], "gradient")
    d[0], e[1] = INF, INF
    got = xrl.xrl_logprob_grad(x, norm, token, d, ent, e, mask=mask, scale=scale)
    assert bool((got[mask == 0] == 0).all())


def test_gradient_against_differences():
    """(f(x + h e_j) - f(x - h e_j)) / 2h of f = sum(dlogp logp + dentropy H) in 64 bits; its error is h^2 f''' / 6 < 1e-7
    for slopes of order one at h = 1e-4, and the fp32 gradient's own 1e-6."""
    x, token, mask, g = make("fp32", 4, 19, 8)
    dlogp, dent = torch.randn(4, device="cuda", generator=g), torch.randn(4, device="cuda", generator=g)
    mask.scatter_(1, token.clamp(min=0).long()[:, None], 1)
    o = xrl.xrl_logprob(x, token, mask=mask, scale=0.8)
    got = xrl.xrl_logprob_grad(x, o["norm"], token, dlogp, o["entropy"], dent, mask=mask, scale=0.8).double()

    def f(z):
        w = define(z, token, mask, 0.8, 0)
        return dlogp.double() * w["logp"] + dent.double() * w["entropy"]

    for j in range(19):
        e = torch.zeros(4, 19, dtype=torch.float64, device="cuda")
        e[:, j] = 1e-4
        slope = (f(x.double() + e) - f(x.double() - e)) / 2e-4
        assert float((slope - got[:, j]).abs().max()) < 2e-6


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 60000), (200, 60000), (3, 2500)])
@pytest.mark.parametrize("top", [1, 8, 32])
def test_alternatives_of_every_kind_of_row(dtype, rows, vocab, top):
    """Few distinct values, one block of large ones, rising and falling rows, few valid entries, all equal."""
    g = torch.Generator(device="cuda").manual_seed(top)
    at = torch.arange(vocab, device="cuda")
    kinds = [torch.randint(0, 3, (vocab,), device="cuda", generator=g).float(), (at // 1000 == 1).float() * 5 + at * 1e-4, at * 1e-3,
             -at * 1e-3, torch.where(torch.rand(vocab, device="cuda", generator=g) < 20 / vocab, 1.0, -INF), torch.zeros(vocab, device="cuda"),
             torch.where(at % 512 == 3, 2.0, -1.0), torch.full((vocab,), -INF, device="cuda")]
    x = torch.stack([kinds[i % len(kinds)] for i in range(max(rows, len(kinds)))]).to(DTYPES[dtype])
    for first in range(0, len(x), rows):
        part = x[first:first + rows]
        check_scores(xrl.xrl_logprob(part, top=top), part, None, None, 1.0, top)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [61, 129, 500, 801, 1031, 4100, 8190, 17000, 60000])
@pytest.mark.parametrize("top", [3, 20, 21, 32])
def test_alternatives_of_many_rows(dtype, vocab, top):
    """Rows enough for a warp or a CTA each: random ones, with and without a mask, the best in one stretch, in one column of threads,
    behind masked larger ones."""
    rows, g = 600, torch.Generator(device="cuda").manual_seed(top)
    x = torch.randn(rows, vocab, device="cuda", generator=g) * 3
    at = torch.arange(vocab, device="cuda")
    x[::5] += 20.0 * (at // 800 == 1)
    x[1::5] += 20.0 * (at % 512 == 17)
    x[2::5] = at * 1e-3
    x[3::5] = -at * 1e-3
    x = x.to(DTYPES[dtype])
    mask = torch.rand(rows, vocab, device="cuda", generator=g) < 0.3
    for m in (None, mask, (x < 2.0) & (at % 3 > 0)):
        check_scores(xrl.xrl_logprob(x, mask=m, top=top), x, None, m, 1.0, top)


def test_offsets_past_32_bits():
    """Rows 2^29 entries apart: the last ones start past 2^31 entries and 2^32 bytes."""
    stride, vocab, rows = 2 ** 29 + 8, 5000, 6
    buf = torch.empty(stride * (rows - 1) + vocab, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, vocab), (stride, 1))
    small, token, _, g = make("bf16", rows, vocab, 9)
    x.copy_(small)
    o = xrl.xrl_logprob(x, token, top=5)
    want = xrl.xrl_logprob(small, token, top=5)
    assert all(torch.equal(o[k], want[k]) for k in o)
    d = torch.randn(rows, device="cuda", generator=g)
    xrl.xrl_logprob_grad(x, o["norm"], token, d, o["entropy"], d, grad=x)
    assert torch.equal(x, xrl.xrl_logprob_grad(small, o["norm"], token, d, o["entropy"], d))


def test_streams_graphs_and_no_rows():
    x, token, mask, g = make("bf16", 24, 9000, 10)
    d = torch.randn(24, device="cuda", generator=g)
    want = xrl.xrl_logprob(x, token, mask=mask, top=7)
    wgrad = xrl.xrl_logprob_grad(x, want["norm"], token, d, want["entropy"], d, mask=mask)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        o = xrl.xrl_logprob(x, token, mask=mask, top=7)
        gr = xrl.xrl_logprob_grad(x, o["norm"], token, d, o["entropy"], d, mask=mask)
    side.synchronize()
    assert all(torch.equal(o[k], want[k]) for k in o) and torch.equal(gr, wgrad)
    o = xrl.xrl_logprob(x, token, mask=mask, top=7, stream=side.cuda_stream)
    gr = xrl.xrl_logprob_grad(x, o["norm"], token, d, o["entropy"], d, mask=mask, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(o[k], want[k]) for k in o) and torch.equal(gr, wgrad)
    assert torch.equal(xrl.xrl_logprob(x, token, mask=mask, stream=0)["logp"], want["logp"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o2 = xrl.xrl_logprob(x, token, mask=mask, top=7)
        gr2 = xrl.xrl_logprob_grad(x, o2["norm"], token, d, o2["entropy"], d, mask=mask)
    x.copy_(x.flip(0).clone()), token.copy_(token.flip(0).clone()), mask.copy_(mask.flip(0).clone()), d.copy_(d.flip(0).clone())
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o2[k], want[k].flip(0)) for k in o2) and torch.equal(gr2, wgrad.flip(0))
    none = xrl.xrl_logprob(x[:0], token[:0], mask=mask[:0], top=7)
    assert none["top_token"].shape == (0, 7)
    assert xrl.xrl_logprob_grad(x[:0], none["norm"], token[:0], d[:0], none["entropy"], d[:0]).shape == (0, 9000)
