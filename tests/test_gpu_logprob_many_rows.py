"""Rows of logits in numbers that give each row a CTA of its own, and masked gradients whose CTAs take many pieces of rows.

Definitions and tolerances are those of test_gpu_logprob."""
import math

import pytest
import torch

import paper_2304_14698_b200 as xrl
from test_gpu_logprob import DTYPES, INF, check_scores, define, fp32_norm, make, near, reference_grad, sum_error

pytestmark = pytest.mark.gpu
ROWS = 320                                 # more than clusters, or a CTA on every SM twice, are used for
WIDTH = {"fp32": 4, "bf16": 8}             # entries of a 16-byte vector

# Vectors of a row: about 512, 2,000, 3,000 and 6,000, where threads and vectors a thread has in flight change; with the rest
# behind whole groups (256 vectors up to there, 512 and 1,024 then) none, a few, just under half of one and just over
VECS = [257, 383, 385, 511, 512, 525, 767, 769, 1023, 1024, 1290, 1999, 2000, 2302, 2306, 2999, 3000, 3583, 3585, 4096, 4100, 5999, 6000, 6144]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("masked", ["none", "one", "rows"])
@pytest.mark.parametrize("vecs", VECS)
def test_scores_of_a_cta_per_row(dtype, masked, vecs):
    vocab = vecs * WIDTH[dtype] + vecs % WIDTH[dtype]
    x, token, mask, _ = make(dtype, ROWS, vocab, vecs, pad=vecs % 3, shift=vecs % 5)
    mask = None if masked == "none" else mask[:1] if masked == "one" else mask
    check_scores(xrl.xrl_logprob(x, token, mask=mask, scale=0.9), x, token, mask, 0.9, 0)


def edge_rows(dtype, vocab):
    """One row of each kind: without support, of one value, at the type's lowest, with infinities, far from 0, ..."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    low = torch.finfo(DTYPES[dtype]).min
    at = torch.arange(vocab, device="cuda")
    noise = lambda: 3 * torch.randn(vocab, device="cuda", generator=g)  # noqa: E731
    one = torch.full((vocab,), -INF, device="cuda")
    one[vocab // 2] = 1.0
    lowest = torch.full((vocab,), low, device="cuda")
    lowest[3] = 2.0
    rows = [noise(), torch.full((vocab,), -INF, device="cuda"), torch.full((vocab,), low, device="cuda"), one, lowest,
            torch.full((vocab,), 1.25, device="cuda"), torch.where(at % 2 == 0, 0.0, -0.0), torch.where(at <= vocab // 2, low, -INF),
            noise() + 1e7, noise() - 1e7, noise() * 1e6, 1e30 + 1e29 * noise(), -1e30 + 1e29 * noise(), at * 1e-3, -at * 1e-3]
    return torch.stack(rows).clamp(min=-INF, max=3e38).to(DTYPES[dtype])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vecs", [129, 300, 700, 3100, 6050])
@pytest.mark.parametrize("masked", [False, True])
def test_edges_of_the_range_in_many_rows(dtype, vecs, masked):
    vocab = vecs * WIDTH[dtype] + 3
    kinds = edge_rows(dtype, vocab)
    n = len(kinds)
    x = kinds.repeat((ROWS + n - 1) // n, 1)
    g = torch.Generator(device="cuda").manual_seed(vecs)
    token = torch.randint(-1, vocab, (len(x),), device="cuda", generator=g, dtype=torch.int32)
    mask = None
    if masked:
        mask = torch.rand(x.shape, device="cuda", generator=g) < 0.5
        mask[7] = False
        x = torch.where(mask | (torch.rand(x.shape, device="cuda", generator=g) < 0.5), x, math.nan)     # not looked at
    for top in (0, 20, 32):
        o, want, e = xrl.xrl_logprob(x, token, mask=mask, top=top), define(x, token, mask, 1.0, top), sum_error(vocab)
        l = want["norm"][:, 1]
        near(o["norm"][:, 0], want["norm"][:, 0], 0.0, "largest")
        near(o["norm"][:, 1], l, e + 2.0 ** -23 * l.abs(), "l")
        near(o["entropy"], want["entropy"], 4 * e * (1 + want["entropy"]), "entropy")
        near(o["logp"], want["logp"], e + 2.0 ** -22 * (want["logp"].abs() + l.abs()), "logp")
        if top:
            assert torch.equal(o["top_token"], want["top_token"])
    # numbers that are none, and infinities, in the support
    x = x.clone()
    x[::n, vocab - 1], x[5::n, 1] = math.nan, INF
    if masked:
        mask[::n, vocab - 1] = mask[5::n, 1] = True
    for top in (0, 20):
        o = xrl.xrl_logprob(x, token, mask=mask, top=top)
        for k in (0, 5):
            assert bool(torch.isnan(o["entropy"][k::n]).all()) and bool(torch.isnan(o["norm"][k::n, 1]).all())
        if top:
            assert bool((o["top_token"][5::n, 0] == 1).all()) and not bool((o["top_token"][::n] == vocab - 1).any())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(4, 50), (4, 1000), (4, 1500), (4, 90000), (ROWS, 1500), (ROWS, 30001)])
@pytest.mark.parametrize("top", [0, 3, 32])
def test_rows_with_numbers_that_are_none(dtype, rows, vocab, top):
    """NaN or +infinity in the support: NaN for a choice inside the support, -infinity for one outside it; NaN entries are no
    alternatives, infinite ones come first, the lower index before the higher."""
    x, token, mask, _ = make(dtype, rows, vocab, rows + vocab)
    x, mask[:] = x.clone(), 1
    broken = x[::2]
    x[::2, 7] = math.nan
    x[1::2, 9], x[1::2, 30] = INF, INF
    x[:, 11] = -INF
    mask[:, 13] = 0
    for t in (7, 9, 11, 13, 20):
        token[:] = t
        o = xrl.xrl_logprob(x, token, mask=mask, top=top)
        if t in (11, 13):
            assert bool((o["logp"] == -INF).all())
        else:
            assert bool(torch.isnan(o["logp"]).all())
        assert bool(torch.isnan(o["entropy"]).all()) and bool(torch.isnan(o["norm"][:, 1]).all())
    if top:
        assert bool((o["top_token"][1::2, 0] == 9).all()) and bool((o["top_token"][1::2, 1] == 30).all())
        z = broken.float().masked_fill(mask[::2] == 0, -INF).masked_fill(torch.isnan(broken), -INF)
        v, i = torch.sort(z, dim=1, descending=True, stable=True)
        assert torch.equal(o["top_token"][::2], i.masked_fill(v == -INF, -1)[:, :top].int())
        assert torch.equal(torch.isnan(o["top_logp"]), o["top_token"] >= 0)


# (rows, vocab): pieces of 1,024 vectors for each of the 592 CTAs that stay, several times over; vocabularies of a few entries more
# than whole pieces, whose last piece is empty in the rows that start with single entries
PIECES = [(700, 4099), (700, 8195), (1300, 2049), (300, 33001), (650, 16389)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", PIECES)
@pytest.mark.parametrize("shared", [False, True])
def test_masked_gradients_of_many_pieces(dtype, rows, vocab, shared):
    x, token, mask, g = make(dtype, rows, vocab, rows + vocab, pad=1 + vocab % 4, shift=3)
    odd = torch.zeros(rows, vocab + 5, device="cuda", dtype=torch.uint8)[:, 2:2 + vocab]       # its words shift from row to row
    odd.copy_(mask)
    mask = odd[3:4] if shared else odd
    if not shared:
        mask[5::17] = 0                                            # rows without support between the others
    token[2::13] = -1
    x[7::11] = -INF
    dlogp, dent = torch.randn(rows, device="cuda", generator=g), torch.randn(rows, device="cuda", generator=g)
    norm, ent = fp32_norm(x, mask, 0.8)
    got = xrl.xrl_logprob_grad(x, norm, token, dlogp, ent, dent, mask=mask, scale=0.8)
    for first in range(0, rows, 100):                              # (a hundred rows of 64-bit numbers at a time)
        r = slice(first, first + 100)
        m = mask if shared else mask[r]
        near(got[r], *reference_grad(x[r], token[r], m, 0.8, norm[r], ent[r], dlogp[r], dent[r]), "gradient")
    over = torch.empty(rows, vocab + 9, device="cuda", dtype=x.dtype)[:, 2:2 + vocab]
    over.copy_(x)
    xrl.xrl_logprob_grad(over, norm, token, dlogp, ent, dent, mask=mask, scale=0.8, grad=over)
    assert torch.equal(over, got)
