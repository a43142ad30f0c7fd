"""How far xrl_orthogonalise's updates are off for matrices whose roundings do not average out: entries of one size, low rank.

Definitions and tolerances are those of test_gpu_orthogonalise, where nothing else is said."""
import pytest
import torch

import paper_2304_14698_b200 as xrl
from test_gpu_orthogonalise import DTYPES, TOL, define, off

pytestmark = pytest.mark.gpu


def one_size_bound(steps=5):
    """Relative error of a rank-one update whose entries all have one size, where no rounding averages out.  X's hi part, F's and B's
    are off by up to u = 2^-12 of themselves, everywhere the same.  With s the square of the singular value x, a step's
    g = a + b s + c s^2 has b's term off by 4 u (X twice in A, X once and B once in the product) and c's by 8 u (X four times,
    F twice, X and B once); x g carries what the steps before left by |x f'(x) / f(x)|."""
    a, b, c, u = 3.4445, -4.7750, 2.0315, 2.0 ** -12
    x, e = 1.0, 0.0
    for _ in range(steps):
        s = x * x
        f = x * (a + b * s + c * s * s)
        e = abs(x * (a + 3 * b * s + 5 * c * s * s) / f) * e + x * (4 * abs(b) * s + 8 * c * s * s) * u / abs(f)
        x = f
    return e


@pytest.mark.parametrize("rows,cols", [(64, 64), (56, 256), (256, 256), (300, 700), (700, 300), (512, 512), (2048, 1500), (32, 8192)])
def test_entries_of_one_size(rows, cols):
    """All of one value, and of both signs in a pattern of rank one: bf16 updates are off by the bound above and their own rounding
    (2^-8 of an entry at most), fp32 ones by what they always are."""
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    sign = lambda n: torch.where(torch.rand(n, device="cuda", generator=g) < 0.5, 1.0, -1.0)  # noqa: E731
    for x in (torch.full((rows, cols), 0.37, device="cuda"), 0.01 * sign(rows)[:, None] * sign(cols)):
        for dtype, tol in (("bf16", one_size_bound() + 2.0 ** -8), ("fp32", TOL["fp32"])):
            m = x.to(DTYPES[dtype])
            e = off(xrl.xrl_orthogonalise(m), define(m))
            print(f"{dtype} {rows} x {cols}: {e:.2e}")
            assert e <= tol, dtype


@pytest.mark.parametrize("rows,cols,rank", [(200, 300, 4), (300, 200, 20), (512, 512, 4), (1024, 1024, 8), (128, 1024, 3)])
def test_rank_is_kept(rows, cols, rank):
    """Matrices of low rank without any rounding (products of small whole numbers): what the update has outside their space comes
    from its own roundings alone, which the map multiplies by 3.4445 a step.  For fp32 updates that is the bound which
    test_gpu_orthogonalise derives for what sits in such directions, 485 * 2^-23 * sqrt(3) < 1.1e-4 (2e-5 is for matrices that fill
    theirs).  Singular values differ by no more than the norm of the difference does (Weyl), and the definition's are 0 there."""
    tol = {"fp32": 1.1e-4, "bf16": TOL["bf16"]}
    g = torch.Generator(device="cuda").manual_seed(rows + cols + rank)
    ints = lambda *s: torch.randint(-3, 4, s, device="cuda", generator=g).float()  # noqa: E731
    x = ints(rows, rank) @ ints(rank, cols)
    for dtype in DTYPES:
        m = x.to(DTYPES[dtype])
        assert torch.equal(m.float(), x)
        got, want = xrl.xrl_orthogonalise(m).double(), define(m)
        print(f"{dtype} {rows} x {cols} of rank {rank}: {off(got, want):.2e}")
        assert off(got, want) <= tol[dtype]
        s = torch.linalg.svdvals(got)
        assert float(s[rank]) <= tol[dtype] * float(want.norm())
