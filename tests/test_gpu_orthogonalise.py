"""xrl_orthogonalise against its definition in 64 bits.

Tolerances.  An update's error is given relative to its norm.  fp32: operands of 22 bits (2^-23 of an entry off) and fp32
accumulation; the map's slope is 3.4445^steps at the smallest singular values (485 for five steps), which multiplies what was lost
in directions that hold little of G.  With R the result's norm, that is at most 485 * 2^-23 * sqrt(3 products) < 1.1e-4 if all of
it sat there; the smallest directions of a matrix hold far less, and 2e-5 is what fp32 updates are held to.  bf16: operands of 11
bits, 2^-12 off in the mean square sense 2^-12 / sqrt(3) = 1.4e-4 per product; three products a step, slopes of up to 3.4 for the
last step's and 12 for the one before it: sqrt(3) * (1 + 3.4 + 12) * 1.4e-4 = 4e-3 if no later step damped them, and the result's
own rounding 2^-9 (mean square: 1.7e-3)."""
import pytest
import torch

import paper_2304_14698_b200 as xrl

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
TOL = {"fp32": 2e-5, "bf16": 4e-3 + 1.7e-3}


def define(g, steps=5, eps=1e-7):
    out = []
    for x in g.double().reshape(-1, *g.shape[-2:]):
        x = x / (torch.linalg.matrix_norm(x) + eps)
        for _ in range(steps):
            if x.shape[0] > x.shape[1]:
                a = x.T @ x
                x = 3.4445 * x + x @ (-4.7750 * a + 2.0315 * a @ a)
            else:
                a = x @ x.T
                x = 3.4445 * x + (-4.7750 * a + 2.0315 * a @ a) @ x
        out.append(x)
    return torch.stack(out).reshape(g.shape)


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def make(dtype, *shape, seed=0, kind="gradient"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x = n(*shape)
    if kind == "gradient":
        k = min(8, *shape[-2:])
        x = 0.02 * x + 0.02 * n(*shape[:-1], k) @ n(*shape[:-2], k, shape[-1])
    return x.to(DTYPES[dtype])


SHAPES = [(1, 1), (1, 7), (7, 1), (2, 3), (8, 8), (33, 31), (64, 64), (127, 129), (129, 127), (128, 128), (200, 136), (56, 256),
          (256, 256), (100, 1000), (1000, 100), (512, 512), (385, 513), (513, 385), (1024, 640), (640, 1025), (1500, 1500), (32, 8192), (2070, 2500), (2500, 2070)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_every_shape(dtype, rows, cols):
    for kind in ("gradient", "normal"):
        g = make(dtype, rows, cols, seed=rows + cols, kind=kind)
        status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
        got = xrl.xrl_orthogonalise(g, device_status=status)
        assert got.dtype == g.dtype and got.shape == g.shape and int(status) == 0
        assert off(got, define(g)) <= TOL[dtype], kind


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("steps", [1, 2, 3, 6, 10])
def test_every_number_of_steps(dtype, steps):
    g = make(dtype, 3, 150, 260, seed=steps)
    assert off(xrl.xrl_orthogonalise(g, steps=steps), define(g, steps)) <= TOL[dtype]


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_steps_stay_where_the_quintic_keeps_them(dtype):
    """From above 0.5 the quintic stays between 0.67 and 1.21; nothing leaves that however often it is applied."""
    s = torch.linalg.svdvals(xrl.xrl_orthogonalise(make(dtype, 200, 333, seed=9, kind="normal"), steps=64).double())
    assert 0.65 < float(s.min()) and float(s.max()) < 1.23


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(5, 256, 256), (7, 65, 70), (3, 700, 90), (2, 1, 1), (40, 32, 48), (45, 200, 150)])
def test_batches_are_their_matrices(dtype, shape):
    g = make(dtype, *shape, seed=1)
    got = xrl.xrl_orthogonalise(g)
    assert off(got, define(g)) <= TOL[dtype]
    for z in range(shape[0]):
        # alone a matrix may be cut into other tiles, whose sums are added in another order
        alone = xrl.xrl_orthogonalise(g[z])
        assert off(alone, got[z].double()) <= 2 * TOL[dtype]
        same = xrl.xrl_orthogonalise(g[z][None].expand(shape[0], -1, -1).contiguous())
        assert torch.equal(same[z], got[z])                       # but not by what the others hold


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(130, 260), (300, 70), (64, 64)])
def test_strides_views_and_results_over_the_input(dtype, rows, cols):
    g = make(dtype, 2, rows, cols, seed=2)
    want = xrl.xrl_orthogonalise(g)
    wide = torch.full((2, rows + 3, cols + 13), 7.0, device="cuda", dtype=g.dtype)
    inner = wide[:, 1:1 + rows, 3:3 + cols]
    inner.copy_(g)
    assert torch.equal(xrl.xrl_orthogonalise(inner), want)
    assert xrl.xrl_orthogonalise(inner, out=inner) is inner
    assert torch.equal(inner, want)
    edge = wide.clone()
    edge[:, 1:1 + rows, 3:3 + cols] = 7
    assert bool((edge == 7).all())                              # nothing outside the matrices was written


@pytest.mark.parametrize("dtype", DTYPES)
def test_zero_tiny_huge_and_broken_matrices(dtype):
    g = make(dtype, 6, 96, 200, seed=3, kind="normal")
    want = define(g)
    g[0] = 0
    g[1] *= 2.0 ** 100
    g[2] *= 2.0 ** -15
    g[3, 5, 7] = float("nan")
    g[4, 0, 0] = float("inf")
    got = xrl.xrl_orthogonalise(g)
    assert bool((got[0] == 0).all())
    assert bool(torch.isnan(got[3:5]).all())
    for z in (1, 2, 5):
        assert off(got[z], define(g[z])) <= TOL[dtype]
    assert off(got[5], want[5]) <= TOL[dtype]
    # far below eps: X_0 = G / eps stays small and grows by 3.4445 a step.  Operands are fixed-point at that end, multiples of
    # 2^-24 of entries scaled by 2^7 (the nearest power of two to sqrt(96 * 200)): off by 2^-32 each, and by 485 times that after
    # five steps, twice as much for what the steps themselves round
    g[2] *= 2.0 ** -60
    got, want = xrl.xrl_orthogonalise(g[2]).double(), define(g[2])
    assert float((got - want).norm()) <= 2 * 485 * 2.0 ** -32 * (96 * 200) ** 0.5


@pytest.mark.parametrize("dtype", DTYPES)
def test_singular_values_come_near_one_and_rank_is_kept(dtype):
    g = (make(dtype, 300, 20, seed=4, kind="normal").float() @ make(dtype, 20, 200, seed=5, kind="normal").float()).to(DTYPES[dtype])
    s = torch.linalg.svdvals(xrl.xrl_orthogonalise(g).double())
    assert float(s[:20].min()) > 0.6 and float(s[:20].max()) < 1.25
    if dtype == "fp32":
        assert float(s[25:].max()) < 1e-2


def test_the_same_bits_every_time_on_streams_in_graphs_and_with_workspaces():
    g = make("bf16", 2, 700, 300, seed=6)
    want = xrl.xrl_orthogonalise(g)
    for _ in range(3):
        assert torch.equal(xrl.xrl_orthogonalise(g), want)
    size = xrl.xrl_orthogonalise_workspace(1, 2, 700, 300)
    ws = torch.full((size + 256,), 255, dtype=torch.uint8, device="cuda")      # NaN patterns: nothing is read before it is written
    assert torch.equal(xrl.xrl_orthogonalise(g, workspace=ws[:size]), want)
    assert bool((ws[size:] == 255).all())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = xrl.xrl_orthogonalise(g, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got, want)
    graphs = []
    for _ in range(2):                                                         # two graphs, a workspace each
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = xrl.xrl_orthogonalise(g)
        graphs.append((graph, out))
    g.copy_(make("bf16", 2, 700, 300, seed=7))
    want = xrl.xrl_orthogonalise(g)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for (graph, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out, want) for _, out in graphs)


def test_empty_batches():
    for shape in ((0, 5, 5), (2, 0, 5), (2, 5, 0)):
        assert xrl.xrl_orthogonalise(torch.zeros(shape, device="cuda")).shape == shape


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 16, 4000), (1, 4000, 16), (3, 130, 2100), (1, 2100, 130), (1, 500, 1111), (1, 100, 513), (8, 64, 900),
                                   (1, 60, 32768), (1, 1, 5000), (1, 700, 3500), (1, 3500, 650), (1, 400, 7000), (1, 7000, 390)])
def test_long_reductions_are_shared_out(dtype, shape):
    for kind in ("gradient", "normal"):
        g = make(dtype, *shape, seed=shape[1], kind=kind)
        got = xrl.xrl_orthogonalise(g)
        assert off(got, define(g)) <= TOL[dtype], kind
        assert torch.equal(xrl.xrl_orthogonalise(g), got)
