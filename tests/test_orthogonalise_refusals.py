"""What xrl_orthogonalise refuses, before any CUDA call (no GPU needed), and where the layers lie in a gradient blob."""
import ctypes as C

import numpy as np
import pytest

P = 1 << 20                                # stands for a device address: nothing is read before the refusals


@pytest.fixture(scope="module")
def lib():
    from paper_2304_14698_b200 import binding, build
    build.build()
    return binding.load_library()


def size(lib, dtype=0, batch=2, rows=40, cols=50):
    n = C.c_size_t(77)
    return lib.xrl_orthogonalise_workspace(dtype, batch, rows, cols, C.byref(n)), n.value


def call(lib, device=0, dtype=0, batch=2, rows=40, cols=50, grad=P, ld=50, bs=2000, steps=5, eps=1e-7, out=2 * P, old=50, obs=2000,
         ws=4 * P, ws_bytes=1 << 30, status=None):
    return lib.xrl_orthogonalise(device, dtype, batch, rows, cols, grad, ld, bs, steps, C.c_float(eps), out, old, obs, ws, ws_bytes,
                                 status, None)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(batch=-1), dict(rows=-1), dict(cols=-1), dict(grad=None), dict(out=None), dict(ws=None), dict(ld=49),
    dict(old=49), dict(bs=1999), dict(obs=1999), dict(bs=-2000), dict(steps=0), dict(steps=65), dict(eps=0.0), dict(eps=-1.0),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(ws=4 * P + 128), dict(ws_bytes=1000), dict(grad=P + 2),
    dict(out=2 * P + 1, dtype=1), dict(status=P + 2)])
def test_refused(lib, bad):
    assert call(lib, **bad) == 1


@pytest.mark.parametrize("bad", [dict(batch=65536), dict(rows=32769), dict(cols=32769), dict(batch=60000, rows=32768, cols=32768)])
def test_too_large(lib, bad):
    assert call(lib, **bad) == 8 and size(lib, **bad)[0] == 8


def test_workspace_sizes(lib):
    st, n = size(lib)
    assert st == 0 and call(lib, ws_bytes=n - 1) == 1
    assert size(lib, batch=0) == (0, 0) and size(lib, rows=0) == (0, 0)
    assert lib.xrl_orthogonalise_workspace(0, 1, 1, 1, None) == 1
    a, b = size(lib, batch=1, rows=4096, cols=4096)[1], 4096 * 4096
    assert 16 * b <= a <= 17 * b                        # X twice, F and B, four bytes each
    assert size(lib, batch=7, rows=32768, cols=32768)[1] > 2 ** 32


def test_nothing_to_do_needs_nothing(lib):
    for empty in (dict(batch=0), dict(rows=0), dict(cols=0)):
        assert call(lib, grad=None, out=None, ws=None, **empty) == 0


def test_without_a_device_it_fails_loudly(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert call(lib) == 5


def test_the_binding_refuses_other_types_shapes_and_places():
    import torch
    import paper_2304_14698_b200 as xrl
    for bad in (torch.zeros(3), torch.zeros(2, 3), torch.zeros(1, 2, 3, 4)):
        with pytest.raises(xrl.XrlError):
            xrl.xrl_orthogonalise(bad)
    from paper_2304_14698_b200 import binding as b
    with pytest.raises(xrl.XrlError):
        b._matrices_of("f", "grad", torch.zeros(5, 4).T, 1, 4, 5)
    with pytest.raises(xrl.XrlError):
        b._matrices_of("f", "out", torch.zeros(2, 4, 5), 2, 4, 6)
    with pytest.raises(xrl.XrlError):
        xrl.orthogonalise_layers(dict(T=8, S=8, H=32, L=1), torch.zeros(4, 4))


@pytest.mark.parametrize("L", [1, 3])
def test_layer_matrices_are_the_blobs(L):
    import torch
    import paper_2304_14698_b200 as xrl
    from workloads import configs
    m = dict(T=13, S=8, H=64, K=2, L=L, Hm=32, Dg=1, dtype="fp32", A_max=8)
    blob, parts = configs.make_weights(m, 3)
    w = xrl.layer_matrices(m, torch.from_numpy(blob))
    for l in range(L):
        assert np.array_equal(w[l].numpy(), parts[f"W{l + 1}"])
