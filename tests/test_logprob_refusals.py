"""What xrl_logprob and xrl_logprob_grad refuse, before any CUDA call (no GPU needed)."""
import ctypes as C

import pytest

ROWS, VOCAB = 4, 100
P = 1 << 20                                # stands for a device address: nothing is read before the refusals


@pytest.fixture(scope="module")
def lib():
    from paper_2304_14698_b200 import binding, build
    build.build()
    return binding.load_library()


def score(lib, device=0, dtype=0, rows=ROWS, vocab=VOCAB, logits=P, stride=VOCAB, token=P, mask=None, mstride=0, scale=1.0,
          top=0, logp=P, entropy=P, norm=P, top_token=None, top_logp=None):
    return lib.xrl_logprob(device, dtype, rows, vocab, logits, stride, token, mask, mstride, C.c_float(scale), top, logp, entropy,
                           norm, top_token, top_logp, None)


def grad(lib, device=0, dtype=0, rows=ROWS, vocab=VOCAB, logits=P, stride=VOCAB, token=P, mask=None, mstride=0, scale=1.0,
         norm=P, dlogp=P, entropy=P, dentropy=P, out=2 * P, gstride=VOCAB):
    return lib.xrl_logprob_grad(device, dtype, rows, vocab, logits, stride, token, mask, mstride, C.c_float(scale), norm, dlogp,
                                entropy, dentropy, out, gstride, None)


COMMON = [dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(vocab=0), dict(logits=None), dict(stride=VOCAB - 1), dict(stride=-VOCAB),
          dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=2e6), dict(scale=9e-7),
          dict(mask=P, mstride=VOCAB - 1), dict(mask=P, mstride=-1), dict(logits=P + 2), dict(logits=P + 1, dtype=1), dict(norm=P + 4)]


@pytest.mark.parametrize("bad", COMMON + [dict(token=None), dict(top=-1), dict(top=VOCAB + 1, top_token=P, top_logp=P), dict(top=3),
                                          dict(top=3, top_token=P), dict(top=3, top_logp=P)])
def test_scoring_refuses(lib, bad):
    assert score(lib, **bad) == 1


@pytest.mark.parametrize("bad", COMMON + [dict(norm=None), dict(out=None), dict(token=None), dict(entropy=None),
                                          dict(gstride=VOCAB - 1), dict(out=P, gstride=VOCAB + 1), dict(out=2 * P + 2)])
def test_the_gradient_refuses(lib, bad):
    assert grad(lib, **bad) == 1


def test_more_alternatives_than_a_warp_holds(lib):
    assert score(lib, top=33, top_token=P, top_logp=P) == 8


def test_without_a_device_it_fails_loudly(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert score(lib) == 5 and grad(lib) == 5


def test_the_binding_refuses_tensors_of_other_shapes_types_and_places():
    import torch
    import paper_2304_14698_b200 as xrl
    x = torch.zeros(ROWS, VOCAB)
    with pytest.raises(xrl.XrlError):
        xrl.xrl_logprob(x)                                  # not on a GPU
    with pytest.raises(xrl.XrlError):
        xrl.xrl_logprob(x[0])
    with pytest.raises(xrl.XrlError):
        xrl.xrl_logprob_grad(x, torch.zeros(ROWS, 2))
    from paper_2304_14698_b200 import binding as b
    for call in (lambda: b._flat("f", "token", torch.zeros(ROWS, dtype=torch.int64), torch.int32, (ROWS,)),
                 lambda: b._flat("f", "token", torch.zeros(2 * ROWS, dtype=torch.int32)[::2], torch.int32, (ROWS,)),
                 lambda: b._flat("f", "token", torch.zeros(ROWS + 1, dtype=torch.int32), torch.int32, (ROWS,)),
                 lambda: b._rows_of("f", "x", torch.zeros(VOCAB, ROWS).T, ROWS, VOCAB),
                 lambda: b._mask_of("f", torch.zeros(ROWS, VOCAB), ROWS, VOCAB),
                 lambda: b._mask_of("f", torch.zeros(ROWS, VOCAB + 1, dtype=torch.uint8), ROWS, VOCAB),
                 lambda: b._mask_of("f", torch.zeros(2, VOCAB, dtype=torch.uint8), ROWS, VOCAB)):
        with pytest.raises(xrl.XrlError) as e:
            call()
        assert e.value.status == 1
    with pytest.raises(xrl.XrlError) as e:
        b._storage("f", torch.zeros(1, dtype=torch.float16))
    assert e.value.status == 8
    mask = torch.zeros(ROWS, VOCAB, dtype=torch.bool)
    assert b._mask_of("f", mask, ROWS, VOCAB) == (mask.data_ptr(), VOCAB)
    assert b._mask_of("f", mask[0], ROWS, VOCAB)[1] == 0 and b._mask_of("f", mask[:1], ROWS, VOCAB)[1] == 0
    assert b._mask_of("f", mask[:1].expand(ROWS, VOCAB), ROWS, VOCAB)[1] == 0
