"""What the calls of the layer behind the attention refuse of tensors on the GPU: an exception, and nothing enqueued."""
import pytest
import torch

from paper_2603_12118_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def z(*shape, dtype=BF16):
    return torch.zeros(*shape, dtype=dtype, device=DEV)


def odd(*shape, dtype=BF16):
    """A tensor one element past a multiple of 16 bytes."""
    n = 1
    for s in shape:
        n *= s
    return z(n + 1, dtype=dtype)[1:].view(*shape)


def test_norm_residual():
    good = dict(x=z(3, 64), residual=z(3, 64, dtype=F32), pre_gain=z(64, dtype=F32))
    kept = torch.full((3, 64), 7.0, dtype=BF16, device=DEV)
    B.cs_norm_residual(**good)
    for error, change in [
            (TypeError, dict(x="rows")), (TypeError, dict(x=z(3, 64).half())), (TypeError, dict(residual=z(3, 64).half())), (TypeError, dict(eps="small")),
            (TypeError, dict(pre_gain=None)), (TypeError, dict(residual=None)),
            (ValueError, dict(x=z(3, 64).cpu())), (ValueError, dict(residual=z(3, 64).cpu())), (ValueError, dict(x=z(192))), (ValueError, dict(residual=z(2, 64))),
            (ValueError, dict(x=z(3, 128)[:, ::2])), (ValueError, dict(pre_gain=z(64))), (ValueError, dict(pre_gain=z(32, dtype=F32))),
            (ValueError, dict(post_gain=z(64))), (ValueError, dict(pre_bias=z(1, dtype=F32))), (ValueError, dict(gate=z(64, dtype=F32))),
            (ValueError, dict(gate=z(32))), (ValueError, dict(gate=z(2, 64))), (ValueError, dict(r=z(3, 64))), (ValueError, dict(norm="l2")),
            (B.CsError, dict(post_bias=z(64, dtype=F32))), (B.CsError, dict(x=odd(3, 64))), (B.CsError, dict(residual=odd(3, 64))), (B.CsError, dict(eps=-1.0)),
            (B.CsError, dict(residual_scale=float("inf"))), (B.CsError, dict(x=z(1, 64).expand(3, 64))), (B.CsError, dict(x=z(3, 68)[:, :64])),
            (B.CsError, dict(gate=z(1, 64).expand(3, 64)))]:
        with pytest.raises(error):
            B.cs_norm_residual(**{**good, "y": kept, **change})
        assert (kept == 7).all(), change
    with pytest.raises(B.CsError):
        B.cs_norm_residual(z(3, 60), z(3, 60), z(60, dtype=F32))


def test_weights():
    for error, args in [(TypeError, (z(16, 64).half(),)), (TypeError, (None,)), (ValueError, (z(64),)), (ValueError, (z(16, 64).cpu(),)),
                        (ValueError, (z(16, 64), "e4m3")), (ValueError, (z(16, 128)[:, ::2],)), (B.CsError, (z(16, 48),)), (B.CsError, (odd(16, 64),)),
                        (B.CsError, (z(0, 64),)), (B.CsError, (z(1, 64).expand(16, 64),)), (ValueError, (z(16, 64), "e2m1", z(1)))]:
        with pytest.raises(error):
            B.cs_weights_pack(*args)
    p = B.cs_weights_pack(z(16, 64))
    kept = torch.full((1, 16, 64), 7.0, dtype=F32, device=DEV)
    for error, change in [(TypeError, dict(dtype=torch.float16)), (TypeError, dict(packed=p.data)), (ValueError, dict(out=kept, dtype=BF16)),
                          (ValueError, dict(out=kept[0])), (ValueError, dict(out=kept.cpu())), (ValueError, dict(out=kept[:, :8])),
                          (ValueError, dict(packed=B.PackedWeights(p.data[:-1], "e2m1", 1, 16, 64), out=kept)),
                          (ValueError, dict(packed=B.PackedWeights(p.data, "e2m1", 2, 16, 64), out=kept)),
                          (ValueError, dict(packed=B.PackedWeights(p.data.cpu(), "e2m1", 1, 16, 64), out=kept))]:
        with pytest.raises(error):
            B.cs_weights_read(**{"packed": p, **change})
        assert (kept == 7).all(), change


def test_linear():
    p, two = B.cs_weights_pack(z(48, 64)), B.cs_weights_pack(z(2, 48, 64))
    kept = torch.full((3, 48), 7.0, dtype=BF16, device=DEV)
    for error, change in [
            (TypeError, dict(x=z(3, 64, dtype=F32))), (TypeError, dict(weights=z(48, 64))), (TypeError, dict(dtype=torch.int32)), (ValueError, dict(x=z(3, 32))),
            (ValueError, dict(x=z(64))), (ValueError, dict(x=z(3, 64).cpu())), (ValueError, dict(x=z(3, 128)[:, ::2])), (ValueError, dict(bias=z(48))),
            (ValueError, dict(bias=z(47, dtype=F32))), (ValueError, dict(dtype=F32)), (ValueError, dict(out=z(2, 48))), (B.CsError, dict(weights=two)),
            (B.CsError, dict(x=odd(3, 64))), (B.CsError, dict(x=z(3, 68)[:, :64])), (B.CsError, dict(out=z(1, 48).expand(3, 48)))]:
        with pytest.raises(error):
            B.cs_linear_packed(**{"x": z(3, 64), "weights": p, "out": kept, **change})
        assert (kept == 7).all(), change
    with pytest.raises(ValueError):
        B.cs_linear_packed(z(30, 8192), B.cs_weights_pack(z(48, 8192)), workspace=torch.zeros(1 << 24, dtype=torch.uint8))


def test_moe():
    up, down = B.cs_weights_pack(z(9, 64, 64)), B.cs_weights_pack(z(9, 64, 32))
    good = dict(x=z(3, 64), router=z(8, 64), up=up, down=down, top=2)
    kept = torch.full((3, 64), 7.0, dtype=BF16, device=DEV)
    B.cs_moe(**good)
    for error, change in [
            (TypeError, dict(x=z(3, 64, dtype=F32))), (TypeError, dict(up=z(9, 64, 64))), (TypeError, dict(top="2")), (TypeError, dict(scale="x")),
            (ValueError, dict(x=z(3, 32))), (ValueError, dict(x=z(3, 64).cpu())), (ValueError, dict(router=z(8, 64, dtype=F32))),
            (ValueError, dict(router=z(10, 64))), (ValueError, dict(router=z(8, 32))), (ValueError, dict(up=down)), (ValueError, dict(down=up)),
            (ValueError, dict(down=B.cs_weights_pack(z(8, 64, 32)))), (ValueError, dict(down=B.cs_weights_pack(z(9, 64, 32), "bf16"))),
            (ValueError, dict(top=0)), (ValueError, dict(top=9)), (ValueError, dict(choice_bias=z(8))), (ValueError, dict(choice_bias=z(9, dtype=F32))),
            (ValueError, dict(live=torch.ones(2, dtype=torch.bool, device=DEV))), (ValueError, dict(live=torch.ones(3, dtype=torch.bool))),
            (ValueError, dict(live=z(3))), (ValueError, dict(y=z(3, 64, dtype=F32))), (ValueError, dict(experts=z(3, 2, dtype=F32))),
            (ValueError, dict(weights=z(3, 1, dtype=F32))), (ValueError, dict(score="relu")), (B.CsError, dict(x=odd(3, 64))), (B.CsError, dict(scale=float("nan"))),
            (B.CsError, dict(router=odd(8, 64)))]:
        with pytest.raises(error):
            B.cs_moe(**{**good, "y": kept, **change})
        assert (kept == 7).all(), change
    for hidden, inter in ((48, 32), (64, 48)):
        with pytest.raises(B.CsError):
            B.cs_weights_pack(z(4, 64, 48))
