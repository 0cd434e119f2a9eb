"""Tensors of forward-mode differentiation are refused by every call that would drop their derivatives."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2201_12023_amd import blocks as B
from paper_2201_12023_amd import layers as L

H, M, W = torch.ones(4, 2, 8), torch.ones(4, 8), torch.ones(6, 8)
POS, F, OFF, STAT = torch.arange(4), torch.ones(4, dtype=torch.float64), torch.tensor([0, 4], dtype=torch.int32), torch.ones(4)
# (call, its arguments, which of them have derivatives)
CALLS = [(L.alpa_linear_forward, dict(x=M, w=W, bias=W[:, 0], residual=torch.ones(4, 6)), ("x", "w", "bias", "residual")),
         (L.alpa_linear_backward, dict(dy=torch.ones(4, 6), x=M, w=W, z=torch.ones(4, 6)), ("dy", "x", "w", "z")),
         (L.alpa_experts_forward, dict(x=M, w=W[None], offsets=OFF, bias=W[None, :, 0]), ("x", "w", "bias")),
         (L.alpa_experts_backward, dict(dy=torch.ones(4, 6), x=M, w=W[None], offsets=OFF), ("dy", "x", "w")),
         (L.alpa_vocab_loss_forward, dict(x=M, w=W, target=POS), ("x", "w")),
         (L.alpa_vocab_loss_backward, dict(dloss=STAT, x=M, w=W, target=POS, lse=STAT), ("dloss", "x", "w", "lse")),
         (B.alpa_attention_forward, dict(q=H, k=H, v=H, slopes=torch.ones(2)), ("q", "k", "v", "slopes")),
         (B.alpa_attention_backward, dict(dy=H, q=H, k=H, v=H, y=H, lse=M[:, :2]), ("dy", "q", "k", "v", "y", "lse")),
         (B.alpa_rotary_forward, dict(x=H, positions=POS, frequencies=F), ("x", "frequencies")),
         (B.alpa_rotary_backward, dict(dy=H, positions=POS, frequencies=F), ("dy", "frequencies")),
         (B.alpa_norm_forward, dict(x=M, weight=M[0], bias=M[0]), ("x", "weight", "bias")),
         (B.alpa_norm_backward, dict(dy=M, x=M, mean=STAT, rstd=STAT, weight=M[0]), ("dy", "x", "mean", "rstd", "weight"))]


@pytest.mark.parametrize("call, args, names", CALLS, ids=[c[0].__name__ for c in CALLS])
@pytest.mark.parametrize("leaf", [False, True])
def test_derivatives_are_not_dropped(call, args, names, leaf):
    with forward_ad.dual_level():
        for name in names:
            t = args[name].clone().requires_grad_() if leaf else args[name]
            with pytest.raises(RuntimeError, match="forward-mode"):
                call(**{**args, name: forward_ad.make_dual(t, torch.ones_like(t))})
        # without one: refused for not being on a GPU, as ever
        with pytest.raises(ValueError, match="GPU"):
            call(**args)
        with pytest.raises(ValueError, match="GPU"):
            call(**{name: forward_ad.unpack_dual(t).primal if name in names else t for name, t in args.items()})


def test_frequencies_are_constants():
    f = F.clone().requires_grad_()
    with pytest.raises(ValueError, match="frequencies have no gradient"):
        B.alpa_rotary_forward(H, POS, f)
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
        B.alpa_rotary_forward(H, POS, f)
