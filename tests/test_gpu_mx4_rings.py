"""The layer's product where the stages of the adapters fall anywhere in its ring: the warp that copies the block scales passes over them and must not take the
barrier of an earlier stage for that of its own.  Contractions of 1 to 17 stages per tile with two and three stages of the adapters, several tiles per pair of
CTAs; every call has to agree bit for bit with a product of the same operands plus nothing, in which no stage is passed over, and report no wait that ran out."""
import pytest

import torch

from paper_2505_14742_b200 import binding as Q

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N", [(2960, 10968), (1500, 8000)])
@pytest.mark.parametrize("stages", [1, 2, 3, 4, 6, 8, 9, 17])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_scales_are_those_of_their_stage(M, N, stages, out):
    from paper_2505_14742_b200.layer import Mx4Linear
    g = torch.Generator(device="cuda").manual_seed(stages)
    K, r = 256 * stages - 56, 16
    # block scales over six powers of two, so that those of another stage show
    X = (torch.randn((M, K), generator=g, device="cuda") * torch.exp2(torch.randint(-3, 4, (M, K // 8), generator=g, device="cuda").float()).repeat_interleave(8, 1)).to(torch.bfloat16)
    W = (torch.randn((N, K), generator=g, device="cuda") * torch.exp2(torch.randint(-3, 4, (N, K // 8), generator=g, device="cuda").float()).repeat_interleave(8, 1)).to(torch.bfloat16)
    A = (torch.randn((K, r), generator=g, device="cuda") * 0.1).to(torch.bfloat16)
    B = torch.zeros((r, N), dtype=torch.bfloat16, device="cuda")
    layer = Mx4Linear(W, A, B, 1.0, M, y_dtype=out, train=False)
    codes, scales = Q.mx4_empty(M, K)
    Q.quaff_mx4_quantize(X, codes, scales)
    want, status = torch.empty((M, N), dtype=out, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    Q.quaff_mx4_matmul(codes, scales, layer.Wc, layer.Ws, K, want, None, status)
    assert int(status[0]) == 0
    scrub = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    for i in range(8):
        if i % 2:
            scrub.fill_(i)                                     # operands from HBM, from L2
        Y = layer.forward(X)
        assert torch.equal(Y, want)
    assert int(layer.status[0]) == 0
