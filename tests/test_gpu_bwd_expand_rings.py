"""The grad-input GEMM that expands the INT8 weight inside the kernel, where its converters' waits have to tell one round of the ring from the next: contractions of 1 to
64 blocks with and without the stages of the adapters, weights from HBM and from L2.  The same products in the same order as through a bf16 copy of the weight, so
the same bits, every time."""
import pytest

import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [64, 128, 192, 448, 1024, 4096])
@pytest.mark.parametrize("r", [0, 16])
@pytest.mark.parametrize("M,K", [(300, 1024), (2048, 6144)])
def test_expanding_in_the_kernel_gives_the_bits_of_the_copy(M, K, N, r):
    from paper_2505_14742_b200.layer import QuaffLinear
    g = torch.Generator(device="cuda").manual_seed(N + r)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    W, X, dY = rn(N, K), rn(M, K), rn(M, N)
    A, B = (rn(K, r), rn(r, N)) if r else (None, None)
    copy, lean = (QuaffLinear(W, None, A, B, 0.5, 0.9, M, lean_bwd=x) for x in (False, True))
    scrub = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    for layer in (copy, lean):
        layer.forward(X)
    want = copy.backward(dY)[0].clone()
    for i in range(12):
        if i % 3 == 0:
            scrub.fill_(i)
        lean.dX.fill_(7.0)
        assert torch.equal(lean.backward(dY)[0], want)
    assert int(lean.status[0]) == 0 and int(copy.status[0]) == 0
