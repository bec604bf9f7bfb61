"""Attention whose scores leap far above those of the keys before: the running base of the exponentials has to follow, whichever key of a
block the far score belongs to (part of the exponentials are taken by another way than the rest)."""
import pytest
import torch

from paper_2606_26344_b200 import gmlp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


@pytest.mark.parametrize("far", [100.0, 150.0, 200.0, 350.0, 500.0, 3000.0])
@pytest.mark.parametrize("key", [128, 129, 130, 131, 136, 137, 144, 255])
def test_one_far_key(key, far):
    """Keys score 0 but one of the second block, whose score is `far` binary orders: the output is that key's value."""
    S, M = 256, 300
    K = torch.zeros(S, 128, device=DEV, dtype=torch.bfloat16)
    Q = torch.zeros(M, 128, device=DEV, dtype=torch.bfloat16)
    V = torch.randn(S, 128, device=DEV, generator=torch.Generator(device=DEV).manual_seed(key)).to(torch.bfloat16)
    Q[:, 0], K[key, 0] = 16.0, far * 0.6931471805599453 * 128 ** 0.5 / 16     # score / sqrt(128) * log2(e) = far
    O = gmlp.gqa_attention(Q, K, V, 1, 1, checked=True)
    assert torch.equal(O, V[key].expand(M, 128))                             # the others weigh 2^-99 or less
