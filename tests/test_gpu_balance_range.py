"""The balance loss and its gradient where an intermediate of the formula leaves FP32's range and
the result does not."""
import math

import pytest
import torch

import _moe as M
import _q8 as Q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    return E


@pytest.mark.parametrize("T", [2, 100, 300, 5000])
@pytest.mark.parametrize("E", [8, 200, 1000])
def test_mean_square_within_the_range(emu, T, E):
    """z of 1.5e19 everywhere (the sum of two squares is beyond 3.4e38, their mean 2.25e38); then
    every third token 2.5e19, the others 0.  The lone logit is z, so z is exact, and its
    square is in FP64; the mean of 5000 is off by 5003 units of 2^-53 and rounded to FP32."""
    for top, every in ((1.5e19, 1), (2.5e19, 3)):
        x = torch.full((T, E), -math.inf)
        x[:, 3] = 0
        x[::every, 3] = top
        b = emu.moe_balance(x.cuda(), torch.full((T, 1), 3, dtype=torch.int32).cuda())
        ref = (x[:, 3].double() ** 2).mean()
        assert ref < 3.2e38
        assert abs(float(b.zloss) - ref) <= 2.0 ** -23 * ref
        assert float(b.loss) == E and int(b.tokens) == T


def test_mean_square_out_of_the_range(emu):
    x = torch.full((300, 8), 2e19)
    b = emu.moe_balance(x.cuda(), torch.zeros((300, 1), dtype=torch.int32).cuda())
    assert float(b.zloss) == math.inf


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dl,dz", [(1e38, 0.0), (1.0, 3e38), (-3e38, -3e38)])
def test_gradients_of_large_losses(emu, kind, dl, dz):
    """dloss E and 2 dzloss are beyond the range, a token's share of them is not."""
    gen = torch.Generator().manual_seed(4)
    T, E, k = 2000, 64, 4
    x = (torch.randn((T, E), generator=gen) / 4).to(M.TYPES[kind])
    ids = torch.topk(x.float(), k).indices.int().contiguous()
    b = emu.moe_balance(x.cuda(), ids.cuda())
    dl, dz = torch.tensor([dl]), torch.tensor([dz])
    ref, bar = Q.balance_grad(x, b.counts.cpu().long(), b.tokens.cpu(), dl, dz, None)
    assert (ref.abs() < 3e37).all() and (ref.abs() > 1e30).any()
    got = emu.moe_balance_grad(x.cuda(), b.counts, b.tokens, dl.cuda(), dz.cuda())
    M.check(got, ref, bar + M.rounded(ref, M.TYPES[kind]))
