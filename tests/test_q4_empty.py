"""Packing of matrices without columns: as far as the check for a GPU, without one."""
import pytest
import torch

import paper_2609_04663_amd as emu


@pytest.mark.parametrize("shape", [(4, 0), (2, 3, 0), (0, 64), (0, 3, 64), (0, 0)])
def test_empty_matrices(shape):
    with pytest.raises(TypeError, match="GPU"):
        emu.q4_pack(torch.zeros(shape))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_an_empty_reduction(dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q, s = emu.q4_pack(torch.zeros((2, 5, 0), dtype=dtype, device="cuda"))
    assert Q.shape == (2, 5, 0) and s.shape == (2, 5, 0)
    X, off = torch.zeros((7, 0), dtype=dtype, device="cuda"), torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    Y = torch.full((7, 5), 9.0, dtype=dtype, device="cuda")
    assert (emu.q4_gemm(X, Q, s, offsets=off, Y=Y) == 0).all()
