"""What a layer norm without a residual hands back as the sum that it normed: its input itself, no copy."""
import pytest

torch = pytest.importorskip("torch")
x = pytest.importorskip("paper_2512_16512_amd")


@pytest.mark.gpu
@pytest.mark.parametrize("quantize", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_sum_without_a_residual_is_the_input(dtype, quantize):
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    rows, w = torch.randn(6, 300).to(dtype).cuda(), torch.ones(300, dtype=dtype).cuda()
    for eps in (1e-5, 1):                # (an int takes the path without the binding)
        n = x.layernorm(rows, w, eps=eps, quantize=quantize)
        assert n.residual.data_ptr() == rows.data_ptr() and n.residual.shape == rows.shape
    with_one = x.layernorm(rows, w, residual=rows, quantize=quantize)
    assert with_one.residual.data_ptr() != rows.data_ptr()
