"""The 8-bit front end past the sizes of its other tests: rows and channels that leave 31
bits or a slab, second turns of persistent kernels, rows whose squares leave fp32, and
tensors that do not belong to the call."""
import pytest
import torch

from paper_2412_00119_gb300 import bmlp as B

DEV = "cuda:0"
gpu = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device(request):
    if request.node.get_closest_marker("gpu"):
        if not torch.cuda.is_available():
            pytest.skip("needs a GPU")
        torch.cuda.set_device(DEV)


# -- refusals ------------------------------------------------------------------------

def test_sizes_past_31_bits_are_refused():
    """Sizes that the C types cannot hold: not the call of the size that is left of them."""
    def t(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="meta")   # (shapes and strides without memory)
    i8, f32 = torch.int8, torch.float32
    for big in (2 ** 31, 2 ** 32 + 8, 2 ** 33 + 1):
        calls = [lambda: B.bmlp_quantize_rows(t((1, big), f32), t((1, big), i8), t((1,), f32)),
                 lambda: B.bmlp_norm_quantize(t((1, big), f32), None, t((1, big), i8), t((1,), f32)),
                 lambda: B.bmlp_int8_matmul(t((1, big), i8), t((4, big), i8), t((1, 4), f32)),
                 lambda: B.bmlp_int8_matmul(t((1, 8), i8), t((big, 8), i8), t((1, big), f32)),
                 lambda: B.bmlp_int8_sign(t((1, big), i8), t((4, big), i8), t((1, 1), torch.int64)),
                 lambda: B.bmlp_int8_sign(t((1, 8), i8), t((big, 8), i8), t((1, (big + 63) // 64), torch.int64))]
        for call in calls:
            with pytest.raises(B.BmlpError, match="31 bits") as e:
                call()
            assert e.value.code == B.BMLP_EINVAL
        assert B.bmlp_int8_workspace(300, big, 4000) == 0
        assert B.bmlp_int8_workspace(300, 2304, big) == 0
    assert B.bmlp_int8_workspace(300, 2 - 2 ** 32, 4000) == 0
