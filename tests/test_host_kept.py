"""What the binding takes for a kept matrix: elements, or a checkpoint with both of its parts."""
import pytest

torch = pytest.importorskip("torch")

import paper_2005_03300_amd as g
from paper_2005_03300_amd import binding


class Operand:
    """Stands for a device tensor where there is no device; nothing is read from it."""
    is_cuda = True

    def __init__(self, shape, dtype, at):
        self.shape, self.dtype, self.at = torch.Size(shape), dtype, at

    def stride(self):
        return self.shape[1], 1

    def data_ptr(self):
        return self.at


def test_a_checkpoint_has_codes_and_scales():
    g.lib()
    codes, scales = Operand((8, 100), torch.int8, 4096), Operand((8, 2), torch.bfloat16, 8192)
    assert binding._kept((codes, scales), (8, 100), torch.bfloat16) == (4096, 100, 8192, 2)
    assert binding._kept(Operand((8, 100), torch.bfloat16, 4096), (8, 100), torch.bfloat16) == (4096, 100, 0, 0)
    assert binding._kept(None, (8, 100), torch.bfloat16) == (0, 0, 0, 0)
    for part in ((codes, None), (None, scales)):                      # codes alone are no elements: half or a quarter of the bytes that would be read
        with pytest.raises(AssertionError, match="codes and scales"):
            binding._kept(part, (8, 100), torch.bfloat16)
    with pytest.raises(AssertionError):
        binding._kept(codes, (8, 100), torch.bfloat16)
