"""What the binding of the decode-step calls checks of its tensors before it hands pointers to the library.  The tensors are
stand-ins with a device of their choice, so no GPU is needed: nothing is ever read from them."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from paper_2605_07114_b200 import hora  # noqa: E402

H, D = 2, 64


class Rows:
    """Shape, strides, type and device of a tensor, without one."""

    def __init__(self, *shape, stride=None, dtype=torch.bfloat16, cuda=True):
        t = torch.empty(shape, dtype=dtype, device="meta")
        self.shape, self.dtype, self.is_cuda = t.shape, dtype, cuda
        self._stride = tuple(t.stride()) if stride is None else stride

    def stride(self):
        return self._stride


@pytest.mark.parametrize("n", [1, 2, 7])
@pytest.mark.parametrize("v", [
    lambda n: Rows(n, H, D, cuda=False),                                  # on the host
    lambda n: Rows(n, H, D // 2),                                         # shorter rows
    lambda n: Rows(n, 1, 1),
    lambda n: Rows(n, H, D, stride=(2 * H * D, 2 * D, 2)),                # values apart
    lambda n: Rows(n, H, D, stride=(H * D, 1, H)),
])
def test_values_are_checked_like_keys_whatever_the_number_of_tokens(n, v):
    with pytest.raises(ValueError):
        hora._kv_rows(Rows(n, H, D), v(n), n, H, D)
    with pytest.raises(ValueError):
        hora._kv_rows(v(n), Rows(n, H, D), n, H, D)


@pytest.mark.parametrize("stride", [(D, D, 1), (0, D, 1), (1, D, 1), (10 ** 9 + 1, D, 1)])
def test_a_single_token_has_no_row_stride(stride):
    """The stride of a dimension of size one says nothing (a transposed view leaves any number there): the call gets one that it takes."""
    got = hora._kv_rows(Rows(1, H, D, stride=stride), Rows(1, H, D, stride=stride), 1, H, D)
    assert got == H * D


@pytest.mark.parametrize("shape", [(), (2, 3), (2, 1)])
def test_slots_are_one_list(shape):
    """A table of slots is refused: its first dimension alone would be taken for the number of tokens."""
    n = shape[0] if shape else 1
    slots, rows = torch.zeros(shape, dtype=torch.int64), torch.zeros(n, H, D, dtype=torch.bfloat16)
    pools = (None, None, None, None, hora.DTYPE_BF16, 4, 16)
    with pytest.raises(ValueError, match="slots"):
        hora._kv_write(pools, H, D, rows, rows, slots, None)
    with pytest.raises(ValueError, match="slots"):
        hora._kv_read(pools, H, D, slots, rows, rows, None)
