"""The host side of the dropout's calls at the ends of their ranges, without a GPU."""
import pytest

from test_attention_calls import calls, create, fake  # noqa: F401
from test_operator_calls import BF16, FP32, OK, lib  # noqa: F401


@pytest.mark.parametrize("rows,mask_rows", [(1 << 30, 1 << 29), ((1 << 30) + 5, 1 << 30), (1500000000, 1000000000), (2 ** 31 - 1, 2 ** 31 - 2),
                                            (2 ** 31 - 1, 1), (2 ** 31 - 1, 4)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_dropout_of_many_rows_launches_for_all_of_them(fake, rows, mask_rows, dtype):
    """Rows and mask rows whose sum passes 31 bits: a grid over the mask's pieces of 8 elements, and over its uses."""
    h = create(fake, "dropout", dtype, (2 ** 31 - 1, 1))
    a = calls()["dropout_forward"][1]
    fake.fake_reset()
    assert fake.stacklstm_dropout_forward(h, rows, *a[1:6], mask_rows, a[7]) == OK
    x, y = (int(v) for v in fake.fake_log().decode().split()[-6:-4])
    uses = -(-rows // mask_rows)
    assert x == -(-(-(-mask_rows // 8)) // 256) and 1 <= y <= 65535 and y <= uses and y * -(-uses // y) >= uses
    fake.stacklstm_op_destroy(h)
