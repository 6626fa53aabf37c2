"""What the 8-bit decoder operators launch, asked on the host without a GPU."""
import pytest

from launch_util import ADDRESS as P
from launch_util import launches


@pytest.mark.parametrize("fail", [0, 1])
def test_launches_that_fail_are_reported(fail):
    """The products and their weighted sums are two launches: whichever fails, the call says so, and nothing follows a failure."""
    args = [P, 64, P, 2, P, P, P, P, 4, 3, P, P, 2, P, 8, 8, 64, 0, P, 128, None]
    (good, both), (status, made) = launches([("w8_experts_matmul", args, -1), ("w8_experts_matmul", args, fail)])
    assert good == 0 and [m["kernel"].split("<")[0] for m in both] == ["w8_rows_kernel", "w8_combine_kernel"]
    assert status == -6 and made == both[:fail + 1]
