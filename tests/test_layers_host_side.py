"""What the layer operators' calls queue and ask for, looked at without a GPU (tests/layer_launches.py)."""
import shutil

import pytest

from tests import layer_launches as Q

F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++ here")
    return Q.build(tmp_path_factory.mktemp("layers"))


@pytest.mark.parametrize("rows", [(1 << 26) - 16, (1 << 26) - 15, 1 << 26, (1 << 27) + 1, 1 << 28])
def test_loss_of_many_rows_is_launched(driver, rows):
    """As many rows as the header allows; HIP counts a grid's threads in 32 bits, and a loss takes 64 a row."""
    call, = Q.calls(driver, [("loss", BF16, rows, 8, 64)])
    assert call.rc == 0 and "loss_kernel" in call.launches[-1][0]
    assert call.launches[-1][1] == min((rows + 15) // 16, 1 << 21)
