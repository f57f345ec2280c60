"""Host side of the routed-expert calls and of the layer on them: what is refused before any device is touched."""
import pytest

from paper_2502_07021_b200 import binding as fs
from paper_2502_07021_b200 import build as fs_build

P = 0x1000  # never dereferenced: every case is refused on the host


@pytest.mark.parametrize("eps", [1e-39, 1e-46, 4e38, 1e300])
def test_balance_refuses_an_eps_beyond_fp32(eps):
    """eps and log2(e)/eps are fp32 numbers in the kernel; where one of them is 0 or infinite every dual would be NaN."""
    fs_build.build()
    need = fs.fs_router_workspace(10, 4, 1)
    assert fs.lib().fs_router_duals(P, fs.FS_F32, 4, 10, 4, None, None, eps, 1, None, None, P, None, P, need, None) == fs.FS_ERR_BAD_EPS
