"""The workspaces that the network operators ask for, without a GPU: what a call needs follows its sizes and layout."""
import pytest

ALIGNED = 1 << 20          # a pointer on a 16-byte boundary; nothing is read


@pytest.fixture(scope="module")
def nets():
    from paper_2512_13359_gb300 import build, nets
    build.build()
    nets.lib()
    return nets


def _scan(nets, T, N, D, inner, dtype, back, data=ALIGNED):
    r = (data, N * inner, inner)
    return nets.lib().net_gate_scan_workspace_bytes(
        nets._SCAN.pack(nets._SCAN.size, dtype, T, N, D, *(6 * r), *(7 * (0,)), 0), back)


@pytest.mark.parametrize("back", [0, 1])
@pytest.mark.parametrize("T,N,D", [(8192, 64, 1), (16384, 100, 2), (30000, 30, 4)])
def test_narrow_rows_apart_are_split_where_blocks_would_be_near_empty(nets, T, N, D, back):
    """A block has 32 channels.  Rows of a few channels that do not follow each other in memory (gate and value halves of
    one projection) leave it the channels of one env: N blocks instead of N D / 32, and pieces of the sequence are faster."""
    assert _scan(nets, T, N, D, 2 * D, 0, back) > 0
