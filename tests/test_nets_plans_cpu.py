"""The workspaces that the network operators ask for, without a GPU: sizes follow the layout that a call
will have, and a query made before the arrays exist covers every one of them."""
import itertools

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


@pytest.mark.parametrize("back", [0, 1])
@pytest.mark.parametrize("T,N,D,dtype", [(8192, 64, 1, 0), (65521, 1, 250, 0), (512, 4096, 8, 1), (8192, 5, 100, 2), (20, 9, 9, 0)])
def test_a_query_without_arrays_covers_every_layout(nets, T, N, D, dtype, back):
    most = _scan(nets, T, N, D, D, dtype, back, data=0)
    for inner in (D, 2 * D, D + 3):
        assert _scan(nets, T, N, D, inner, dtype, back) <= most


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("B,S,C,G", [(500, 300, 128, 1), (256, 1, 90, 9), (64, 4096, 256, 32), (1, 65536, 256, 1),
                                     (70, 40, 48, 6), (5000, 1, 24, 3), (14, 65, 4160, 1)])
def test_a_norm_query_without_arrays_covers_every_alignment(nets, B, S, C, G, dtype):
    F, ask = nets._NORM, nets.lib().net_group_norm_workspace_bytes
    size = 2 if dtype else 4

    def need(pointers, weights, back, odd=0):
        rows = [q for p in pointers for q in (p, S * C + odd, C)]
        return ask(F.pack(F.size, dtype, 2, 1e-5, B, S, C, G, *rows, *(6 * (0,)), 0, 0)
                   if not weights else
                   F.pack(F.size, dtype, 2, 1e-5, B, S, C, G, *rows, 0, 0, 0, 0, ALIGNED, ALIGNED, 0, 0), back)
    for back in (0, 1):
        most = need((0, 0, 0, 0), False, back)
        assert need((0, 0, 0, 0), False, back, odd=1) == most
        for offs in itertools.product((0, size, 8), repeat=4):
            assert need([ALIGNED + o for o in offs], True, back) <= most, (offs, back)
