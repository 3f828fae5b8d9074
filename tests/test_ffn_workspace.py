"""The feed-forward block's workspaces hold what its grouped products write: the plan against the size functions (no GPU here)."""
import random

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2606_29758_gb300 import _binding, _build
    _build.build()
    _binding.lib()
    return _binding


def _holds(B, N, d, F, larger=()):
    """The partial tiles of Y and of every choice of gradients lie in the workspaces, also in those for more rows."""
    header = 256
    for rows in (N, *larger):
        room = B.ps_gated_ffn_fwd_workspace_size(rows, d, F, True) - header
        assert B.ps_diag_gated_ffn_partial_bytes(N, d, F, 0, False) <= room, ("Y", N, d, F, rows)
        room = B.ps_gated_ffn_bwd_workspace_size(rows, d, F) - header
        for products in range(1, 8):
            for f32 in (False, True):
                need = B.ps_diag_gated_ffn_partial_bytes(N, d, F, products, f32)
                assert need <= room, (products, f32, N, d, F, rows, need, room)


@pytest.mark.parametrize("N", [1, 8, 63, 64, 65, 128, 129, 700])
@pytest.mark.parametrize("F", [8, 72, 2048, 2056, 16384])
def test_very_wide_blocks(B, N, F):
    """Few rows of a narrow block give dX in two parts whatever its width is: planes that no share of a K loop bounds."""
    for d in (8, 38912, 38920, 77832, 155648, 155656, 160000, 262144, 400000):
        _holds(B, N, d, F, larger=(64, 65, 1000) if N <= 64 else (1000,))
    with_parts = N <= 64 and F <= 2048
    assert (B.ps_diag_gated_ffn_partial_bytes(N, 160000, F, 1, True) >= 2 * N * 160000 * 4) or not with_parts


def test_drawn_sizes(B):
    rng = random.Random(0)
    spread = lambda hi: int(8 * (hi / 8) ** rng.random()) // 8 * 8  # noqa: E731
    for _ in range(600):
        N = int(40000 ** rng.random())
        _holds(B, N, spread(200000), spread(40000), larger=(N + rng.randrange(1, 3000),))


@pytest.mark.parametrize("size,bytes_", [
    ((1, 1536, 8192), 69206272),
    ((8, 304, 1000), 1868032),
    ((64, 304, 1000), 1868032),
    ((64, 3584, 2048), 44040448),
    ((571, 392, 1048), 4817152),
    ((6030, 1536, 8192), 318767360),
    ((7835, 3584, 16384), 318767360),
])
def test_ordinary_sizes_ask_for_their_shares_alone(B, size, bytes_):
    """What holds the widest blocks costs the ordinary ones nothing."""
    assert B.ps_gated_ffn_bwd_workspace_size(*size) == bytes_


@pytest.mark.gpu
@pytest.mark.parametrize("N,d,F", [(8, 160000, 72), (64, 155656, 264)])
def test_a_very_wide_block_writes_its_workspace_alone(B, N, d, F):
    """Forward and backward of a block whose dX has more planes than a cut product may have, at the tolerances of the other
    sizes; what follows the backward's workspace keeps its bytes."""
    import torch
    from test_gpu_ffn import _close, _data, _wanted
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=N)
    size = B.ps_gated_ffn_bwd_workspace_size(N, d, F)
    u8 = dict(dtype=torch.uint8, device="cuda")
    ws = torch.full((size + (1 << 24),), 0x5A, **u8)
    store, ws_fwd = (torch.zeros(n, **u8) for n in (B.ps_gated_ffn_store_size(N, F),
                                                    B.ps_gated_ffn_fwd_workspace_size(N, d, F, True)))
    Y, dX = torch.empty_like(X), torch.empty_like(X)
    grads = [torch.empty_like(w) for w in (Wg, Wu, Wd)]
    B.ps_gated_ffn_fwd(N, d, F, B.PS_DTYPE_BF16, 0, X, Wg, Wu, Wd, Y, store, ws_fwd)
    B.ps_gated_ffn_bwd(N, d, F, B.PS_DTYPE_BF16, dY, X, Wg, Wu, Wd, store, dX, B.PS_DTYPE_BF16, *grads, B.PS_DTYPE_BF16, 0,
                       ws[:size])
    assert B.ps_workspace_status(ws_fwd)[0] == B.PS_OK and B.ps_workspace_status(ws[:size])[0] == B.PS_OK
    assert bool((ws[size:] == 0x5A).all())
    for got, want, name in zip((Y, dX, *grads), _wanted(X, Wg, Wu, Wd, dY, "silu"), ("y", "dx", "dwg", "dwu", "dwd")):
        _close(got, want, name)
