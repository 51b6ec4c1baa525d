"""The weight gradient from an 8-bit store with and without its bias gradient."""
import pytest
import torch

import ops_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,N,pad", [(1, 64, 40, 0), (100, 1000, 72, 16), (513, 256, 1024, 0), (2048, 520, 136, 8),
                                          (4096, 512, 2048, 0), (3000, 48, 1024, 0)])
def test_same_bits_without_the_bias(lib, rows, K, N, pad, dtype):
    """Products whose kernel also forms the bias sums (bf16 from 65 columns on) and others: one product, one
    order of its sums, whoever asks for what beside it."""
    g = torch.Generator().manual_seed(rows + K)
    x = torch.randn(rows, K, generator=g).to(R.TORCH[dtype]).cuda()
    dy = torch.randn(rows, N + pad, generator=g).to(R.TORCH[dtype]).cuda()
    code = R.CODE[dtype]
    store = torch.empty(lib.orbit_act8_bytes(rows, K), dtype=torch.uint8, device="cuda")
    lib.orbit_act8_pack(code, rows, K, x, K, store)
    ws = torch.empty(lib.orbit_act8_weight_grad_workspace_bytes(code, rows, K, N), dtype=torch.uint8, device="cuda")
    got = []
    for db in (torch.zeros(N, device="cuda"), None, torch.zeros(N, device="cuda")):
        dw = torch.zeros(K, N, device="cuda")
        lib.orbit_act8_weight_grad(code, rows, K, N, store, dy, N + pad, dw, db, 0, ws.fill_(0xFF))
        got.append((dw, db))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][0], got[2][0])
    assert torch.equal(got[0][1], got[2][1])
