"""Limits of the extended block's sizes, refused before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2404_14712_amd import _lib as L

ROWS = (1 << 26) - 64      # a gated norm's launch: a wave per row, fewer than 2^32 threads
VALUES = 1 << 34           # a store's


@pytest.fixture(scope="module")
def lib():
    return L.OrbitLib()


def _desc(B, Lq, d=8, heads=1, head_dim=32, mlp=8):
    return L.BlockDesc(B, Lq, d, heads, head_dim, mlp, 0, 1e-5, 1)


def _calls(lib, desc, ext):
    """(saved bytes, workspace bytes, forward's and backward's status) with pointers nothing may read."""
    p = L.BlockParams(*[0x1000 + 0x100 * i for i in range(16)])
    ep = L.BlockExtParams(*[0x4000 + 0x100 * i for i in range(6)])
    g = L.BlockGrads(*[0x5000 + 0x100 * i for i in range(16)])
    eg = L.BlockExtGrads(*[0x7000 + 0x100 * i for i in range(6)])
    r = ctypes.byref
    # a workspace of 16 bytes: what is not refused for its sizes is refused for that
    fwd = lib.lib.orbit_vit_block_ext_fwd(r(desc), r(ext), r(p), r(ep), 0x100, 0x200, 0x300, 0x400, 16, None)
    bwd = lib.lib.orbit_vit_block_ext_bwd(r(desc), r(ext), r(p), r(ep), 0x100, 0x300, 0x200, 0x500, r(g), r(eg), 0, 0x400,
                                          16, None)
    return lib.orbit_vit_block_ext_saved_bytes(desc, ext), lib.orbit_vit_block_ext_workspace_bytes(desc, ext), fwd, bwd


REFUSED = (0, 0, L.ORBIT_E_UNSUPPORTED, L.ORBIT_E_UNSUPPORTED)
EXTS = {"act8": (1, 0, 0, 1.0), "post": (0, 1, 0, 1.0), "gate": (0, 0, 1, 1.0), "scale": (0, 0, 0, 0.5)}


@pytest.mark.parametrize("ext", EXTS)
def test_rows(lib, ext):
    e = L.BlockExt(*EXTS[ext])
    B = ROWS // 64
    got = _calls(lib, _desc(B, 64), e)
    assert got[0] > 0 and got[1] > 0 and got[2:] == (L.ORBIT_E_ARG,) * 2 and "workspace" in lib.last_error()
    for desc in (_desc(B + 1, 64), _desc(1 << 26, 1), _desc(ROWS + 1, 1)):
        assert _calls(lib, desc, e) == REFUSED and "tokens" in lib.last_error()


@pytest.mark.parametrize("width", [dict(d=16384), dict(mlp=16384), dict(heads=171)])
def test_values_of_a_store(lib, width):
    """q|k|v, u and the sub-layers' outputs are stores of at most 2^34 - 1 values; nothing else is bound by it."""
    e = L.BlockExt(*EXTS["act8"])
    n = 3 * 32 * width["heads"] if "heads" in width else 16384
    T = (VALUES - 1) // n
    got = _calls(lib, _desc(T, 1, **width), e)
    assert got[0] > 0 and got[1] > 0 and got[2:] == (L.ORBIT_E_ARG,) * 2
    assert _calls(lib, _desc(T + 1, 1, **width), e) == REFUSED and "2^34" in lib.last_error()
    assert _calls(lib, _desc(T + 1, 1, **width), L.BlockExt(*EXTS["scale"]))[1] > 0


def test_plain_form_keeps_its_limits(lib):
    """With nothing asked for the block is the plain one, at the plain one's sizes."""
    d = _desc(1 << 26, 1)
    assert lib.orbit_vit_block_ext_workspace_bytes(d, L.BlockExt(0, 0, 0, 1.0)) == lib.orbit_vit_block_workspace_bytes(d) > 0


@pytest.mark.parametrize("n", [8, 1000, 16416])
def test_store_alone_takes_what_the_block_does(lib, n):
    rows = (VALUES - 1) // n
    assert lib.orbit_act8_bytes(rows, n) > 0 and lib.orbit_act8_bytes(rows + 1, n) == 0
    assert lib.lib.orbit_act8_pack(1, rows, n, 0x100, n, 0x200, 16, None) == L.ORBIT_E_ARG and "smaller" in lib.last_error()
    assert lib.lib.orbit_act8_pack(1, rows + 1, n, 0x100, n, 0x200, 1 << 50, None) == L.ORBIT_E_UNSUPPORTED
