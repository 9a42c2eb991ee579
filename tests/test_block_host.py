"""The trained block without a GPU: configurations and batches that are refused, sizes, and what calls answer before there is
anything on a device.  The reference's generator is pinned to the published vectors."""
import ctypes as C

import numpy as np
import pytest

import block_reference as R
from paper_1805_01993_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def make(lib, **other):
    c = dict(width=64, hidden=96, mode=B.BF16_SUM_XOR, activation=0, norm=0, layer=0, eps=1e-6, residual_scale=1.0,
             dropout_hidden=0.0, dropout_out=0.0)
    h = C.c_void_p()
    return lib.ccdc_block(C.byref(B.BlockConfig(**{**c, **other})), C.byref(h)), h


def test_generator_of_the_reference():
    """Random123's known answers for Philox4x32-10."""
    ones = 0xFFFFFFFF
    for counter, key, want in (([0] * 4, (0, 0), [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
                               ([ones] * 4, (ones, ones), [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD])):
        assert R.philox(np.array([counter], np.uint64), key)[0].tolist() == want


@pytest.mark.parametrize("other", [
    {"width": 0}, {"width": -1}, {"width": (1 << 20) + 1}, {"hidden": 0}, {"hidden": (1 << 20) + 1}, {"mode": B.U32_XOR}, {"mode": 9},
    {"mode": -1}, {"activation": 3}, {"activation": -1}, {"norm": 2}, {"layer": 1 << 31}, {"eps": 0.0}, {"eps": -1.0},
    {"eps": float("nan")}, {"eps": float("inf")}, {"residual_scale": float("nan")}, {"dropout_hidden": -0.1},
    {"dropout_out": 1.01}, {"dropout_out": float("nan")}])
def test_configurations_that_are_refused(lib, other):
    rc, h = make(lib, **other)
    assert rc == B.EINVAL and not h


def test_null_pointers(lib):
    assert lib.ccdc_block(None, C.byref(C.c_void_p())) == B.EINVAL
    lib.ccdc_block_destroy(None)
    assert lib.ccdc_block_bind(None, 1, (C.c_int64 * 1)(1), None) == B.EINVAL
    assert lib.ccdc_block_upload(None) == B.EINVAL
    assert lib.ccdc_block_query(None, 0, C.byref(C.c_int64()), 8) == B.EINVAL


def test_batches(lib):
    rc, h = make(lib)
    assert rc == B.OK
    v = C.c_int64()
    bind = lambda tokens, ids=None: lib.ccdc_block_bind(  # noqa: E731
        h, len(tokens), (C.c_int64 * max(1, len(tokens)))(*tokens), None if ids is None else (C.c_int32 * len(ids))(*ids))
    assert lib.ccdc_block_query(h, B.BLOCK_Q_TOKENS, C.byref(v), 8) == B.ESTATE
    assert lib.ccdc_block_upload(h) == B.ESTATE
    assert bind([]) == B.EINVAL and bind([3, -1]) == B.EINVAL and bind([3], [-1]) == B.EINVAL
    assert lib.ccdc_block_bind(h, 1, None, None) == B.EINVAL
    assert bind([1 << 31]) == B.ESIZE and bind([1 << 30, 1 << 30]) == B.ESIZE and bind([1 << 62, 1 << 62]) == B.ESIZE
    assert lib.ccdc_block_query(h, B.BLOCK_Q_TOKENS, C.byref(v), 8) == B.ESTATE       # a refused batch is none
    assert bind([3, 0, 40], [5, 5, 1]) == B.OK
    got = []
    for q in range(4):
        assert lib.ccdc_block_query(h, q, C.byref(v), 8) == B.OK
        got.append(v.value)
    assert got[:2] == [43, 3] and got[2] >= 43 * 96 * 2 and got[3] > 0
    assert bind([-1]) == B.EINVAL
    assert lib.ccdc_block_query(h, 0, C.byref(v), 8) == B.OK and v.value == 43          # the one before stays
    for what, room in ((4, 8), (-1, 8), (0, 4)):
        assert lib.ccdc_block_query(h, what, C.byref(v), room) == B.EINVAL
    assert lib.ccdc_block_query(h, 0, None, 8) == B.EINVAL
    # bound, not on a device
    p = C.c_void_p(4096)
    assert lib.ccdc_ffn_forward(h, 1, p, 64, p, p, p, 64, None, 0, None) == B.ESTATE
    assert lib.ccdc_ffn_backward(h, p, 64, p, p, p, p, 64, p, 64, p, 1 << 20, p, 1 << 20, None) == B.ESTATE
    assert lib.ccdc_join_forward(h, 1, p, p, p, p, 0, p, p, p, 64, 0, None) == B.ESTATE
    assert lib.ccdc_join_backward(h, p, p, p, p, p, p, 0, p, p, p, 64, p, p, p, 64, 0, None) == B.ESTATE
    assert lib.ccdc_dropout(h, 1, 64, 0.1, 0, 0, p, 64, None, 0, p, 64, None) == B.ESTATE
    for call in (lib.ccdc_ffn_forward(None, 1, p, 64, p, p, p, 64, None, 0, None),
                 lib.ccdc_dropout(None, 1, 64, 0.1, 0, 0, p, 64, None, 0, p, 64, None)):
        assert call == B.EINVAL
    lib.ccdc_block_destroy(h)


def test_a_batch_too_large_for_its_buffers(lib):
    rc, h = make(lib, width=1 << 20, hidden=1 << 20, mode=B.F32_SUM)
    assert rc == B.OK
    assert lib.ccdc_block_bind(h, 1, (C.c_int64 * 1)(1), None) == B.ESIZE              # W_in alone
    lib.ccdc_block_destroy(h)


def test_saved_bytes_grow_with_tokens_and_type():
    sizes = {}
    for mode in ("bf16", "f16", "f32"):
        for tokens in (16, 32):
            block = B.Block(64, 100, mode).bind([tokens])
            sizes[mode, tokens] = block.saved_bytes
            block.close()
    assert sizes["bf16", 16] == sizes["f16", 16] < sizes["f32", 16]
    assert all(sizes[m, 32] > sizes[m, 16] for m in ("bf16", "f16", "f32"))


def test_block_of_the_binding_checks_its_arguments():
    with pytest.raises(B.CcdcError):
        B.Block(64, 96, "u32")
    block = B.Block(64, 96, "bf16")
    with pytest.raises(ValueError):
        block.bind([1, 2], ids=[0])
    import torch
    block.bind([4])
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        block.dropout(x, x, 0.1, site=0)                                                # not on a device
    block.close()
