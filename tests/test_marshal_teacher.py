"""The native hand-over of the calls that learn from a teacher without a GPU, as test_marshal_block.py has it for a block's; and what
the library says before it looks at a device."""
import ctypes as C
import importlib.machinery
import importlib.util
import os

import pytest
import torch

from paper_1805_01993_amd import binding as B
from paper_1805_01993_amd import build

ROWS, COLUMNS, OUTPUTS, K = 5, 300, 7, 3


@pytest.fixture(scope="module")
def module(tmp_path_factory):
    at = tmp_path_factory.mktemp("marshal")
    with open(os.path.join(build.CSRC, "marshal.cpp")) as fh:
        text = fh.read()
    # (the device of a host tensor is -1)
    for old, new in (("t.is_cuda()", "t.is_cpu()"), ("c10::hip::getCurrentHIPStream().stream()", "nullptr"), ("c10::hip::current_device()", "-1")):
        assert old in text
        text = text.replace(old, new)
    (at / "marshal.cpp").write_text(text)
    with pytest.MonkeyPatch.context() as patch:
        patch.setattr(build, "CSRC", str(at))
        patch.setattr(build, "MARSHAL", str(at / "_marshal.so"))
        path = build.build_marshal()
    spec = importlib.util.spec_from_loader("_marshal", importlib.machinery.ExtensionFileLoader("_marshal", path))
    made = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(made)
    return made


@pytest.fixture
def calls(module):
    lib, taken, kept = B.load_library(), [], []

    def recorder(name):
        fn = getattr(lib, name)
        made = C.CFUNCTYPE(C.c_int, *fn.argtypes)(lambda *a: taken.append((name,) + a[1:]) or 0)
        kept.append(made)
        return C.cast(made, C.c_void_p).value

    def failed(status, call):
        raise AssertionError(f"call {call}: status {status}")

    yield module.Block(1, failed, 2, 24, 16, 10, 1, 0, *(recorder(n) for n in B._BLOCK_CALLS)), taken
    kept.clear()


def new(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def padded(rows, columns, pad=3):
    return new(rows, columns + pad)[:, :columns]


U8, I32, F32, F8 = torch.uint8, torch.int32, torch.float32, torch.float8_e4m3fn


@pytest.mark.parametrize("eight", [U8, F8])
def test_packed_matrices_are_handed_over(calls, eight):
    call, taken = calls
    x, q, s = padded(ROWS, COLUMNS), new(ROWS, 384, dtype=eight), new(ROWS, 4, dtype=U8)
    assert call(B._QUANTISE, x, q, s) == 0
    assert taken.pop() == ("ccdc_quantise", ROWS, COLUMNS, x.data_ptr(), COLUMNS + 3, q.data_ptr(), s.data_ptr(), None)
    W, Ws, y = new(OUTPUTS, 384, dtype=eight), new(OUTPUTS, 4, dtype=U8), padded(ROWS, OUTPUTS)
    assert call(B._PACKED_PRODUCT, q, s, W, Ws, y) == 0
    assert taken.pop() == ("ccdc_packed_product", ROWS, OUTPUTS, 384, q.data_ptr(), s.data_ptr(), W.data_ptr(), Ws.data_ptr(), y.data_ptr(),
                           OUTPUTS + 3, None)


def test_lists_are_handed_over(calls):
    call, taken = calls
    z, index, value, rest = padded(ROWS, COLUMNS), new(ROWS, K, dtype=I32), new(ROWS, K, dtype=F32), new(ROWS, dtype=F32)
    assert call(B._TOP, z, index, value, rest, 2.5) == 0
    assert taken.pop() == ("ccdc_top", ROWS, COLUMNS, z.data_ptr(), COLUMNS + 3, K, 2.5, index.data_ptr(), value.data_ptr(), rest.data_ptr(), None)
    assert call(B._TOP, z, index, value, None, 1.0) == 0
    assert taken.pop()[9] is None
    loss, dz, weight = new(ROWS, dtype=F32), padded(ROWS, COLUMNS, 1), new(ROWS, dtype=F32)
    assert call(B._DISTILL, z, index, value, loss, dz, rest, 2.0, weight, 0.5) == 0
    assert taken.pop() == ("ccdc_distill", ROWS, COLUMNS, z.data_ptr(), COLUMNS + 3, K, index.data_ptr(), value.data_ptr(), rest.data_ptr(), 2.0,
                           weight.data_ptr(), 0.5, loss.data_ptr(), dz.data_ptr(), COLUMNS + 1, None)
    assert call(B._DISTILL, z, index, value, None, dz, None, 2.0, None, 0.5) == 0
    assert call(B._DISTILL, z, index, value, loss, None, None, 2.0, None, 0.5) == 0


def test_what_is_no_ordinary_call_is_left(calls):
    """To the checks in Python, which word the refusal: nothing reaches the library."""
    call, taken = calls
    x, q, s = new(ROWS, COLUMNS), new(ROWS, 384, dtype=U8), new(ROWS, 4, dtype=U8)
    for bad in ((x.float(), q, s), (x.t(), q, s), (x[0], q, s), (x, q[:, :256], s), (x, q[:4], s), (x, new(ROWS, 512, dtype=U8)[:, :384], s),
                (x, q.int(), s), (x, q, s[:, :3]), (x, q, s.int()), (None, q, s), (x, None, s), (x, q, None), (new(ROWS, 0), q, s)):
        assert call(B._QUANTISE, *bad) is None
    W, Ws, y = new(OUTPUTS, 384, dtype=U8), new(OUTPUTS, 4, dtype=U8), new(ROWS, OUTPUTS)
    for bad in ((q, s, W[:, :256], Ws, y), (q, s, W, s, y), (q, s, W, Ws, y.float()), (q, s, W, Ws, y[:4]), (q, s, W, Ws, y.t()), (q[:, :100], s, W[:, :100], Ws, y),
                (q, None, W, Ws, y), (q, s, W, Ws, None), (new(ROWS, 0, dtype=U8), s, W, Ws, y)):
        assert call(B._PACKED_PRODUCT, *bad) is None
    index, value, rest = new(ROWS, K, dtype=I32), new(ROWS, K, dtype=F32), new(ROWS, dtype=F32)
    for bad in ((x, index.long(), value, rest, 1.0), (x, index, value[:, :2], rest, 1.0), (x, index, value, rest[:4], 1.0), (x, index, value, rest, 1),
                (x, index[:4], value, rest, 1.0), (x, new(K, ROWS, dtype=I32).t(), value, rest, 1.0), (x, None, value, rest, 1.0), (x[0], index, value, rest, 1.0)):
        assert call(B._TOP, *bad) is None
    loss, dz = new(ROWS, dtype=F32), new(ROWS, COLUMNS)
    good = [x, index, value, loss, dz, rest, 1.0, None, 1.0]
    for at, bad in ((0, x.float()), (1, index.long()), (2, value.half()), (3, loss[:3]), (4, dz[:, :9]), (4, dz.float()), (5, rest.double()), (6, 1), (7, loss[:1]),
                    (7, loss.half()), (8, None), (2, None)):
        assert call(B._DISTILL, *(bad if i == at else v for i, v in enumerate(good))) is None
    assert taken == []


def test_calls_without_a_device():
    """A null block, and one that is not uploaded, whatever else is asked."""
    lib = B.load_library()
    h = C.c_void_p()
    config = B.BlockConfig(8, 8, B.BF16_SUM_XOR, 0, 0, 0, 1e-6, 1.0, 0.0, 0.0)
    assert lib.ccdc_block(C.byref(config), C.byref(h)) == B.OK
    p = 4096
    for block, status in ((None, B.EINVAL), (h, B.ESTATE)):
        assert lib.ccdc_quantise(block, 1, 1, p, 1, p, p, None) == status
        assert lib.ccdc_packed_product(block, 1, 1, 128, p, p, p, p, p, 1, None) == status
        assert lib.ccdc_top(block, 1, 1, p, 1, 1, 1.0, p, p, None, None) == status
        assert lib.ccdc_distill(block, 1, 1, p, 1, 1, p, p, None, 1.0, None, 1.0, p, p, 1, None) == status
    lib.ccdc_block_destroy(h)


def test_shapes_of_packed_matrices():
    assert B.packed_shapes(3, 1) == ((3, 128), (3, 4))
    assert B.packed_shapes(0, 512) == ((0, 512), (0, 4))
    assert B.packed_shapes(2, 513) == ((2, 640), (2, 8))
