"""The native hand-over of a block's calls (csrc/marshal.cpp) without a GPU: the module is built for host tensors, and the entry
points that it calls are recorders, so that what would be handed to the library is looked at and nothing runs."""
import ctypes as C
import importlib.machinery
import importlib.util
import os

import pytest
import torch

from paper_1805_01993_amd import binding as B
from paper_1805_01993_amd import build

WIDTH, HIDDEN, FILES, TOKENS = 24, 16, 3, 10


@pytest.fixture(scope="module")
def module(tmp_path_factory):
    """_marshal for tensors of the CPU, on no stream."""
    at = tmp_path_factory.mktemp("marshal")
    with open(os.path.join(build.CSRC, "marshal.cpp")) as fh:
        text = fh.read()
    for old, new in (("t.is_cuda()", "t.is_cpu()"), ("c10::hip::getCurrentHIPStream().stream()", "nullptr")):
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
    """(call, taken): the hand-over of a block of WIDTH x HIDDEN on FILES files, and what the library was given."""
    lib, taken, kept = B.load_library(), [], []

    def recorder(name):
        fn = getattr(lib, name)
        made = C.CFUNCTYPE(C.c_int, *fn.argtypes)(lambda *a: taken.append((name,) + a[1:]) or 0)
        kept.append(made)
        return C.cast(made, C.c_void_p).value

    def failed(status, call):
        raise AssertionError(f"call {call}: status {status}")

    block = module.Block(1, failed, 4, WIDTH, HIDDEN, TOKENS, FILES, 0, *(recorder(n) for n in B._BLOCK_CALLS))
    yield block, taken
    kept.clear()


def backward(call, *gradients):
    """ccdc_join_backward with these gradients of w_post, the gate and w_pre."""
    rows = [torch.zeros(TOKENS, WIDTH) for _ in range(6)]
    return call(B._JOIN_BACKWARD, *rows, None, None, None, *gradients, 0)


def by_file(stride, columns=WIDTH):
    """[FILES][columns] with this stride from file to file."""
    return torch.zeros(max(1, stride) * FILES + columns).as_strided((FILES, columns), (stride, 1))


@pytest.mark.parametrize("strides", [(0, WIDTH, WIDTH), (WIDTH, 0, WIDTH), (WIDTH, WIDTH, 0), (0, 0, WIDTH), (0, 0, 0), (0, None, 3 * WIDTH),
                                     (None, 0, WIDTH), (WIDTH - 1, None, None), (None, None, 1), (WIDTH, 2 * WIDTH, None)])
def test_gradients_that_have_no_stride_in_common_are_left(calls, strides):
    """One stride is handed over for all three: a gradient whose files lie on one another (an expanded tensor) would be written with
    the stride of the next, past its storage."""
    call, taken = calls
    assert backward(call, *(None if s is None else by_file(s) for s in strides)) is None
    assert taken == []


@pytest.mark.parametrize("strides", [(WIDTH, WIDTH, WIDTH), (3 * WIDTH + 1, None, 3 * WIDTH + 1), (None, None, WIDTH), (None, None, None)])
def test_gradients_of_one_stride_are_handed_over(calls, strides):
    call, taken = calls
    gradients = [None if s is None else by_file(s) for s in strides]
    assert backward(call, *gradients) == 0
    (name, *got), = taken
    assert name == "ccdc_join_backward"
    post, gate, pre, ld_file = got[11:15]
    assert [post, gate, pre] == [None if g is None else g.data_ptr() for g in gradients]
    assert ld_file == next((s for s in strides if s is not None), 0)


@pytest.mark.parametrize("which", [0, 1])
def test_weights_gradients_on_one_another_are_left(calls, which):
    call, taken = calls
    grads = [torch.zeros(FILES, 2 * HIDDEN, WIDTH), torch.zeros(FILES, WIDTH, HIDDEN)]
    x, saved = torch.zeros(TOKENS, WIDTH), torch.zeros(0, dtype=torch.uint8)
    arguments = [x, torch.zeros(2 * HIDDEN, WIDTH), torch.zeros(WIDTH, HIDDEN), saved, x, torch.zeros(TOKENS, WIDTH)]
    assert call(B._FFN_BACKWARD, *arguments, *grads) == 0 and len(taken) == 1
    grads[which] = grads[which][:1].expand(FILES, -1, -1)
    assert call(B._FFN_BACKWARD, *arguments, *grads) is None and len(taken) == 1


@pytest.mark.gpu
def test_both_ways_refuse_gradients_on_one_another():
    """The call itself, natively and through the checks in Python (a stream is named), which word the refusal."""
    import paper_1805_01993_amd as L
    block = L.ccdc_block(WIDTH, HIDDEN, "f32").bind([4, 0, 6]).upload()
    new = lambda: torch.ones(TOKENS, WIDTH, device="cuda")  # noqa: E731
    room = torch.full((5 * FILES * WIDTH,), 7.0, device="cuda")
    expanded, proper = room[:WIDTH].expand(FILES, -1), room[FILES * WIDTH:2 * FILES * WIDTH].view(FILES, WIDTH)
    for stream in (None, torch.cuda.current_stream()):
        for post, gate in ((expanded, proper), (proper, expanded)):
            with pytest.raises(ValueError, match="the same stride"):
                block.join_backward(None, new(), None, new(), new(), new(), dw_post=post, dgate=gate, stream=stream)
        with pytest.raises(L.CcdcError):
            block.join_backward(None, new(), None, new(), new(), new(), dw_post=expanded, dgate=expanded, stream=stream)
        torch.cuda.synchronize()
        assert bool((room == 7).all())
