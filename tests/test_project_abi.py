"""Argument checks of the checkpoint and projection calls, without a GPU: every refusal comes before the context is touched."""
import ctypes as C

import pytest
import torch

from paper_1611_05402_b200 import binding

BAD, UNSUPPORTED, WORKSPACE = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE
AT = 1 << 20                                     # stands in for a device address; nothing looks there


@pytest.fixture(scope="module")
def lib():
    from paper_1611_05402_b200.build import build
    build()
    return binding.lib()


@pytest.fixture()
def ctx():
    return C.cast(C.create_string_buffer(1 << 14), C.c_void_p)


def dataset(**kw):
    d = binding.CDataset(C.sizeof(binding.CDataset), 8, binding.LEVELS_UNIFORM, binding.LAYOUT_ROWS, 64, 48, 48, AT, AT, AT, AT, None)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def adapters(**kw):
    d = binding.CAdapters(C.sizeof(binding.CAdapters), binding.BF16, 2, 8, AT, AT, None, 3, 0, AT, AT)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def checkpoint(**kw):
    d = binding.CCheckpoint(C.sizeof(binding.CCheckpoint), 32, 10, 64, 64, AT, AT)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_struct_sizes():
    assert C.sizeof(binding.CCheckpoint) == 48 and C.sizeof(binding.CAdapters) == 64


@pytest.mark.parametrize("code,kw", [
    (BAD, dict(struct_size=8)), (UNSUPPORTED, dict(group=16)), (UNSUPPORTED, dict(group=512)), (UNSUPPORTED, dict(group=0)), (BAD, dict(m=-1)), (BAD, dict(n=0)),
    (BAD, dict(row_bytes=48)), (BAD, dict(row_bytes=72)), (WORKSPACE, dict(row_bytes=1 << 32)), (BAD, dict(codes=None)), (BAD, dict(grids=None)),
    (BAD, dict(codes=AT + 8)), (BAD, dict(grids=AT + 4))])
def test_checkpoint_refusals(lib, ctx, code, kw):
    c = checkpoint(**kw)
    assert lib.zipml_checkpoint_encode(ctx, AT, binding.BF16, 10, 64, 64, 0, C.byref(c)) == code
    assert lib.zipml_checkpoint_decode(ctx, C.byref(c), binding.BF16, AT, 64) == code


def test_checkpoint_matrix_refusals(lib, ctx):
    c = checkpoint()
    for x, dtype, m, n, ld in ((None, 1, 10, 64, 64), (AT, 3, 10, 64, 64), (AT, -1, 10, 64, 64), (AT, 1, 9, 64, 64), (AT, 1, 10, 63, 64), (AT, 1, 10, 64, 63),
                               (AT + 1, 1, 10, 64, 64), (AT + 2, 0, 10, 64, 64)):
        assert lib.zipml_checkpoint_encode(ctx, x, dtype, m, n, ld, 0, C.byref(c)) == BAD
    for x, dtype, ld in ((None, 1, 64), (AT, 3, 64), (AT, 1, 63), (AT + 1, 2, 64), (AT + 2, 0, 64)):
        assert lib.zipml_checkpoint_decode(ctx, C.byref(c), dtype, x, ld) == BAD
    assert lib.zipml_checkpoint_encode(ctx, AT, 1, 10, 64, 64, 0, None) == BAD
    assert lib.zipml_checkpoint_encode(None, AT, 1, 10, 64, 64, 0, C.byref(c)) == BAD
    assert lib.zipml_checkpoint_encode(ctx, None, 1, 0, 64, 64, 0, C.byref(checkpoint(m=0, codes=None, grids=None))) == binding.OK


def project(lib, ctx, w=None, a=None, x=AT, dtype=binding.BF16, tokens=10, ldx=64, y=2 * AT, ldy=48, hidden=None, none=False):
    w, a = w or dataset(), a or adapters()
    return lib.zipml_project(ctx, C.byref(w), None if none else C.byref(a), x, dtype, tokens, ldx, y, ldy, hidden)


def backward(lib, ctx, w=None, a=None, dy=AT, dtype=binding.BF16, tokens=10, lddy=48, hidden=AT, cp="", dx=2 * AT, lddx=64, ga=AT, gb=AT, none=False):
    w, a = w or dataset(), a or adapters()
    cp = checkpoint() if cp == "" else cp
    return lib.zipml_project_backward(ctx, C.byref(w), None if none else C.byref(a), dy, dtype, tokens, lddy, hidden, None if cp is None else C.byref(cp), dx, lddx,
                                      ga, gb)


@pytest.mark.parametrize("code,w", [
    (BAD, dict(struct_size=8)), (UNSUPPORTED, dict(bits=9)), (UNSUPPORTED, dict(level_mode=1, bits=4, levels=AT)), (UNSUPPORTED, dict(layout=1)),
    (BAD, dict(m=0)), (BAD, dict(n=0)), (BAD, dict(plane1=None)), (BAD, dict(plane1=AT + 8)), (BAD, dict(row_bytes=40)), (BAD, dict(feat_step=None)),
    (WORKSPACE, dict(m=(1 << 24) + 1)), (WORKSPACE, dict(n=(1 << 24) + 1, row_bytes=1 << 25))])
def test_projection_weights(lib, ctx, code, w):
    assert project(lib, ctx, w=dataset(**w), ldx=1 << 25, ldy=1 << 25) == code
    assert backward(lib, ctx, w=dataset(**w), lddy=1 << 25, lddx=1 << 25) == code


@pytest.mark.parametrize("code,a", [
    (BAD, dict(struct_size=8)), (BAD, dict(reserved=1)), (BAD, dict(dtype=binding.F16)), (BAD, dict(count=0)), (BAD, dict(rank=0)), (BAD, dict(requests=0)),
    (UNSUPPORTED, dict(count=65536)), (UNSUPPORTED, dict(rank=129)), (BAD, dict(a=None)), (BAD, dict(b=None)), (BAD, dict(starts=None)), (BAD, dict(which=None)),
    (BAD, dict(a=AT + 1)), (BAD, dict(starts=AT + 2)), (BAD, dict(scale=AT + 2))])
def test_projection_adapters(lib, ctx, code, a):
    assert project(lib, ctx, a=adapters(**a)) == code
    assert backward(lib, ctx, a=adapters(**a)) == code


def test_projection_arguments(lib, ctx):
    assert project(lib, None) == BAD and backward(lib, None) == BAD
    for kw in (dict(x=None), dict(y=None), dict(x=AT + 1), dict(y=AT + 1), dict(y=AT), dict(ldx=63), dict(ldy=47), dict(tokens=-1), dict(dtype=7), dict(hidden=AT + 2),
               dict(hidden=AT, none=True)):
        assert project(lib, ctx, **kw) == BAD, kw
    assert project(lib, ctx, dtype=binding.F32, none=True) == UNSUPPORTED and backward(lib, ctx, dtype=binding.F32, none=True, ga=None, gb=None) == UNSUPPORTED
    assert project(lib, ctx, tokens=(1 << 30) + 1) == WORKSPACE
    assert project(lib, ctx, tokens=0, x=None, y=None) == binding.OK
    for kw in (dict(dy=None), dict(dy=AT + 1), dict(dx=AT), dict(dx=AT + 1), dict(lddy=47), dict(lddx=63), dict(hidden=None), dict(cp=None), dict(ga=AT + 2),
               dict(gb=AT + 2), dict(cp=checkpoint(n=63)), dict(cp=checkpoint(m=9)), dict(none=True)):
        assert backward(lib, ctx, **kw) == BAD, kw


CPU = torch.device("cpu")


@pytest.mark.parametrize("matrix", [
    torch.zeros(8).expand(5, 8),                             # what autograd gives a sum over rows: every row the same memory
    torch.zeros(1, 1).expand(5, 1),
    torch.zeros(40).as_strided((5, 8), (7, 1)),              # each row begins in the one before
    torch.zeros(40).as_strided((5, 8), (1, 1)),
    torch.zeros(8, 5).t(),                                   # columns contiguous, not rows
    torch.zeros(5, 16)[:, ::2],
    torch.zeros(5, 8, dtype=torch.float64),
], ids=["expanded", "expanded column", "overlapping", "sliding", "transposed", "every other column", "fp64"])
def test_matrices_that_are_not_rows(matrix):
    with pytest.raises(AssertionError):
        binding._rows(matrix, CPU)


@pytest.mark.parametrize("matrix,ld", [
    (torch.zeros(5, 8), 8), (torch.zeros(5, 16)[:, 3:11], 16), (torch.zeros(1, 8), 8), (torch.zeros(8).expand(1, 8), 8), (torch.zeros(40).as_strided((1, 8), (3, 1)), 8),
    (torch.zeros(10, 8)[::2], 16), (torch.zeros(5, 1), 1), (torch.zeros(5, 4)[:, :1], 4), (torch.zeros(0, 8), 8)],
    ids=["whole", "columns of a wider one", "a row", "an expanded row", "a row of any stride", "every other row", "a column", "a column of a wider one", "no rows"])
def test_matrices_that_are_rows(matrix, ld):
    assert binding._rows(matrix, CPU) == (matrix.data_ptr(), binding.F32, *matrix.shape, ld)
