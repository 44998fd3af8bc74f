"""CPU-side checks of the embedding's entry points: sizes and refusals, before anything is launched (the addresses are made
up: argument checks touch no memory)."""
import ctypes

import pytest
import torch

from paper_2305_12201_amd import binding as B


def _lookup(table=0x1000, table_type=B.FLOAT32, vocab=100, dim=16, table_stride=16, tokens=0x2000, token_bytes=8, n=0,
            scale=1.0, out=0x3000, out_type=B.FLOAT32, out_stride=16):
    return B.lib().gravac_embedding_lookup(table, table_type, vocab, dim, table_stride, tokens, token_bytes, n,
                                           ctypes.c_float(scale), out, out_type, out_stride, None)


def _gradient(grad=0x1000, grad_type=B.FLOAT32, n=10, dim=16, grad_stride=16, tokens=0x2000, token_bytes=8, padding=-1,
              scale=1.0, table=0x3000, vocab=100, table_stride=16, ws=0x10000, ws_bytes=None, flags=0):
    if ws_bytes is None:
        ws_bytes = 1 << 40
    return B.lib().gravac_embedding_gradient(grad, grad_type, n, dim, grad_stride, tokens, token_bytes, padding,
                                             ctypes.c_float(scale), table, vocab, table_stride, ws, ws_bytes, flags, None)


def test_lookup_of_no_tokens_launches_nothing():
    assert _lookup() == B.OK
    assert _lookup(tokens=0, out=0) == B.OK


@pytest.mark.parametrize("bad", [
    {"table": 0}, {"table": 0x1002}, {"table_type": 3}, {"table_type": -1}, {"vocab": 0}, {"vocab": 1 << 31}, {"dim": 0},
    {"dim": B.EMBEDDING_MAX_DIM + 1, "table_stride": 1 << 21, "out_stride": 1 << 21}, {"table_stride": 15},
    {"table_stride": 1 << 31}, {"out_stride": 15}, {"out_stride": 1 << 31}, {"n": -1}, {"n": B.EMBEDDING_MAX_TOKENS + 1},
    {"n": 4, "tokens": 0}, {"n": 4, "out": 0}, {"n": 4, "tokens": 0x2004}, {"n": 4, "token_bytes": 4, "tokens": 0x2002},
    {"n": 4, "out": 0x3001, "out_type": B.BFLOAT16}, {"n": 4, "out": 0x3002}, {"token_bytes": 2}, {"out_type": 7}])
def test_lookup_refuses(bad):
    assert _lookup(**bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    {"grad": 0}, {"grad": 0x1001, "grad_type": B.FLOAT16}, {"grad": 0x1002}, {"grad_type": 3}, {"n": -1},
    {"n": B.EMBEDDING_MAX_TOKENS + 1}, {"dim": 0}, {"dim": B.EMBEDDING_MAX_DIM + 1, "grad_stride": 1 << 21, "table_stride": 1 << 21},
    {"grad_stride": 15}, {"grad_stride": 1 << 31}, {"tokens": 0}, {"tokens": 0x2004}, {"token_bytes": 3}, {"table": 0},
    {"table": 0x3002}, {"vocab": 0}, {"vocab": 1 << 31}, {"table_stride": 15}, {"table_stride": 1 << 31}, {"flags": 1},
    {"flags": 32}])
def test_gradient_refuses(bad):
    assert _gradient(**bad) == B.ERR_INVALID_ARG


def test_gradient_refuses_workspaces():
    need = B.gravac_embedding_gradient_workspace_bytes(10, 100, 16)
    assert need > 0
    assert _gradient(ws=0) == B.ERR_WORKSPACE
    assert _gradient(ws=0x10080) == B.ERR_WORKSPACE
    assert _gradient(ws_bytes=need - 1) == B.ERR_WORKSPACE


def test_gradient_workspace_bytes():
    size = B.gravac_embedding_gradient_workspace_bytes
    for bad in ((-1, 10, 10), (10, 0, 10), (10, 10, 0), (10, 1 << 31, 10), (B.EMBEDDING_MAX_TOKENS + 1, 10, 10),
                (10, 10, B.EMBEDDING_MAX_DIM + 1)):
        with pytest.raises(B.GravacError) as e:
            size(*bad)
        assert e.value.code == B.ERR_INVALID_ARG
    assert size(0, 1, 1) <= size(1, 1, 1)
    # 16 bytes per token and two rows of partial sums per 4 tokens at most, beside half a megabyte
    for n, dim in ((1, 1), (129, 650), (4097, 64), (131_072, 4096), (1 << 20, 768)):
        assert 16 * n <= size(n, 50_000, dim) <= 16 * n + 2 * (n // 4 + 1) * 4 * (dim + 3) + 4 * n + (1 << 19)


def test_binding_refuses_host_tensors():
    if torch.cuda.is_available():
        pytest.skip("the binding asks for the current device first")
    with pytest.raises(Exception):
        B.gravac_embedding_lookup(torch.zeros(4, 4), torch.zeros(2, dtype=torch.int64), torch.zeros(2, 4))


# ---- buffers that share memory --------------------------------------------------------------------------------------
@pytest.mark.parametrize("bad", [
    {"out": 0x1000}, {"out": 0x1000 + 6400 - 4}, {"out": 0x1000 - 252},                       # 100 rows of 64 bytes, 4 of 64
    {"out": 0x1000 - 126, "out_type": B.BFLOAT16},
    {"table_stride": 40, "out": 0x1000 + 60, "out_stride": 40},                              # the last element of the row
    {"table_stride": 40, "out": 0x1000 + 100, "out_stride": 41},                             # ends in the next row
    {"table_stride": 40, "out": 0x1000 + 64, "out_stride": 50},                              # its second row lies in a row of the table
    {"table": 0x100000, "out": 0x2000}, {"table": 0x100000, "out": 0x201C}, {"table": 0x100000, "out": 0x2000 - 252},        # the tokens
    {"table": 0x100000, "out": 0x2000 - 60, "out_stride": 1 << 20}])
def test_lookup_refuses_shared_memory(bad):
    assert _lookup(**{"n": 4, **bad}) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    {"grad": 0x3000}, {"grad": 0x3000 + 6396}, {"grad": 0x3000 - 636}, {"grad": 0x3000 - 318, "grad_type": B.FLOAT16},
    {"table_stride": 40, "grad": 0x3000 + 60, "grad_stride": 40}, {"tokens": 0x3000}, {"tokens": 0x3000 - 72}, {"tokens": 0x4900 - 8},
    {"ws": 0x1000}, {"ws": 0x1200}, {"ws": 0x2000}, {"ws": 0x3000}, {"ws": 0x4800}, {"grad": 0x10000}, {"tokens": 0x10008}, {"table": 0x10000 + 4},
    {"table": 0x10000 - 6396}])
def test_gradient_refuses_shared_memory(bad):
    assert _gradient(**bad) == B.ERR_INVALID_ARG
