"""The native marshalling of the token-step calls (csrc/py_step.cpp), through a callback in place of the C entry point: what is
handed over, and what is refused before the call is made.  No GPU needed: without one every tensor is in host memory, which is
refused itself."""
import ctypes

import pytest
import torch

from paper_2601_08743_amd import _py_step
from paper_2601_08743_amd import binding as B

_I, _P = ctypes.c_int32, ctypes.c_void_p
CTX = (0x77, 8, 2, 64, 0, 1000, 0)


def _fail(*args):
    raise AssertionError("the call was made")


def _addr(n):
    return ctypes.cast(ctypes.CFUNCTYPE(_I, *([_P] * n))(_fail), _P).value


def test_host_tensors_are_refused():
    z = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt)
    tables = [z(2), z(2), z(2, 5), z(9), z(1), z(1), z(2), z(3), z(4, dt=torch.int64), z(4), z(4), z(4), z(2)]
    with pytest.raises(B.TcError, match="host memory") as e:
        _py_step.step_tables(_addr(3), CTX, *tables, None)
    assert e.value.code == B.TC_ERR_INVALID
    q, kv = torch.zeros(4, 8, 64), torch.zeros(4, 2, 64)
    with pytest.raises(B.TcError, match="host memory"):
        _py_step.rope_append(_addr(3), CTX, 0, q, kv, kv, z(4), None, 0, 1e4, z(4, dt=torch.int64), q, None)
    with pytest.raises(B.TcError, match="entries.*host memory"):
        _py_step.digest_blocks(_addr(3), CTX, 0, 1, z(4), z(1000, dt=torch.int8), 0)
    ws = z(100, dt=torch.uint8)
    with pytest.raises(B.TcError, match="workspace"):
        _py_step.select_blocks(_addr(3), CTX, 0, q, z(4), z(4), z(2, 5), z(1000, dt=torch.int8), 1, 2, 3, z(4, 2, 6), ws, None)
    with pytest.raises(B.TcError, match="workspace"):
        _py_step.block_attn(_addr(3), CTX, 0, q, z(4), z(4), z(2, 5), z(4, 2, 6), q, 0.1, ws, None)


def test_arguments_of_another_kind_are_errors_not_calls():
    z = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(B.TcError, match="entries is no tensor"):
        _py_step.digest_blocks(_addr(3), CTX, 0, 1, [1, 2], z, None)
    with pytest.raises(TypeError):
        _py_step.digest_blocks(_addr(3), CTX, 0, 1, z, z)
    with pytest.raises(TypeError):
        _py_step.digest_blocks(0, ("f", 8, 2, 64, 0, 1000, 0), 0, 1, z, z, None)
    with pytest.raises(B.TcError, match="block_table: expected 2 dimensions"):
        _py_step.select_blocks(_addr(3), CTX, 0, z, z, z, z, z, 1, 2, 3, z, z, None)
    with pytest.raises(B.TcError, match="bad context"):
        _py_step.digest_blocks(_addr(3), (1, 2), 0, 1, z, z, None)
