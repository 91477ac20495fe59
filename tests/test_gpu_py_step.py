"""What the native marshalling of the token-step calls (csrc/py_step.cpp) hands over: every address, size, stride and stream, recorded by a
callback of the C entry point's own signature, from tensors of sizes that are all different."""
import ctypes

import pytest
import torch

from paper_2601_08743_amd import _py_step
from paper_2601_08743_amd import binding as B

pytestmark = pytest.mark.gpu
HQ, HKV, D = 6, 2, 64
DIGEST_BYTES = 1000


def _recorded(name, call, rc=0):
    """The arguments that the C entry point would have been given."""
    seen = []

    def record(*args):
        seen.append(args)
        return rc

    entry = getattr(B._lib, name)
    thunk = ctypes.CFUNCTYPE(entry.restype, *entry.argtypes)(record)       # (kept until the call is over)
    assert call(ctypes.cast(thunk, ctypes.c_void_p).value) == rc
    assert len(seen) == 1
    return [0 if x is None else x for x in seen[0]]


def _z(*shape, dt=torch.int32):
    return torch.zeros(shape, dtype=dt, device="cuda")


def _ctx():
    return (0x1234560, HQ, HKV, D, 0, DIGEST_BYTES, torch.cuda.current_device())


def _p(*tensors):
    return [t.data_ptr() for t in tensors]


def test_step_tables():
    a = dict(seq=_z(3), new=_z(3), table=_z(3, 7), spare=_z(11), used=_z(1), nxt=_z(1), end=_z(3), cu=_z(4), slot=_z(5, dt=torch.int64),
             pos=_z(5), tseq=_z(5), full=_z(5), status=_z(2))
    st = torch.cuda.Stream()
    got = _recorded("tc_step_tables", lambda fn: _py_step.step_tables(fn, _ctx(), *a.values(), st))
    p = dict(zip(a, _p(*a.values())))
    assert got == [0x1234560, p["seq"], p["new"], 3, p["table"], 7, p["spare"], 11, p["used"], p["nxt"], p["end"], p["cu"], p["slot"], p["pos"],
                   p["tseq"], p["full"], 5, p["status"], st.cuda_stream]
    assert len(set(p.values())) == len(p)


def test_rope_append():
    rows = torch.zeros((5, HQ + 2 * HKV + 1, D), device="cuda")
    q, k, v, slot, out = rows[:, :HQ], rows[:, HQ:HQ + HKV], rows[:, HQ + HKV:HQ + 2 * HKV], _z(5, dt=torch.int64), torch.zeros((5, HQ, D), device="cuda")
    pos, sections = _z(3, 5), (ctypes.c_int32 * 3)(10, 12, 10)
    stride = (HQ + 2 * HKV + 1) * D
    got = _recorded("tc_rope_append", lambda fn: _py_step.rope_append(fn, _ctx(), 9, q, k, v, pos, ctypes.addressof(sections), 3, 1234.5, slot, out, 77))
    assert got == [0x1234560, 9, q.data_ptr(), stride, k.data_ptr(), stride, v.data_ptr(), stride, pos.data_ptr(), 3, ctypes.addressof(sections),
                   1234.5, slot.data_ptr(), 5, out.data_ptr(), 77]
    q1, k1, v1 = (torch.zeros((5, h, D), device="cuda") for h in (HQ, HKV, HKV))
    got = _recorded("tc_rope_append", lambda fn: _py_step.rope_append(fn, _ctx(), 0, q1, k1, v1, pos[1], None, 0, 2.0, slot, q1, None))
    assert got == [0x1234560, 0, q1.data_ptr(), HQ * D, k1.data_ptr(), HKV * D, v1.data_ptr(), HKV * D, pos[1].data_ptr(), 1, 0, 2.0, slot.data_ptr(), 5,
                   q1.data_ptr(), 0]


def test_digest_blocks():
    entries, digests = _z(4, 3), _z(DIGEST_BYTES, dt=torch.int8)
    got = _recorded("tc_digest_blocks", lambda fn: _py_step.digest_blocks(fn, _ctx(), 2, 5, entries, digests, 99))
    assert got == [0x1234560, 2, 5, entries.data_ptr(), 12, digests.data_ptr(), 99]


def test_select_blocks():
    q, seq, pos, table, dig = torch.zeros((5, HQ, D), device="cuda"), _z(5), _z(5), _z(3, 7), _z(DIGEST_BYTES, dt=torch.int8)
    lists, ws = _z(5, HKV, 1 + 4 + 6), _z(333, dt=torch.uint8)
    got = _recorded("tc_select_blocks", lambda fn: _py_step.select_blocks(fn, _ctx(), 8, q, seq, pos, table, dig, 1, 4, 6, lists, ws, 55))
    assert got == [0x1234560, 8, q.data_ptr(), seq.data_ptr(), pos.data_ptr(), 5, table.data_ptr(), 3, 7, dig.data_ptr(), 1, 4, 6, lists.data_ptr(),
                   ws.data_ptr(), 333, 55]


def test_block_attn():
    q, seq, pos, table = torch.zeros((5, HQ, D), device="cuda"), _z(5), _z(5), _z(3, 7)
    lists, out, ws = _z(5, HKV, 13), torch.zeros((5, HQ, D), device="cuda"), _z(333, dt=torch.uint8)
    got = _recorded("tc_block_attn", lambda fn: _py_step.block_attn(fn, _ctx(), 8, q, seq, pos, table, lists, out, 0.25, ws, None))
    assert got == [0x1234560, 8, q.data_ptr(), seq.data_ptr(), pos.data_ptr(), 5, table.data_ptr(), 3, 7, lists.data_ptr(), 13, out.data_ptr(), 0.25,
                   ws.data_ptr(), 333, 0]


def test_a_status_comes_back_as_it_is():
    got = _recorded("tc_digest_blocks", lambda fn: _py_step.digest_blocks(fn, _ctx(), 0, 1, _z(1), _z(DIGEST_BYTES, dt=torch.int8), None), rc=-5)
    assert got[6] == 0


def test_what_is_refused_makes_no_call():
    def fail(*args):
        raise AssertionError("the call was made")

    entry = B._lib.tc_block_attn
    thunk = ctypes.CFUNCTYPE(entry.restype, *entry.argtypes)(fail)
    fn = ctypes.cast(thunk, ctypes.c_void_p).value
    a = dict(q=torch.zeros((5, HQ, D), device="cuda"), seq=_z(5), pos=_z(5), table=_z(3, 7), lists=_z(5, HKV, 13),
             out=torch.zeros((5, HQ, D), device="cuda"), scale=0.25, ws=_z(64, dt=torch.uint8))
    for name, bad in (("q", a["q"].transpose(0, 1).contiguous().transpose(0, 1)), ("q", a["q"][:, :4]), ("q", a["q"].half()), ("seq", _z(10)[::2]),
                      ("pos", _z(4)), ("table", _z(7, 3).T), ("lists", _z(5, 13, HKV).transpose(1, 2)), ("out", a["out"][:4]), ("out", a["out"].cpu()),
                      ("ws", _z(64)), ("ws", _z(8, 8, dt=torch.uint8).T)):
        with pytest.raises(B.TcError) as e:
            _py_step.block_attn(fn, _ctx(), 0, *dict(a, **{name: bad}).values(), None)
        assert e.value.code == B.TC_ERR_INVALID
