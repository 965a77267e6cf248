"""Host side of pwlq_block.h without a GPU: workspace sizes, empty batches, and what is refused before anything is launched.
No pointer is dereferenced on the host but the argument structures."""
import ctypes

import pytest

from test_abi_cpu import lib  # noqa: F401  (the module's fixture)

VP, I64, CI, SZ, CF = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_float
FAKE, ROOM = 0x10000, 1 << 62
EINVAL, ENULL, EWORKSPACE = 1, 2, 3
F32, BF16, F16, I8 = 0, 1, 2, 3


class Rows(ctypes.Structure):
    _fields_ = [("data", VP), ("step", VP), ("stride", I64), ("type", CI)]


class Norm(ctypes.Structure):
    _fields_ = [("T", I64), ("D", I64), ("x", Rows), ("f", Rows), ("x_out", Rows), ("u", Rows), ("post", VP), ("pre", VP),
                ("gate", VP), ("gate_rows", I64), ("alpha", CF), ("eps", CF)]


class NormBackward(ctypes.Structure):
    _fields_ = [("T", I64), ("D", I64), ("du", Rows), ("dx_out", Rows), ("x_out", Rows), ("f", Rows), ("dx", Rows), ("df", Rows),
                ("post", VP), ("pre", VP), ("gate", VP), ("gate_rows", I64), ("alpha", CF), ("eps", CF), ("d_pre", VP),
                ("d_post", VP), ("d_gate", VP)]


class Adapter(ctypes.Structure):
    _fields_ = [("T", I64), ("K", I64), ("N", I64), ("R", CI), ("adapters", CI), ("weight_type", CI), ("down", VP), ("up", VP),
                ("ids", VP), ("scale", VP), ("x", Rows), ("base", Rows), ("out", Rows), ("h", VP)]


class AdapterBackward(ctypes.Structure):
    _fields_ = [("T", I64), ("K", I64), ("N", I64), ("R", CI), ("adapters", CI), ("weight_type", CI), ("down", VP), ("up", VP),
                ("ids", VP), ("scale", VP), ("dy", Rows), ("x", Rows), ("dx_base", Rows), ("dx", Rows), ("h", VP), ("d_down", VP),
                ("d_up", VP)]


@pytest.fixture(scope="module")
def calls(lib):  # noqa: F811
    for name, types in (("pwlq_pack_rows", [VP, I64, I64, VP, VP, VP]), ("pwlq_unpack_rows", [VP, VP, I64, I64, VP, VP]),
                        ("pwlq_norm_block", [VP, VP]), ("pwlq_norm_block_backward", [VP, VP, SZ, VP]),
                        ("pwlq_adapter", [VP, VP, SZ, VP]), ("pwlq_adapter_backward", [VP, VP, SZ, VP])):
        getattr(lib, name).restype, getattr(lib, name).argtypes = CI, types
    for name, types in (("pwlq_norm_block_backward_workspace_bytes", [I64, I64, I64]), ("pwlq_adapter_workspace_bytes", [I64, I64, CI]),
                        ("pwlq_adapter_backward_workspace_bytes", [I64, I64, I64, CI, CI])):
        getattr(lib, name).restype, getattr(lib, name).argtypes = SZ, types
    lib.pwlq_last_error.restype = ctypes.c_char_p
    return lib


def rows(cols, type_=BF16, data=FAKE, step=None, stride=None):
    return Rows(data, step, cols if stride is None else stride, type_)


def changed(args, **kw):
    new = type(args).from_buffer_copy(args)
    for k, v in kw.items():
        setattr(new, k, v)
    return new


def test_workspace_sizes(calls):
    for T in (0, 1, 12, 13, 17, 63, 64, 65, 511, 513, 4096, 100000):
        for K in (1, 63, 128, 4096, 11008):
            for R in (1, 16, 17, 256):
                # parts of long reductions only, and none where few rows take one launch
                if (T <= 12 and (R + 15) // 16 * ((K + 4095) // 4096) <= 3) or K <= 512:
                    assert calls.pwlq_adapter_workspace_bytes(T, K, R) == 0
                for n in (1, 32):
                    # the adapters' gradients come in parts only where rows leave something to split
                    need = calls.pwlq_adapter_backward_workspace_bytes(T, K, 1000, R, n)
                    assert need >= 4 * T * R and (need > 0) == (T > 0)
            for G in {0, 1, T}:
                if G <= T:
                    assert calls.pwlq_norm_block_backward_workspace_bytes(T, min(K, 16384), G) >= (4 * G if T else 0)
    assert calls.pwlq_adapter_workspace_bytes(-1, 8, 8) == 0
    assert calls.pwlq_adapter_workspace_bytes(8, 8, 257) == 0
    assert calls.pwlq_adapter_backward_workspace_bytes(8, 8, 8, 8, 0) == 0
    assert calls.pwlq_adapter_backward_workspace_bytes(8, 8, 0, 8, 1) == 0
    assert calls.pwlq_norm_block_backward_workspace_bytes(8, 16385, 0) == 0
    assert calls.pwlq_norm_block_backward_workspace_bytes(8, 64, 9) == 0


def test_packed_rows(calls):
    def pack(x=rows(64), T=4, K=64, codes=FAKE, step=FAKE):
        return calls.pwlq_pack_rows(ctypes.byref(x) if x else None, T, K, codes, step, None)

    assert pack(T=0) == 0
    assert pack(x=None) == ENULL and pack(codes=None) == ENULL and pack(step=None) == ENULL and pack(x=rows(64, data=None)) == ENULL
    assert pack(T=-1) == EINVAL and pack(K=0) == EINVAL and pack(K=65537) == EINVAL and pack(T=1 << 27) == EINVAL
    assert pack(x=rows(64, I8, step=FAKE)) == EINVAL and pack(x=rows(64, 7)) == EINVAL and pack(x=rows(64, -1)) == EINVAL
    assert pack(x=rows(64, stride=63)) == EINVAL and pack(x=rows(64, data=FAKE + 1)) == EINVAL and pack(x=rows(64, step=FAKE)) == EINVAL
    assert b"steps" in calls.pwlq_last_error()
    out = rows(64)
    assert calls.pwlq_unpack_rows(None, FAKE, 4, 64, ctypes.byref(out), None) == ENULL
    assert calls.pwlq_unpack_rows(FAKE, FAKE, 4, 64, None, None) == ENULL
    assert calls.pwlq_unpack_rows(FAKE, FAKE, 4, 65, ctypes.byref(out), None) == EINVAL
    assert calls.pwlq_unpack_rows(FAKE, FAKE, 0, 64, ctypes.byref(out), None) == 0


def test_norms(calls):
    ok = Norm(4, 64, rows(64), rows(64), rows(64), rows(64), FAKE, FAKE, FAKE, 2, 1.0, 1e-6)

    def call(**kw):
        return calls.pwlq_norm_block(ctypes.byref(changed(ok, **kw)), None)

    assert call(T=0) == 0
    assert calls.pwlq_norm_block(None, None) == ENULL
    assert call(pre=None) == ENULL and call(x=rows(64, data=None)) == ENULL and call(u=rows(64, data=None)) == ENULL
    assert call(x_out=rows(64, data=None)) == ENULL and call(u=rows(64, I8)) == ENULL
    assert call(D=16385) == EINVAL and call(gate_rows=3) == EINVAL and call(gate_rows=0) == EINVAL
    assert call(x=rows(64, F16)) == EINVAL and call(x_out=rows(64, F32)) == EINVAL and call(u=rows(64, F32)) == EINVAL
    assert call(f=rows(64, I8, step=FAKE)) == EINVAL and call(f=rows(64, data=None)) == EINVAL and call(f=rows(64, F32)) == EINVAL

    ok = NormBackward(4, 64, rows(64), rows(64), rows(64), rows(64), rows(64), rows(64), FAKE, FAKE, FAKE, 2, 1.0, 1e-6, FAKE, FAKE, FAKE)

    def back(workspace=FAKE, room=ROOM, **kw):
        return calls.pwlq_norm_block_backward(ctypes.byref(changed(ok, **kw)), workspace, room, None)

    assert calls.pwlq_norm_block_backward(None, FAKE, ROOM, None) == ENULL
    assert back(d_pre=None) == ENULL and back(d_post=None) == ENULL and back(post=None) == ENULL and back(d_gate=None) == ENULL
    assert back(dx=rows(64, data=None)) == ENULL and back(df=rows(64, data=None)) == ENULL and back(x_out=rows(64, I8)) == ENULL
    assert back(x_out=rows(64, I8, step=FAKE)) == EINVAL and back(f=rows(64, I8, step=FAKE)) == EINVAL
    assert back(du=rows(64, F32)) == EINVAL and back(dx_out=rows(64, F32)) == EINVAL and back(dx=rows(64, F32)) == EINVAL
    assert back(f=rows(64, data=None)) == EINVAL and back(gate_rows=3) == EINVAL
    assert back(workspace=None) == EWORKSPACE and back(workspace=FAKE + 16) == EWORKSPACE and back(room=64) == EWORKSPACE


def test_adapters(calls):
    ok = Adapter(40, 1024, 48, 8, 2, BF16, FAKE, FAKE, FAKE, FAKE, rows(1024), rows(48, F32, step=FAKE), rows(48), FAKE)

    def call(workspace=FAKE, room=ROOM, **kw):
        return calls.pwlq_adapter(ctypes.byref(changed(ok, **kw)), workspace, room, None)

    assert call(T=0) == 0 and call(T=0, ids=None) == 0
    assert calls.pwlq_adapter(None, FAKE, ROOM, None) == ENULL
    for name in ("down", "up", "ids", "scale", "h"):
        assert call(**{name: None}) == ENULL, name
    assert call(x=rows(1024, I8)) == ENULL and call(out=rows(48, data=None)) == ENULL
    assert call(R=0) == EINVAL and call(R=257) == EINVAL and call(adapters=0) == EINVAL and call(adapters=65536) == EINVAL
    assert call(K=0) == EINVAL and call(N=0) == EINVAL and call(N=(1 << 20) + 1) == EINVAL and call(T=-1) == EINVAL
    assert call(T=1 << 26, N=1 << 20) == EINVAL and call(T=1 << 26, K=1 << 20) == EINVAL
    assert call(weight_type=I8) == EINVAL and call(weight_type=F16) == EINVAL and call(down=FAKE + 1) == EINVAL
    assert call(x=rows(1024, F32)) == EINVAL and call(out=rows(48, I8, step=FAKE)) == EINVAL and call(base=rows(48, F16)) == EINVAL
    assert call(x=rows(1024, stride=1020)) == EINVAL and call(x=rows(1024, step=FAKE)) == EINVAL
    assert call(workspace=None) == EWORKSPACE and call(workspace=FAKE + 8) == EWORKSPACE and call(room=8) == EWORKSPACE

    ok = AdapterBackward(40, 64, 48, 8, 2, BF16, FAKE, FAKE, FAKE, FAKE, rows(48), rows(64, I8, step=FAKE), rows(64, F32), rows(64, F32),
                         FAKE, FAKE, FAKE)

    def back(workspace=FAKE, room=ROOM, **kw):
        return calls.pwlq_adapter_backward(ctypes.byref(changed(ok, **kw)), workspace, room, None)

    assert calls.pwlq_adapter_backward(None, FAKE, ROOM, None) == ENULL
    for name in ("down", "up", "ids", "scale", "h", "d_down", "d_up"):
        assert back(**{name: None}) == ENULL, name
    assert back(dy=rows(48, F32)) == EINVAL and back(dy=rows(48, I8, step=FAKE)) == EINVAL and back(dx=rows(64, F16)) == EINVAL
    assert back(dx_base=rows(64, I8, step=FAKE)) == EINVAL and back(dx=rows(64, data=None)) == ENULL
    assert back(workspace=None) == EWORKSPACE and back(room=100) == EWORKSPACE
