"""Host side of pwlq_attention.h without a GPU: workspace sizes, empty batches, and what is refused before anything is launched.
No pointer is dereferenced on the host but the argument structures."""
import ctypes

import pytest

from test_abi_cpu import lib  # noqa: F401  (the module's fixture)

VP, I64, CI, SZ, CF = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_float
FAKE, ROOM = 0x10000, 1 << 62
EINVAL, ENULL, EWORKSPACE = 1, 2, 3
F32, BF16, F16, I8 = 0, 1, 2, 3


class Cache(ctypes.Structure):
    _fields_ = [("keys", VP), ("values", VP), ("key_step", VP), ("value_step", VP), ("pages", I64), ("heads", CI), ("page", CI), ("D", CI),
                ("type", CI)]


class Batch(ctypes.Structure):
    _fields_ = [("S", I64), ("T", I64), ("table", VP), ("table_stride", I64), ("table_pages", I64), ("lengths", VP), ("starts", VP)]


class Heads(ctypes.Structure):
    _fields_ = [("data", VP), ("stride", I64), ("head_stride", I64), ("type", CI)]


class Append(ctypes.Structure):
    _fields_ = [("cache", Cache), ("batch", Batch), ("q", Heads), ("k", Heads), ("v", Heads), ("q_out", Heads), ("q_heads", CI),
                ("rotated", CI), ("interleaved", CI), ("positions", VP), ("frequencies", VP)]


class Read(ctypes.Structure):
    _fields_ = [("cache", Cache), ("batch", Batch), ("k", Heads), ("v", Heads)]


class Attend(ctypes.Structure):
    _fields_ = [("cache", Cache), ("batch", Batch), ("q", Heads), ("out", Heads), ("q_heads", CI), ("scale", CF), ("cap", CF),
                ("slopes", VP), ("window", I64), ("prefix", VP), ("tree", VP), ("tree_words", I64), ("longest", I64)]


@pytest.fixture(scope="module")
def calls(lib):  # noqa: F811
    for name, types in (("pwlq_append", [VP, VP]), ("pwlq_read", [VP, VP]), ("pwlq_attend", [VP, VP, SZ, VP])):
        getattr(lib, name).restype, getattr(lib, name).argtypes = CI, types
    lib.pwlq_attend_workspace_bytes.restype, lib.pwlq_attend_workspace_bytes.argtypes = SZ, [VP]
    lib.pwlq_last_error.restype = ctypes.c_char_p
    return lib


def cache(**kw):
    return Cache(**{**dict(keys=FAKE, values=FAKE, key_step=None, value_step=None, pages=100, heads=8, page=64, D=128, type=BF16), **kw})


def batch(**kw):
    return Batch(**{**dict(S=4, T=4, table=FAKE, table_stride=32, table_pages=32, lengths=FAKE, starts=None), **kw})


def heads(n, type_=BF16, data=FAKE, stride=None, head_stride=128):
    return Heads(data, n * 128 if stride is None else stride, head_stride, type_)


NONE = Heads(None, 0, 0, 0)


def shared_refusals(call):
    for field in ("keys", "values"):
        assert call(cache=cache(**{field: None})) == ENULL
    for field in ("table", "lengths"):
        assert call(batch=batch(**{field: None})) == ENULL
    for bad in (dict(type=F32), dict(type=7), dict(type=-1), dict(D=0), dict(D=8), dict(D=72), dict(D=272), dict(D=-16), dict(page=8), dict(page=48),
                dict(page=0), dict(page=1 << 17), dict(heads=0), dict(heads=1025), dict(pages=-1), dict(pages=1 << 31), dict(pages=0),
                dict(keys=FAKE + 8), dict(values=FAKE + 2), dict(key_step=FAKE), dict(value_step=FAKE)):
        assert call(cache=cache(**bad)) == EINVAL, bad
    for bad in (dict(key_step=None), dict(value_step=None)):
        assert call(cache=cache(**{**dict(type=I8, key_step=FAKE, value_step=FAKE), **bad})) == ENULL, bad
    assert call(cache=cache(type=I8, key_step=FAKE + 4, value_step=FAKE)) == EINVAL
    for bad in (dict(T=-1), dict(S=-1), dict(T=5), dict(T=(1 << 20) + 1, starts=FAKE), dict(S=(1 << 20) + 1, starts=FAKE), dict(table_pages=0),
                dict(table_pages=-1), dict(table_pages=1 << 25), dict(table_stride=31), dict(table=FAKE + 2), dict(lengths=FAKE + 1),
                dict(starts=FAKE + 2)):
        assert call(batch=batch(**bad)) == EINVAL, bad
    # a sequence has room for 2^30 rows at most: one page more is refused, before anything else is looked at
    for page in (16, 64, 65536):
        most = (1 << 30) // page
        assert call(cache=cache(page=page), batch=batch(S=0, T=0, table_pages=most)) == 0
        assert call(cache=cache(page=page), batch=batch(S=0, T=0, table_pages=most + 1)) == EINVAL
    assert call(batch=batch(S=0, T=0, table=None, lengths=None), cache=cache(keys=None)) == 0
    assert call(batch=batch(S=0, T=4, starts=FAKE)) == 0 and call(batch=batch(S=4, T=0, starts=FAKE)) == 0


def refused_heads(call, name, n, output):
    assert call(**{name: heads(n, data=None)}) == ENULL
    for bad in (heads(n, F32), heads(n, F16), heads(n, I8), heads(n, data=FAKE + 1), heads(n, stride=-1), heads(n, head_stride=-128),
                heads(n, stride=1 << 41)):
        assert call(**{name: bad}) == EINVAL, name
    if output:
        for bad in (heads(n, stride=0), heads(n, head_stride=0), heads(n, stride=n * 128 - 1), heads(n, head_stride=127)):
            assert call(**{name: bad}) == EINVAL, name


def test_append(calls):
    ok = Append(cache(), batch(), heads(32), heads(8), heads(8), heads(32), 32, 128, 0, FAKE, FAKE)

    def call(**kw):
        new = Append.from_buffer_copy(ok)
        for k, v in kw.items():
            setattr(new, k, v)
        return calls.pwlq_append(ctypes.byref(new), None)

    assert calls.pwlq_append(None, None) == ENULL
    shared_refusals(call)
    for name, n in (("k", 8), ("v", 8), ("q", 32)):
        if name != "q":
            refused_heads(call, name, n, False)
    refused_heads(call, "q_out", 32, True)
    assert call(q=heads(32, F16)) == EINVAL and call(q=heads(32, data=None)) == ENULL
    assert call(q_heads=0) == EINVAL and call(q_heads=12) == EINVAL and call(q_heads=4) == EINVAL and call(q_heads=2048) == EINVAL
    assert call(rotated=8) == EINVAL and call(rotated=144) == EINVAL and call(rotated=-16) == EINVAL and call(frequencies=None) == ENULL
    assert call(frequencies=FAKE + 1) == EINVAL and call(positions=FAKE + 2) == EINVAL
    assert call(cache=cache(type=F16)) == EINVAL


def test_read(calls):
    ok = Read(cache(), batch(), heads(8), heads(8))

    def call(**kw):
        new = Read.from_buffer_copy(ok)
        for k, v in kw.items():
            setattr(new, k, v)
        return calls.pwlq_read(ctypes.byref(new), None)

    assert calls.pwlq_read(None, None) == ENULL
    shared_refusals(call)
    assert call(k=NONE, v=NONE) == ENULL and call(k=heads(8, F16)) == EINVAL and call(k=heads(8, I8)) == EINVAL
    assert call(v=heads(8, stride=0)) == EINVAL and call(k=heads(8, head_stride=100)) == EINVAL


def test_attend(calls):
    ok = Attend(cache(), batch(), heads(32), heads(32), 32, 0.1, 0.0, None, 0, None, None, 0, 0)

    def call(workspace=FAKE, room=ROOM, **kw):
        new = Attend.from_buffer_copy(ok)
        for k, v in kw.items():
            setattr(new, k, v)
        return calls.pwlq_attend(ctypes.byref(new), workspace, room, None)

    def need(**kw):
        new = Attend.from_buffer_copy(ok)
        for k, v in kw.items():
            setattr(new, k, v)
        return calls.pwlq_attend_workspace_bytes(ctypes.byref(new))

    assert calls.pwlq_attend(None, FAKE, ROOM, None) == ENULL and calls.pwlq_attend_workspace_bytes(None) == 0
    shared_refusals(call)
    refused_heads(call, "out", 32, True)
    assert call(q=heads(32, data=None)) == ENULL and call(q=heads(32, F16)) == EINVAL and call(q=heads(32, F32)) == EINVAL
    for bad in (dict(q_heads=0), dict(q_heads=12), dict(q_heads=2048), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")),
                dict(window=-1), dict(longest=-1), dict(slopes=FAKE + 2), dict(prefix=FAKE + 1), dict(tree=FAKE), dict(tree=FAKE, tree_words=1 << 15),
                dict(tree=FAKE, tree_words=1, window=5), dict(tree=FAKE, tree_words=1, slopes=FAKE), dict(tree=FAKE, tree_words=1, prefix=FAKE),
                dict(tree=FAKE + 4, tree_words=1)):
        assert call(**bad) == EINVAL, bad
    for bad in (dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-2.0 ** 61), dict(cap=2.0 ** -61), dict(cap=1e-44), dict(cap=2.0 ** 61),
                dict(cap=2.9e38)):
        assert call(**bad) == EINVAL, bad
    for good in (dict(scale=2.0 ** 60), dict(scale=-2.0 ** 60), dict(cap=2.0 ** -60), dict(cap=2.0 ** 60)):
        assert call(workspace=None, **good) == EWORKSPACE, good
    assert call(workspace=None) == EWORKSPACE and call(workspace=FAKE + 128) == EWORKSPACE and call(room=1000) == EWORKSPACE
    assert need() > 0 and need(batch=batch(S=0, T=0)) == 0 and need(q_heads=12) == 0 and need(cache=cache(D=8)) == 0
    # no parts, and so no workspace, where the items fill the chip by themselves
    assert need(batch=batch(S=4, T=1 << 16, starts=FAKE)) == 0
    assert need(batch=batch(S=1 << 20, T=1 << 20)) == 0
    for S in (1, 7, 300, 2047, 2048):
        for q_heads in (8, 40, 1024):
            for D in (16, 64, 80, 128, 256):
                for T in (S, 5 * S, 50 * S):
                    bytes_ = need(batch=batch(S=S, T=T, starts=FAKE), q_heads=q_heads, cache=cache(D=D))
                    assert 0 <= bytes_ < 1 << 30
