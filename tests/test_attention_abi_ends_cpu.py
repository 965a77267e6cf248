"""The ends of what pwlq_attend takes for window and longest, on the host: they choose as the largest numbers that mean anything do."""
import ctypes

import pytest

from test_abi_cpu import lib  # noqa: F401  (the module's fixture)
from test_attention_abi_cpu import EWORKSPACE, FAKE, Attend, batch, cache, calls, heads  # noqa: F401

MOST = 2 ** 63 - 1


@pytest.mark.parametrize("T,S", [(4, 4), (1000, 4), (1 << 20, 1), (1 << 20, 1 << 20)])
@pytest.mark.parametrize("q_heads,kv_heads", [(32, 8), (1024, 1), (8, 8)])
def test_windows_and_longest_sequences_of_any_size(calls, T, S, q_heads, kv_heads):  # noqa: F811
    def args(**kw):
        a = Attend(cache(heads=kv_heads), batch(S=S, T=T, starts=FAKE), heads(q_heads), heads(q_heads), q_heads, 0.1, 0.0, None, 0, None, None, 0, 0)
        for k, v in kw.items():
            setattr(a, k, v)
        return a

    def need(**kw):
        return calls.pwlq_attend_workspace_bytes(ctypes.byref(args(**kw)))

    room = 32 * 64                                          # rows of a table
    for window in (room, room + 1, 2 ** 31 - 1, 2 ** 31, 2 ** 40, MOST - 1000, MOST):
        assert need(window=window) == need()                # it holds nothing back
    for longest in (T + 1, 2 ** 31, 2 ** 53, MOST // 1000, MOST):
        assert need(longest=longest) == need(longest=T)
    for kw in (dict(window=MOST), dict(longest=MOST), dict(window=MOST, longest=MOST)):
        if need(**kw):
            assert calls.pwlq_attend(ctypes.byref(args(**kw)), None, 0, None) == EWORKSPACE
