"""Adapters of many rows on the host: every batch that pwlq_block.h allows passes the checks of its sizes.  h, which is checked behind
them, is left out, so nothing is launched."""
import ctypes

import pytest

from test_block_abi_cpu import BF16, EINVAL, ENULL, F32, FAKE, ROOM, Adapter, AdapterBackward, calls, rows  # noqa: F401
from test_abi_cpu import lib  # noqa: F401

SIZES = [(340000, 4096, 11008), (700000, 4096, 4096), (5000000, 64, 64), (1 << 26, 1 << 20, 64), (1 << 26, 64, 1 << 20), (1 << 26, 1 << 20, 1 << 20)]


def forward(T, K, N):
    return Adapter(T, K, N, 8, 2, BF16, FAKE, FAKE, FAKE, FAKE, rows(K), rows(N, F32), rows(N), None)


def backward(T, K, N):
    return AdapterBackward(T, K, N, 8, 2, BF16, FAKE, FAKE, FAKE, FAKE, rows(N), rows(K), rows(K, F32), rows(K, F32), None, FAKE, FAKE)


@pytest.mark.parametrize("T,K,N", SIZES)
def test_many_rows_are_taken(calls, T, K, N):  # noqa: F811
    assert calls.pwlq_adapter(ctypes.byref(forward(T, K, N)), FAKE, ROOM, None) == ENULL
    assert calls.pwlq_last_error() == b"h is NULL"
    assert calls.pwlq_adapter_backward(ctypes.byref(backward(T, K, N)), FAKE, ROOM, None) == ENULL
    assert calls.pwlq_last_error() == b"h is NULL"
    assert calls.pwlq_adapter_backward_workspace_bytes(T, K, N, 8, 2) >= 4 * 8 * T


def test_what_lies_beyond_is_not(calls):  # noqa: F811
    for T, K, N in (((1 << 26) + 1, 64, 64), (40, (1 << 20) + 1, 64), (40, 64, (1 << 20) + 1)):
        assert calls.pwlq_adapter(ctypes.byref(forward(T, K, N)), FAKE, ROOM, None) == EINVAL
        assert calls.pwlq_adapter_backward(ctypes.byref(backward(T, K, N)), FAKE, ROOM, None) == EINVAL
        assert calls.pwlq_adapter_backward_workspace_bytes(T, K, N, 8, 2) == 0
