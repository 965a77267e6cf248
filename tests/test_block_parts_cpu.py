"""How the rows of the adapters' gradients are split, as the workspace shows it: a part leaves a sum for each adapter."""
import pytest

from test_block_abi_cpu import calls  # noqa: F401
from test_abi_cpu import lib  # noqa: F401


def parts(calls, T, K, N, R, n):  # noqa: F811
    """The parts that the workspace has room for beside H and its parts, and the workgroups of one part."""
    room = calls.pwlq_adapter_backward_workspace_bytes(T, K, N, R, n) - 4 * T * R - calls.pwlq_adapter_workspace_bytes(T, N, R)
    return room // (4 * n * R * (K + N)), ((K + 127) // 128 + (N + 127) // 128) * (1 if R <= 16 else (R + 31) // 32)


@pytest.mark.parametrize("T,K,N,R", [(8192, 4096, 4096, 16), (32768, 4096, 4096, 16), (65536, 1024, 1024, 16), (16384, 4096, 11008, 32),
                                     (1 << 20, 512, 512, 8)])
@pytest.mark.parametrize("n", [2, 64, 512, 4096])
def test_a_large_bank_does_not_leave_long_parts(calls, T, K, N, R, n):  # noqa: F811
    """Rows that all have one adapter of many: a part of them is walked by one workgroup for each 128 columns, so there are parts
    for the whole chip or of 4096 rows, however many other adapters there are, as far as their sums fit 4 GiB."""
    got, workgroups = parts(calls, T, K, N, R, n)
    want = min((1024 if R <= 16 else 512) // workgroups, T // 4096, 2 ** 32 // (4 * n * R * (K + N)))
    assert got >= want or want == 1


def test_the_sums_of_a_huge_bank_fit_beside_it(calls):  # noqa: F811
    each = 4 * 65535 * 16 * 8192
    assert calls.pwlq_adapter_backward_workspace_bytes(1 << 20, 4096, 4096, 16, 65535) <= each


def test_few_rows_of_many_adapters_leave_few_sums(calls):  # noqa: F811
    assert parts(calls, 534, 4096, 4096, 16, 32)[0] <= 1
    assert parts(calls, 4095, 4096, 4096, 16, 512)[0] <= 1
