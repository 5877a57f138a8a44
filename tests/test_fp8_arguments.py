"""What the native 8-bit calls refuse before any pointer is handed on; no GPU needed."""
import pytest
import torch

from tests.test_fp8_host import E8M0, E4M3, all_arguments, eight, recorded  # noqa: F401  (a fixture)


def calls_with(name, **over):
    return next(dict(a, **over) for n, a, _ in all_arguments() if n == name)


@pytest.mark.parametrize("name", [n for n, a, _ in all_arguments() if "meta" in a])
def test_a_row_count_that_the_kernels_cannot_read(recorded, name):
    """meta is int32 on the tensors' device, as the others are: a pointer to anything else would be read all the same."""
    calls, seen = recorded
    for meta in (torch.zeros(2, dtype=torch.int32, device="meta"), torch.zeros(2, dtype=torch.int64), torch.zeros(2), torch.zeros(0, dtype=torch.int32)):
        with pytest.raises(AssertionError):
            getattr(calls, name)(**calls_with(name, meta=meta))
    assert name not in seen
    getattr(calls, name)(**calls_with(name, meta=None))
    assert seen[name]["meta_dev"] is None


def test_a_workspace_that_the_kernels_cannot_use(recorded):
    calls, seen = recorded
    for work in (torch.zeros(64, dtype=torch.uint8, device="meta"), torch.zeros(64, dtype=torch.uint8)[::2]):
        with pytest.raises(AssertionError):
            calls.mb_linear_fp8_wgrad(**calls_with("mb_linear_fp8_wgrad", workspace=work))
    assert "mb_linear_fp8_wgrad" not in seen
