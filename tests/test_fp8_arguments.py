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


def test_sizes_of_more_than_32_bits_do_not_wrap(recorded):
    """They arrive as the largest int, which the library refuses; modulo 2^32 they would be small sizes that look right."""
    calls, seen = recorded
    most, far = 2 ** 31 - 1, 2 ** 32 + 16

    def rows(n, width, dtype=E4M3, block=1):
        q = torch.empty((n, width), dtype=dtype, device="meta")
        return q, torch.empty((-(-n // block), -(-width // 128)), dtype=E8M0, device="meta")

    calls.mb_fp8_quant(rows(far, 16, torch.bfloat16)[0])
    assert seen["mb_fp8_quant"]["T_cap"] == most
    calls.mb_fp8_dequant(*rows(far, 16))
    assert seen["mb_fp8_dequant"]["T_cap"] == most
    calls.mb_fp8_dequant(*rows(1, far))
    assert seen["mb_fp8_dequant"]["W"] == most
    calls.mb_fp8_quant_weight(rows(far, 16, torch.bfloat16)[0])
    assert seen["mb_fp8_quant_weight"]["n_out"] == most and seen["mb_fp8_quant_weight"]["n_in"] == 16
    calls.mb_linear_fp8_fwd(*rows(1, far), *rows(16, far, block=128))
    assert seen["mb_linear_fp8_fwd"]["n_in"] == most
    calls.mb_linear_fp8_wgrad(rows(far, 16, torch.bfloat16)[0], *rows(far, 16))
    assert seen["mb_linear_fp8_wgrad"]["T_cap"] == most
    calls.mb_geglu_fp8_act(*rows(far, 16), *rows(256, 16, block=128))
    assert seen["mb_geglu_fp8_act"]["T_cap"] == most
    calls.mb_gelu_gate_fp8_bwd(rows(far, 128, torch.bfloat16)[0], rows(far, 256, torch.bfloat16)[0])
    assert seen["mb_gelu_gate_fp8_bwd"]["T_cap"] == most
    seen.clear()
    x = torch.zeros(20, 144)
    for count in (2 ** 32 + 5, 21):
        with pytest.raises(AssertionError):
            calls.mb_fp8_quant(x, T_cap=count)
    calls.mb_fp8_quant(rows(far, 16, torch.bfloat16)[0], T_cap=5)                # few rows of many: as before
    assert seen["mb_fp8_quant"]["T_cap"] == 5
    calls.mb_fp8_quant(x, T_cap=-1)                                              # (the library refuses it)
    assert seen["mb_fp8_quant"]["T_cap"] == -1
