"""What the channel products take as rows where it lies (no GPU needed)."""
import pytest
import torch

from paper_2204_03643_amd.linear import _as_rows


def test_rows_too_far_apart_are_copied():
    """Strides of 2^31 and more are refused by the library; such rows are copied instead."""
    for stride, ld in (((1 << 31) - 1, (1 << 31) - 1), (1 << 31, 4), (1 << 33, 4)):
        rows, got = _as_rows(torch.empty_strided((3, 4), (stride, 1), device="meta"))
        assert got == ld and (rows.is_contiguous() == (ld == 4))


@pytest.mark.parametrize("t", [torch.randn(6, 1, dtype=torch.complex64).conj().imag, torch.randn(6, 5, dtype=torch.complex64).conj().imag,
                               torch.randn(6, 8)[:, :5], torch.randn(6, 8)[::2, 3:], torch.randn(8, 6).t(), torch.randn(2, 3, 8)[..., :5],
                               torch.randn(5).expand(6, 5), torch.randn(6, 8)[:, ::2], torch.randn(1, 8)[:, :5]],
                         ids=["a negated column", "negated", "part of rows", "every other row", "transposed", "three axes", "one row for all",
                              "every other column", "one row"])
def test_memory_holds_what_the_tensor_does(t):
    rows, ld = _as_rows(t)
    count = t.numel() // t.shape[-1]
    raw = torch.empty(0, dtype=t.dtype).set_(rows.untyped_storage())
    memory = torch.as_strided(raw, (count, t.shape[-1]), (ld, 1), rows.storage_offset())
    assert torch.equal(memory, t.reshape(count, t.shape[-1]).clone())
