"""The empty 8-bit cache that kv8_cache makes."""

import pytest

torch = pytest.importorskip("torch")

import paper_2606_12487_amd as dptq  # noqa: E402


@pytest.mark.parametrize("default", [torch.float16, torch.bfloat16, torch.float32, torch.float64])
def test_dtypes_do_not_depend_on_torch_s_default(default):
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        cache = dptq.kv8_cache(3, 2, 64, device="cpu")
    finally:
        torch.set_default_dtype(before)
    assert cache.k_pages.dtype == cache.v_pages.dtype == torch.float8_e4m3fn
    assert cache.k_scales.dtype == cache.v_scales.dtype == torch.float32
    assert cache.k_pages.shape == (3, 2, 64, 64) and cache.v_scales.shape == (3, 2)
