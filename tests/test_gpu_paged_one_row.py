"""A single row has no next one: whatever its stride says, calls take it (slices of odd widths, expanded tensors)."""
import pytest
import torch

from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu
H, D = 2, 64


def rows(dtype, stride):
    """[1][H][D] whose row stride is `stride` elements."""
    g = torch.Generator(device="cuda").manual_seed(1)
    return torch.randn(3 * max(stride, H * D), generator=g, device="cuda").to(dtype).as_strided((1, H, D), (stride, D, 1))


@pytest.mark.parametrize("stride", [0, 1, H * D + 1, H * D + 3, 1000003])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_any_stride(dtype, stride):
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=1, n_seqs=1, max_pages=1, n_q_heads=H, n_kv_heads=H, head_dim=D)
    c.pages.reserve([0], [1])
    b = c.batch([0], [0], [1])
    x = rows(dtype, stride)
    same = x.clone(memory_format=torch.contiguous_format)
    want, got = torch.empty_like(same), torch.empty(2 * H * D, dtype=dtype, device="cuda").as_strided((1, H, D), (stride, D, 1))
    c.append(0, b, same, same)
    c.read(0, b, want, None)
    c.append(0, b, x, x)
    c.read(0, b, None, got)
    assert torch.equal(got, want)
    pos, table = torch.tensor([1], dtype=torch.int32, device="cuda"), torch.empty(4, D // 2, 2, device="cuda")
    native.rope_table(native.rope_frequencies(D)[0], table)
    turned = torch.empty_like(same)
    native.qk_rope(native.rope_args(same, None, turned, None, pos, table))
    native.qk_rope(native.rope_args(x, None, got, None, pos, table))
    assert torch.equal(got, turned)
    native.qk_rope(native.rope_args(x, None, x, None, pos, table))
    assert torch.equal(x, turned)
    if dtype == torch.bfloat16:
        c.attention(0, b, x, got)
        assert ((got.float() - want.float()).abs() <= want.float().abs() * 2.0 ** -8).all()  # (one key, one rounding)
    assert c.sync_status() == native.TSS_OK
