"""GPU: matrices of codes and scales in another layout than the library's are refused; flat ones are taken as they lie."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_other_layouts_are_refused():
    import paper_1908_05033_b200 as dsq
    n, k, group = 48, 192, 64
    w = torch.randn(n, k, device="cuda").bfloat16()
    codes, scales = dsq.dsq_quantize_groups(w, 4, group)
    x = torch.randn(3, k, device="cuda").bfloat16()

    def values(c, s):
        return dsq.dsq_dequantize_groups(c, s, n, k, 4, group)

    def product(c, s):
        return dsq.dsq_wgemm_group(x, c, 3, n, k, 4, group, s)

    turned = scales.t().contiguous()                      # [N, groups]
    wider = torch.zeros(n, codes.shape[1] + 16, dtype=torch.uint8, device="cuda")
    wider[:, :codes.shape[1]] = codes
    for call in (values, product):
        ref = call(codes, scales)
        assert torch.equal(call(codes.view(-1), scales.view(-1)), ref)
        for c, s in ((codes, turned), (wider, scales)):
            with pytest.raises(ValueError):
                call(c, s)
    with pytest.raises(dsq.DsqError):                     # (another width is the library's to refuse)
        dsq.dsq_dequantize_groups(codes, scales, n, k, 3, group)
