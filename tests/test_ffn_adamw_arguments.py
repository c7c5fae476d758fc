"""Arguments of the feed-forward and AdamW calls that are refused, or taken, at the ends of their ranges (no device needed)."""
import pytest

from test_ffn_adamw_refusals import AT, _ffn, _status


@pytest.mark.parametrize("dtype", ["float16", "float64", "int32"])
def test_adamw_gradients_of_other_types_are_refused_as_the_other_lists_are(dtype):
    import torch
    from paper_2408_11500_b200 import binding as B
    t = torch.zeros(4)
    with pytest.raises(ValueError):
        B.make_adamw_desc([t], [t.to(getattr(torch, dtype))], [t], [t])
    B.make_adamw_desc([t], [t.to(torch.bfloat16)], [t], [t])


@pytest.mark.parametrize("scale", [1e39, -1e300])
def test_a_scale_past_fp32_is_refused(scale):
    """The kernels hold it in fp32, where it would be infinite, and its product with a zero none."""
    from paper_2408_11500_b200 import binding as B
    d = _ffn(scale=scale)
    for call in (lambda: B.slicegcn_ffn_workspace_bytes(d, AT, AT), lambda: B.slicegcn_ffn_forward(d, AT, None, AT, None, AT, 1 << 20),
                 lambda: B.slicegcn_ffn_backward(d, AT, AT, None, None, None, None, None, None, AT, 1 << 20)):
        assert _status(call) == B.ERR_INVALID_ARG
    B.slicegcn_ffn_workspace_bytes(_ffn(scale=3.4e38), AT, AT)
