"""Arguments of the feed-forward and AdamW calls that are refused, or taken, at the ends of their ranges (no device needed)."""
import pytest


@pytest.mark.parametrize("dtype", ["float16", "float64", "int32"])
def test_adamw_gradients_of_other_types_are_refused_as_the_other_lists_are(dtype):
    import torch
    from paper_2408_11500_b200 import binding as B
    t = torch.zeros(4)
    with pytest.raises(ValueError):
        B.make_adamw_desc([t], [t.to(getattr(torch, dtype))], [t], [t])
    B.make_adamw_desc([t], [t.to(torch.bfloat16)], [t], [t])
