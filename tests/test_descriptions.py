"""Descriptions of the operators around the layers are ordinary values: a copy is the one that a call uses, not what it was made from."""
import copy
import pickle

import numpy as np
import pytest


@pytest.mark.parametrize("make", [copy.copy, copy.deepcopy, lambda d: pickle.loads(pickle.dumps(d))], ids=["copy", "deepcopy", "pickle"])
def test_a_copied_description_is_the_one_used(make):
    """Both are refused before anything runs, the original for its number of ids, the edited copy for a negative one."""
    from paper_2408_11500_b200 import binding as B
    b = np.zeros(64, np.float32)
    d = B.make_embed_desc(1 << 31, 7, 4)
    e = make(d)
    e.n = -1
    calls = [lambda x: B.slicegcn_embed_forward(x, b, b, b), lambda x: B.slicegcn_embed_backward(x, b, b, b, None, b, b.nbytes),
             lambda x: B.slicegcn_embed_workspace_bytes(x)]
    for call in calls:
        for desc, status in ((d, B.ERR_OVERFLOW), (e, B.ERR_INVALID_ARG)):
            with pytest.raises(B.SliceGCNError) as err:
                call(desc)
            assert err.value.status == status
    del d
    with pytest.raises(B.SliceGCNError) as err:
        calls[0](e)
    assert err.value.status == B.ERR_INVALID_ARG


def test_a_description_keeps_what_it_points_to():
    from paper_2408_11500_b200 import binding as B
    import weakref

    class Vector:
        data_ptr = staticmethod(lambda: 256)
    v = Vector()
    d, gone = B.make_residual_norm_desc(1, 1, 4, w_pre=v), weakref.ref(v)
    del v
    assert gone() is not None and d.w_pre == 256
