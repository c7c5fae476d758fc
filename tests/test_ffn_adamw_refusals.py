"""What the feed-forward and AdamW calls refuse, before anything runs (no device needed)."""
import ctypes

import numpy as np
import pytest


def _status(call, *args):
    from paper_2408_11500_b200 import binding as B
    with pytest.raises(B.SliceGCNError) as e:
        call(*args)
    return e.value.status


BUF = np.zeros(8192, np.uint8)
AT = BUF.ctypes.data + (-BUF.ctypes.data) % 256       # an address on 256 bytes


def _ffn(**kw):
    from paper_2408_11500_b200 import binding as B
    args = dict(n=40, num_slices=2, in_s=40, out_s=16, W=AT, act=B.ACT_SILU, dtype=B.BF16)
    args.update(kw)
    return B.make_ffn_desc(**args)


def test_ffn_descriptions():
    from paper_2408_11500_b200 import binding as B
    bad = [(dict(n=-1), B.ERR_INVALID_ARG), (dict(num_slices=0), B.ERR_INVALID_ARG), (dict(in_s=0), B.ERR_INVALID_ARG), (dict(out_s=0), B.ERR_INVALID_ARG),
           (dict(num_slices=65), B.ERR_UNSUPPORTED), (dict(in_s=B.MAX_FFN_WIDTH + 1), B.ERR_UNSUPPORTED), (dict(n=1 << 31), B.ERR_OVERFLOW),
           (dict(act=4), B.ERR_INVALID_ARG), (dict(act=-1), B.ERR_INVALID_ARG), (dict(dtype=2), B.ERR_INVALID_ARG), (dict(grad_dtype=7), B.ERR_INVALID_ARG),
           (dict(dtype=B.F32, grad_dtype=B.BF16), B.ERR_UNSUPPORTED), (dict(scale=float("nan")), B.ERR_INVALID_ARG), (dict(scale=float("inf")), B.ERR_INVALID_ARG),
           (dict(W=None), B.ERR_INVALID_ARG), (dict(W=AT + 1), B.ERR_INVALID_ARG), (dict(W2=AT + 1), B.ERR_INVALID_ARG), (dict(b=AT + 2), B.ERR_INVALID_ARG),
           (dict(b2=AT), B.ERR_INVALID_ARG), (dict(x_ld=79), B.ERR_INVALID_ARG), (dict(dtype=B.F32, W=AT + 2), B.ERR_INVALID_ARG)]
    for kw, want in bad:
        d = _ffn(**kw)
        calls = [lambda: B.slicegcn_ffn_workspace_bytes(d, AT, AT), lambda: B.slicegcn_ffn_forward(d, AT, None, AT, None, AT, 1 << 20),
                 lambda: B.slicegcn_ffn_backward(d, AT, AT, None, None, None, None, None, None, AT, 1 << 20)]
        for call in calls:
            assert _status(call) == want, kw


def test_ffn_matrices():
    from paper_2408_11500_b200 import binding as B
    d = _ffn()
    fwd = lambda **k: B.slicegcn_ffn_forward(d, *[{**dict(x=AT, r=None, out=AT, status=None, ws=AT, n=1 << 20), **k}[s] for s in ("x", "r", "out", "status", "ws", "n")])   # noqa: E731
    for kw in (dict(x=None), dict(out=None), dict(x=AT + 1), dict(r=AT + 1), dict(out=AT + 1), dict(status=AT + 2), dict(ws=AT + 64)):
        assert _status(lambda: fwd(**kw)) == B.ERR_INVALID_ARG, kw
    names = ("x", "dout", "dx", "dW", "dW2", "db", "db2", "status", "ws", "n")
    base = dict(x=AT, dout=AT, dx=AT, dW=AT, dW2=None, db=AT, db2=None, status=None, ws=AT, n=1 << 20)
    bwd = lambda **k: B.slicegcn_ffn_backward(d, *[{**base, **k}[s] for s in names])   # noqa: E731
    for kw in (dict(x=None), dict(dout=None), dict(dout=AT + 1), dict(dx=AT + 1), dict(dW=AT + 1), dict(db=AT + 2), dict(dW2=AT), dict(db2=AT), dict(ws=AT + 64)):
        assert _status(lambda: bwd(**kw)) == B.ERR_INVALID_ARG, kw
    assert _status(lambda: bwd(n=64)) == B.ERR_ALLOC and _status(lambda: bwd(ws=None)) == B.ERR_ALLOC
    d.dout_ld = 31
    assert _status(bwd) == B.ERR_INVALID_ARG
    d.dout_ld, d.out_ld = 32, 31
    assert _status(fwd) == B.ERR_INVALID_ARG
    d.out_ld, d.n, d.in_s, d.out_s, d.x_ld = 1024, 40_000, 400, 512, 801     # rows off 16 bytes are laid out anew and need room for it
    assert _status(lambda: fwd(n=0)) == B.ERR_ALLOC
    assert B.slicegcn_ffn_workspace_bytes(d, AT) >= 2 * 40_000 * 800
    with pytest.raises(B.SliceGCNError):
        B.slicegcn_ffn_workspace_bytes(d, None)


def test_ffn_workspace_follows_what_is_laid_out():
    from paper_2408_11500_b200 import binding as B
    size, large = B.slicegcn_ffn_workspace_bytes, dict(n=40_000, in_s=400, out_s=512)
    assert size(_ffn(**large), AT) == 0
    assert size(_ffn(**large), AT + 2) > 0 and size(_ffn(**{**large, "in_s": 399}, x_ld=800), AT) > 0 and size(_ffn(**large, W=AT + 2), AT) > 0
    assert size(_ffn(**{**large, "out_s": 509}), AT) > 0
    assert size(_ffn(**large, dtype=B.F32), AT) >= 3 * 2 * (40_000 * 800 + 2 * 400 * 512)
    assert size(_ffn(n=0), None) == 0
    assert size(_ffn(n=4, in_s=7, out_s=9, dtype=B.F32), AT + 4) == 0     # a few rows need none, whatever their layout
    assert size(_ffn(dtype=B.F32), AT) == 0                               # nor does little work
    assert size(_ffn(n=4), AT, AT) > 0
    with pytest.raises(TypeError):
        _ffn(y_ld=3)


def _adamw(q8=False, **kw):
    """A description with one tensor of four elements, its arrays at AT, and fields replaced."""
    from paper_2408_11500_b200 import binding as B

    class T:                                             # a tensor on a device, as far as the descriptions look at it
        def __init__(self, t, n=4, at=AT):
            self.dtype, self.n, self.at = "torch." + t, n, at

        def numel(self):
            return self.n

        def is_contiguous(self):
            return True

        def data_ptr(self):
            return self.at
    lists = dict(params=[T("float32")], grads=[T("float32")], m=[T("int8" if q8 else "float32")], v=[T("uint8" if q8 else "float32")])
    if q8:
        lists.update(m_scale=[T("float32", 1)], v_scale=[T("float32", 1)])
    at = kw.pop("at", {})
    for name, address in at.items():
        lists[name][0].at = address
    d = B.make_adamw_desc(**lists, **{k: v for k, v in kw.items() if k in ("lr", "beta1", "beta2", "eps", "weight_decay", "max_norm", "lr_scale")})
    for k, v in kw.items():
        if k not in ("lr", "beta1", "beta2", "eps", "weight_decay", "max_norm", "lr_scale"):
            setattr(d, k, v)
    return d


@pytest.mark.parametrize("q8", [False, True], ids=["f32", "q8"])
def test_adamw_descriptions(q8):
    from paper_2408_11500_b200 import binding as B
    nan, inf = float("nan"), float("inf")
    bad = [(dict(count=-1), B.ERR_INVALID_ARG), (dict(count=513), B.ERR_UNSUPPORTED), (dict(state_dtype=1), B.ERR_INVALID_ARG), (dict(lr=-1.0), B.ERR_INVALID_ARG),
           (dict(lr=nan), B.ERR_INVALID_ARG), (dict(lr=inf), B.ERR_INVALID_ARG), (dict(beta1=1.0), B.ERR_INVALID_ARG), (dict(beta2=-0.1), B.ERR_INVALID_ARG),
           (dict(eps=0.0), B.ERR_INVALID_ARG), (dict(eps=nan), B.ERR_INVALID_ARG), (dict(weight_decay=-1.0), B.ERR_INVALID_ARG), (dict(weight_decay=inf), B.ERR_INVALID_ARG),
           (dict(max_norm=0.0), B.ERR_INVALID_ARG), (dict(max_norm=nan), B.ERR_INVALID_ARG), (dict(lr_scale=AT + 1), B.ERR_INVALID_ARG),
           (dict(at=dict(params=AT + 2)), B.ERR_INVALID_ARG), (dict(at=dict(grads=AT + 2)), B.ERR_INVALID_ARG), (dict(at=dict(params=0)), B.ERR_INVALID_ARG),
           (dict(at=dict(m=0)), B.ERR_INVALID_ARG), (dict(params=None), B.ERR_INVALID_ARG), (dict(elems=None), B.ERR_INVALID_ARG),
           (dict(elems=ctypes.pointer(ctypes.c_int64(-1))), B.ERR_INVALID_ARG), (dict(grad_dtypes=ctypes.pointer(ctypes.c_int32(2))), B.ERR_INVALID_ARG)]
    bad += [(dict(m_scale=None), B.ERR_INVALID_ARG), (dict(at=dict(v_scale=0)), B.ERR_INVALID_ARG)] if q8 else [(dict(at=dict(m=AT + 2)), B.ERR_INVALID_ARG)]
    for kw, want in bad:
        assert _status(B.slicegcn_adamw_step, _adamw(q8, **kw), AT) == want, kw
    for step, norm in ((None, None), (AT + 4, None), (AT, AT + 2)):
        assert _status(B.slicegcn_adamw_step, _adamw(q8), step, norm) == B.ERR_INVALID_ARG


def test_adamw_lists_must_match():
    import torch
    from paper_2408_11500_b200 import binding as B
    t, u = torch.zeros(4), torch.zeros(5)
    for args in (([t], [t], [t], [u]), ([t, t], [t], [t], [t]), ([t], [t], [t.to(torch.int8)], [t]), ([t], [t], [t], [t], [torch.zeros(1)], [torch.zeros(1)]),
                 ([t.to(torch.bfloat16)], [t], [t], [t]), ([torch.zeros(4, 2)[:, 0]], [t], [t], [t])):
        with pytest.raises(ValueError):
            B.make_adamw_desc(*args)
    with pytest.raises(ValueError):
        B.make_adamw_desc([t], [t], [t], [t], copies=[t])
    with pytest.raises(ValueError):
        B.make_adamw_desc([t], [t], [t], [t], decayed=[])
