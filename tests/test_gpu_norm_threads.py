"""Calls from several host threads, each on a stream of its own, whose sizes ask for different amounts of shared memory: what one
call asks for must not be what another is launched with.  Enough calls that threads meet between one's setting and its launch.
"""
import sys
import threading

import pytest


@pytest.mark.gpu
@pytest.mark.parametrize("backward", [False, True], ids=["step", "gradient"])
@pytest.mark.parametrize("sizes", [[(3, 300), (600, 300), (3, 300), (600, 300)], [(2, 9000), (2, 16384), (2, 12000), (2, 16384)]], ids=["staged", "beyond a warp"])
def test_threads_do_not_disturb_each_other(sizes, backward):
    import torch
    from paper_2408_11500_b200 import binding as B
    torch.manual_seed(0)
    failed, error = [], []

    def worker(n, width):
        x = torch.randn((n, width), device="cuda")
        h, dx = torch.empty_like(x), torch.empty_like(x)
        d = B.make_residual_norm_desc(n, 1, width)
        wsb = B.slicegcn_residual_norm_workspace_bytes(d)
        ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
        st = torch.cuda.Stream()
        torch.cuda.synchronize()

        def calls():
            for _ in range(20_000):
                try:
                    if backward:
                        B.slicegcn_residual_norm_backward(d, x, None, None, x, None, dx, None, None, None, None, None, None, ws, wsb, st.cuda_stream)
                    else:
                        B.slicegcn_residual_norm_forward(d, x, x, None, h, None, st.cuda_stream)
                except B.SliceGCNError as e:
                    failed.append(str(e))
            st.synchronize()
            want = x.double() + (0.0 if backward else x.double() / torch.sqrt(x.double().pow(2).mean(1, keepdim=True) + 1e-5))
            error.append(float(((dx if backward else h).double() - want).abs().max()))
        return threading.Thread(target=calls)
    kept = sys.getswitchinterval()
    sys.setswitchinterval(1e-5)
    try:
        threads = [worker(n, width) for n, width in sizes]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(kept)
    assert not failed, (len(failed), failed[0])
    assert len(error) == len(sizes) and max(error) < 1e-4
