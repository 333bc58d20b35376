"""A cm_rotary_set whose kernels cannot be enqueued leaves an object without positions: calls that need them refuse it."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_positions_that_were_not_enqueued_do_not_count():
    """The stream's capture is made invalid by a synchronization, which a capture does not allow: every launch on it fails until the capture is ended."""
    import torch
    from paper_2602_11470_amd import binding as B
    ctx = B.config1()
    try:
        kv = ctx.kv_create(8, 32, 2, r_i=8)
        rotary = ctx.rotary(8, 32, 3, 16, halves=True)
        sk = ctx.keygen_secret(1)
        keys = ctx.keygen_rotations(sk, kv.steps() + rotary.steps(), 2, with_relin=True)
        x, k, v = (B.Ct(ctx, 3) for _ in range(3))
        for c in (x, k, v):
            c.buf.zero_()
            c.d.scale = ctx.scale
        run = [1, 2, 3] + [-1] * 5
        ctx.rotary_set(rotary, [0] * 8)
        ctx.rotary_apply(keys, rotary, [x])
        torch.cuda.synchronize()
        stream, graph = torch.cuda.Stream(), C.c_void_p()
        handle, p = C.c_void_p(stream.cuda_stream), np.array(run, dtype=np.int32)
        assert B.lib.hipStreamBeginCapture(handle, 2) == 0
        assert B.lib.hipStreamSynchronize(handle) != 0
        assert B.lib.cm_rotary_set(ctx.h, rotary.h, p.ctypes.data, 0, handle) == -7
        B.lib.hipStreamEndCapture(handle, C.byref(graph))
        B.lib.hipGetLastError()
        with pytest.raises(B.CachemirError) as e:
            ctx.rotary_apply(keys, rotary, [x])
        assert e.value.status == -5
        with pytest.raises(B.CachemirError) as e:
            kv.append_run(keys, k, v, 3, rotary=rotary)
        assert e.value.status == -5 and kv.tokens() == 0
        ctx.rotary_set(rotary, run)
        ctx.rotary_apply(keys, rotary, [x])
        kv.append_run(keys, k, v, 3, rotary=rotary)
        assert kv.tokens() == 3
    finally:
        ctx.close()
