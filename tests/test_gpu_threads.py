"""Calls of several host threads at once through the C interface: each on a stream of its own, of widths that share a kernel."""
import ctypes
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16,widths", [(True, (1024, 2048, 1536, 1280)), (False, (516, 1024, 700, 900)), (True, (2504, 4096, 3200, 2800))],
                         ids=["bf16", "fp32", "bf16_wide"])
def test_norms_of_several_widths(bf16, widths):
    """The gradients' kernels keep rows in shared memory, more for wider rows: what one thread's call needs is not another's to take away."""
    import paper_2609_32114_b200 as ha

    lib, dtype, keep, calls, streams = ha.load_library(), torch.bfloat16 if bf16 else torch.float32, [], [], []
    for cols in widths:
        t = {n: torch.randn(6, cols, device="cuda").to(dtype) for n in ("x", "r_out", "dy", "dx", "dr")}
        t.update({n: torch.ones(cols, device="cuda") for n in ("w", "w_post", "dw", "dw_post")})
        args = ha.ha_la_add_norm_args(dtype=0 if bf16 else 1, cols=cols, rows=6, scale=1.0, eps=1e-6, **{n: x.data_ptr() for n, x in t.items()})
        ws = torch.empty(ha.ha_la_add_norm_workspace_bytes(args), dtype=torch.uint8, device="cuda")
        args.workspace, args.workspace_bytes = ws.data_ptr(), ws.numel()
        streams.append(torch.cuda.Stream())
        calls.append((ctypes.byref(args), ctypes.c_void_p(streams[-1].cuda_stream)))
        keep.append((t, ws, args))
    torch.cuda.synchronize()
    assert [lib.ha_la_add_norm_backward(*c) for c in calls] == [0] * len(calls)
    torch.cuda.synchronize()
    want = [{n: t[n].clone() for n in ("dx", "dr", "dw", "dw_post")} for t, _, _ in keep]
    wrong, start = [], threading.Barrier(len(calls))

    def work(i):
        start.wait(30)
        for _ in range(4000):
            status = lib.ha_la_add_norm_backward(*calls[i])
            if status != 0:
                wrong.append((widths[i], status))
                return

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong
    assert all(torch.equal(t[n], x[n]) for (t, _, _), x in zip(keep, want) for n in x)
