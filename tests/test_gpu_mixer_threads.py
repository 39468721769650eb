"""Calls of several host threads at once through the C interface, each on a stream of its own, of head sizes that share a kernel."""
import ctypes
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def at_once(entry, calls):
    """Each call again and again by a thread of its own; the statuses that were not 0."""
    wrong, start = [], threading.Barrier(len(calls))

    def work(i):
        start.wait(30)
        for _ in range(4000):
            status = entry(*calls[i])
            if status != 0:
                wrong.append((i, status))
                return

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return wrong


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("form", ["prompt", "token"])
def test_latent_attention_of_several_head_sizes(form, dtype):
    """The kernels on the CUDA cores take shared memory by head size, up to 100 KB: what one thread's call needs is not another's to take away."""
    import paper_2609_32114_b200 as ha

    lib, keep, calls = ha.load_library(), [], []
    n = lambda *s: torch.randn(*s, device="cuda").to(dtype)  # noqa: E731
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")            # noqa: E731
    for key, rope, value in ((256, 128, 256), (16, 8, 16), (200, 64, 100), (33, 5, 65)):
        if form == "prompt":
            t = dict(q=n(1, 9, 2, key + rope), kn=n(1, 9, 2, key), kr=n(1, 9, rope), v=n(1, 9, 2, value), o=n(1, 9, 2, value))
            args = ha.ha_la_latent_prefill_args(dtype=int(dtype == torch.float32), batch=1, seqlen=9, seqlen_k=9, num_heads=2, d_nope=key, d_rope=rope, d_v=value, scale=0.1)
        else:
            key = 2 * key if key > 33 else key               # up to 512 + 128
            t = dict(q=n(1, 1, 9, key + rope), cache=n(2, 8, key + rope), page_table=i([[1, 0]]), lengths=i([13]), o=n(1, 1, 9, key), workspace=torch.empty(512, dtype=torch.uint8, device="cuda"))
            args = ha.ha_la_latent_decode_args(dtype=int(dtype == torch.float32), num_seqs=1, new_tokens=1, num_heads=9, d_latent=key, d_rope=rope, page_size=8, num_pages=2, max_pages=2, scale=0.1,
                                               workspace_bytes=512)
        for name, x in t.items():
            setattr(args, name, x.data_ptr())
        stream = torch.cuda.Stream()
        keep.append((t, args, stream))
        calls.append((ctypes.byref(args), ctypes.c_void_p(stream.cuda_stream)))
    entry = lib.ha_la_latent_prefill if form == "prompt" else lib.ha_la_latent_decode
    path = ha.ha_la_latent_prefill_path if form == "prompt" else ha.ha_la_latent_decode_path
    assert [path(args) for _, args, _ in keep] == ["simt"] * 4
    torch.cuda.synchronize()
    assert [entry(*c) for c in calls] == [0] * 4
    torch.cuda.synchronize()
    want = [t["o"].clone() for t, _, _ in keep]
    assert at_once(entry, calls) == []
    assert all(torch.equal(t["o"], w) for (t, _, _), w in zip(keep, want))
