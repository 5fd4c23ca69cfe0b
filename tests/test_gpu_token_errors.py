"""The CUDA runtime's last error and the token losses: what the caller left there is not taken
for a failure of the call, and a call that fails leaves nothing behind for the next check."""
import ctypes as C

import pytest

from gpu_util import context, need_gpu

pytestmark = pytest.mark.gpu


def runtime():
    """The CUDA runtime that this process has loaded."""
    need_gpu()
    with open("/proc/self/maps") as f:
        paths = {line.split()[-1] for line in f if "libcudart.so" in line}
    return [C.CDLL(p) for p in sorted(paths)]


def calls(ctx, torch, V):
    z = torch.zeros((3, V), device="cuda")
    tok, v, g = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, device="cuda"), torch.empty_like(z)
    off, ids, t = torch.tensor([0, 1, 3], device="cuda"), torch.zeros((3, 2), dtype=torch.int32, device="cuda"), z[:, :2].clone()
    return [lambda: ctx.token_logprob(z, tok, v), lambda: ctx.learn_token_ppo(z, tok, v, v, g),
            lambda: ctx.learn_token_pref(z, tok, off, g), lambda: ctx.learn_token_distill(z, ids, t, g)]


def test_an_error_of_the_caller_is_not_the_calls():
    torch = need_gpu()
    with context() as ctx:
        rts = runtime()
        for V in (12, 300, 5000, 40_000):                          # every kernel family
            for f in calls(ctx, torch, V):
                for rt in rts:
                    assert rt.cudaSetDevice(9999) != 0            # a refused argument, kept as the last error
                try:
                    f()
                finally:
                    for rt in rts:
                        rt.cudaGetLastError()
        ctx.sync()


def test_a_refused_launch_leaves_no_error():
    """Work on the legacy stream is refused while a stream that waits for it is captured."""
    torch = need_gpu()
    from paper_2106_07551_gb300 import Context, MalibError
    assert torch.cuda.current_stream().cuda_stream == 0
    with Context(0, 0) as ctx:
        todo = calls(ctx, torch, 40_000)
        for f in todo:
            f()                                                    # work space and modules are there
        ctx.sync()
        torch.cuda.synchronize()
        rts = runtime()
        rt = rts[0]
        stream, graph = C.c_void_p(), C.c_void_p()
        assert rt.cudaStreamCreate(C.byref(stream)) == 0
        assert rt.cudaStreamBeginCapture(stream, 0) == 0
        failed, left = [], []
        for f in todo:
            try:
                f()
            except MalibError as e:
                failed.append(str(e))
            left.append([r.cudaPeekAtLastError() for r in rts])
        rt.cudaStreamEndCapture(stream, C.byref(graph))
        for r in rts:
            r.cudaGetLastError()
        rt.cudaStreamDestroy(stream)
        assert len(failed) == 4 and all("ECUDA" in e for e in failed), failed
        assert not any(any(x) for x in left), left
        for f in todo:
            f()
        ctx.sync()
