"""The product and its gradients with a workspace of exactly the size asked for: the bytes behind it stay as they are, and results
are those of any other workspace; also with dy off the 16-byte boundaries, rows that have to be copied, and split sums."""
import pytest
import torch

import paper_2606_05597_amd as grpo
from paper_2606_05597_amd import _lib
from tests.test_gpu_linear import BF16, F32, tensors

pytestmark = pytest.mark.gpu

GUARD = 1 << 16


@pytest.mark.parametrize("w", ["kn", "nk"])
@pytest.mark.parametrize("M,K,N,act,out,lie", [
    (300, 264, 515, "silu", F32, dict(offset=1)), (300, 264, 515, "none", F32, dict(offset=1)),
    (300, 264, 515, "none", BF16, dict(offset=1)), (5, 8192, 64, "none", BF16, {}), (40, 1000, 1024, "gelu", BF16, dict(ldy=1049)),
    (130, 5000, 131, "none", F32, dict(offset=3)), (2000, 40, 24, "silu", BF16, {}), (4096, 64, 128, "none", F32, dict(offset=1))],
    ids=str)
def test_exact_workspace(M, K, N, act, out, w, lie):
    x, wt, b, res, dy = tensors(M, K, N, w, F32, out, **lie)
    want = grpo.grpo_linear(x, wt, b, res, act=act, out_dtype=out, keep_z=True)
    grads = grpo.grpo_linear_bwd(dy, x, wt, want[1], act=act, dbias=torch.empty_like(b))
    lib = _lib.load()
    for call, name, first in ((lambda ws: grpo.grpo_linear(x, wt, b, res, act=act, out_dtype=out, keep_z=True, workspace=ws),
                               "grpo_linear_workspace_bytes", want),
                              (lambda ws: grpo.grpo_linear_bwd(dy, x, wt, want[1], act=act, dbias=torch.empty_like(b), workspace=ws),
                               "grpo_linear_bwd_workspace_bytes", grads)):
        asked = []

        class Spy:  # notes what the binding asks the library for
            def __getattr__(self, key):
                f = getattr(lib, key)
                if key != name:
                    return f
                return lambda *a: asked.append(f(*a)) or asked[-1]
        load, _lib.load = _lib.load, lambda: Spy()
        try:
            call(None)
        finally:
            _lib.load = load
        buf = torch.full((asked[0] + GUARD,), 0x7f, dtype=torch.uint8, device="cuda")
        got = call(buf[:asked[0]])
        assert all(torch.equal(p, q) for p, q in zip(got, first))
        assert (buf[asked[0]:] == 0x7f).all()
