"""What the gradients of the product ask for as workspace (CPU only): dz, the bias's partial sums and the larger of the two
products' parts, whatever dy's address where dz is formed anew."""
import ctypes

import pytest

from paper_2606_05597_amd import _lib
from tests.test_linear_abi import an_op, grads, lib  # noqa: F401  (lib: the fixture)


def need(lib, op, g, dy, lddy, dtype):  # noqa: F811
    return lib.grpo_linear_bwd_workspace_bytes(ctypes.byref(op), dy, lddy, dtype, ctypes.byref(g))


@pytest.mark.parametrize("M,K,N", [(2048, 3584, 151936), (300, 264, 515), (40, 1000, 1024), (5, 64, 1000)])
@pytest.mark.parametrize("act,dtype", [(0, _lib.GRPO_F32), (4, _lib.GRPO_F32), (4, _lib.GRPO_BF16)])
@pytest.mark.parametrize("out_in", [0, 1])
def test_the_address_of_dy_does_not_count_where_dz_is_formed(lib, M, K, N, act, dtype, out_in):  # noqa: F811
    op = an_op(M=M, K=K, N=N, ldx=K, ldw=K if out_in else N, w_out_in=out_in, act=act)
    sizes = {need(lib, op, grads(), 0x9000000 + off, N, dtype) for off in (0, 4, 8, 12)}
    assert len(sizes) == 1 and sizes.pop() >= 2 * M * N


@pytest.mark.parametrize("M,K,N", [(2048, 3584, 151936), (300, 264, 515), (4001, 3584, 3584), (5, 64, 1000)])
@pytest.mark.parametrize("act", [0, 2])
@pytest.mark.parametrize("out_in", [0, 1])
def test_the_two_products_share_a_place(lib, M, K, N, act, out_in):  # noqa: F811
    op = an_op(M=M, K=K, N=N, ldx=K, ldw=K if out_in else N, w_out_in=out_in, act=act)
    of = lambda **kw: need(lib, op, grads(dbias=None, **kw), 0x9000000, N, _lib.GRPO_BF16)  # noqa: E731
    assert of() == max(of(dx=None), of(dw=None))
