"""Limits of the layer calls (no GPU): what one launch cannot hold is refused before anything is enqueued."""
import pytest

from tests.test_layers_host import BAD, F32, OK, Context, call, rp, shim  # noqa: F401 (shim is a fixture)


@pytest.mark.parametrize("width,status", [(2048, OK), (2049, OK), (8192, OK), (8193, BAD), (16_384, BAD)])
def test_norm_of_the_most_rows(shim, width, status):  # noqa: F811
    """2^27 rows, 16 to a workgroup: 2^23 workgroups of 512 threads above 8192 columns, which no launch holds."""
    ctx = Context(shim)
    shim.shim_launches()
    got = call(ctx, "gasloc_layer_norm", ptr=rp(1 << 27, 0, 0, 0), act=F32, width=width, bias=width, x_ld=width,
               out_ld=width)
    assert got == status, shim.shim_error()
    assert shim.shim_launches() == (status == OK)
    if status == BAD:
        assert b"one launch" in shim.shim_error()


@pytest.mark.parametrize("n,accumulate,status", [(63, 0, OK), (64, 0, BAD), (64, 1, OK)])
def test_table_gradient_of_the_most_columns(shim, n, accumulate, status):  # noqa: F811
    """Zeroing 64 tables of 2^20 x 2047 takes 2^24 workgroups of 256 threads, and adding to them none."""
    ctx = Context(shim, n=n, P=(1 << 31) - 1)
    shim.shim_launches()
    got = call(ctx, "gasloc_embedding_grad", ptr=rp(5, *[0] * (n - 1)), vocab=1 << 20, width=2047, dout_ld=2047,
               grad_ld=1 << 31, accumulate=accumulate)
    assert got == status, shim.shim_error()
    assert (shim.shim_launches() > 0) == (status == OK)
    if status == BAD:
        assert b"one launch" in shim.shim_error()
