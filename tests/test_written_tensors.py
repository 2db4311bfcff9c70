"""Tensors that a call is given to write to: autograd learns of it, so that a product that had kept what stood there refuses its backward pass instead of taking
the new values."""
import pytest

from paper_2012_15667_amd import binding as B

ROWS, COLS = 6, 64


def _tensor(*shape, seed=1):
    import torch
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).cuda()


def _calls():
    h, w = _tensor(ROWS, COLS, seed=2), _tensor(COLS, COLS, seed=3)
    images, kernels = _tensor(1, 3, 8, COLS // 8, seed=4), _tensor(ROWS, 3, 3, 3, seed=5)

    def as_images(x):
        return x.view(1, ROWS, 8, COLS // 8)
    return dict(
        block_norm_stream=lambda x: B.block_norm(x, h, x_out=x),
        block_norm_stream_alone=lambda x: B.block_norm(x, h, pre="none", x_out=x),
        block_norm_norm=lambda x: B.block_norm(h, y=x),
        dropout=lambda x: B.dropout(x, 0.5, 1, y=x),
        dropout_checkpoint=lambda x: B.dropout(h, 0.5, 1, y=x, checkpoint=True),
        dropout_residual=lambda x: B.dropout(h, 0.5, 1, residual=x, y=x),
        dropout_some_rows=lambda x: B.dropout(h[:2], 0.5, 1, y=x[1:3]),
        linear=lambda x: B.linear(h, w, y=x),
        linear_residual=lambda x: B.linear(h, w, residual=x, y=x),
        linear_mx4=lambda x: B.linear_mx4(h, B.mx4_pack(w), residual=x, y=x),
        mx4_unpack=lambda x: B.mx4_unpack(B.mx4_pack(h), y=x),
        checkpoint_unpack=lambda x: B.checkpoint_unpack(B.checkpoint_pack(h), y=x),
        conv_direct=lambda x: B.conv_direct(images, kernels, 1, 1, y=as_images(x)),
        conv_direct_pad2=lambda x: B.conv_direct(images, kernels, 1, (1, 1), y=as_images(x)),
        conv_direct_layout=lambda x: B.conv_direct_layout(images, kernels, 1, 1, layout=B.LAYOUT_CHW, y=as_images(x)),
        conv_direct_noalloc=lambda x: B.conv_direct_noalloc(images, kernels, 1, 1, as_images(x)),
        conv_winograd=lambda x: B.conv_winograd(images, kernels, 2, y=as_images(x)),
        conv_winograd_workspace=lambda x: B.conv_winograd(images, kernels, 2, y=as_images(x), workspace=_workspace()),
        conv_winograd_pad=lambda x: B.conv_winograd(images, _tensor(ROWS, 3, 3, 3), 2, y=x.view(-1)[:ROWS * 6 * 6].view(1, ROWS, 6, 6), pad=0),
        conv_winograd_pre=lambda x: B.conv_winograd_pre(images, B.winograd_transform_kernels(kernels, 2)[0], ROWS, 2, y=as_images(x)))


def _workspace():
    import torch
    return torch.empty(B.winograd_workspace_bytes(1, 3, 8, COLS // 8, ROWS, 2), dtype=torch.uint8, device="cuda")


NAMES = ["block_norm_stream", "block_norm_stream_alone", "block_norm_norm", "dropout", "dropout_checkpoint", "dropout_residual", "dropout_some_rows", "linear", "linear_residual",
         "linear_mx4", "mx4_unpack", "checkpoint_unpack", "conv_direct", "conv_direct_pad2", "conv_direct_layout", "conv_direct_noalloc", "conv_winograd",
         "conv_winograd_workspace", "conv_winograd_pad", "conv_winograd_pre"]


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("recording", [True, False])
def test_what_was_kept_before_is_known_to_be_overwritten(name, recording):
    import torch
    call = _calls()[name]
    x, v = _tensor(ROWS, COLS), _tensor(5, COLS, seed=9).requires_grad_()
    kept = x @ v.T                              # (keeps x for the gradient of v)
    with torch.set_grad_enabled(recording):
        call(x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.sum().backward()
    # what was kept of others is not touched
    (_tensor(ROWS, COLS, seed=11) @ v.T).sum().backward()
    assert v.grad is not None


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_tensors_without_versions_are_written_as_before(name):
    import torch
    want = _tensor(ROWS, COLS)
    _calls()[name](want)
    with torch.inference_mode():
        x = _tensor(ROWS, COLS)
        _calls()[name](x)
        assert torch.equal(x, want)


@pytest.mark.gpu
def test_inputs_are_not_taken_for_written():
    import torch
    x, w = _tensor(ROWS, COLS), _tensor(COLS, COLS, seed=3)
    before = x._version, w._version
    B.linear(x, w, y=torch.empty_like(x))
    B.block_norm(x, w[:ROWS], y=torch.empty_like(x), x_out=torch.empty_like(x))
    B.dropout(x, 0.5, 1, residual=w[:ROWS], y=torch.empty_like(x))
    assert (x._version, w._version) == before
