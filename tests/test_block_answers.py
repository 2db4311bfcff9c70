"""Answers of residual blocks in 4 bits are of the weights that the blocks have when they are asked."""
import pytest

pytestmark = pytest.mark.gpu


def _model(seed=0):
    import torch
    from paper_2012_15667_amd.block import Blocks
    model = Blocks(64, 160, 2, torch.float32, "rms", seed=seed)
    x = torch.randn((5, 64), generator=torch.Generator().manual_seed(1)).cuda()
    return model, x


def _from_scratch(model, x):
    """The answer of blocks that have never answered."""
    import torch
    fresh, _ = _model()
    fresh.first.copy_(model.first)
    fresh.blocks = [type(w)(*[t.clone() for t in w]) for w in model.blocks]
    torch.cuda.synchronize()
    return fresh.answer(x, in_4_bits=True)


@pytest.mark.parametrize("which", ["up", "down"])
@pytest.mark.parametrize("how", ["copied", "added", "replaced", "by address"])
def test_after_weights_have_changed(which, how):
    import torch
    from paper_2012_15667_amd import binding as B
    model, x = _model()
    before = model.answer(x, in_4_bits=True)
    old = getattr(model.blocks[1], which)
    new = 0.5 * torch.randn(old.shape, generator=torch.Generator().manual_seed(7)).cuda()
    if how == "copied":
        old.copy_(new)
    elif how == "added":
        old.add_(new)
    elif how == "replaced":
        model.blocks[1] = model.blocks[1]._replace(**{which: new})
    else:
        B.dropout(new, 0.0, 1, y=old.data)      # (autograd does not learn of what is written through .data)
    after = model.answer(x, in_4_bits=True)
    assert not torch.equal(after, before)
    assert torch.equal(after, _from_scratch(model, x))


def test_after_descending():
    import torch
    model, x = _model()
    model.answer(x, in_4_bits=True)
    n, kept = model.forward(x)
    _, dfirst, grads = model.backward(n, x, kept)
    model.descend(dfirst, grads, 0.1)
    assert torch.equal(model.answer(x, in_4_bits=True), _from_scratch(model, x))


def test_weights_packed_once_by_the_caller():
    """Who answers often packs once, and says with which weights to answer."""
    import torch
    model, x = _model()
    four = model.packed()
    want = model.answer(x, in_4_bits=True)
    assert torch.equal(model.answer(x, four), want) and torch.equal(model.answer(x, in_4_bits=four), want)
    model.blocks[0].up.zero_()
    assert torch.equal(model.answer(x, four), want)
    assert not torch.equal(model.answer(x, in_4_bits=True), want)
    for wrong in ([], four[:1], four + four):
        with pytest.raises(ValueError):
            model.answer(x, wrong)
