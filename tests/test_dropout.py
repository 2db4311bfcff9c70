"""Dropout from a counter-based generator: the mask bit by bit, the values to a rounding, the checkpoint as checkpoint_pack gives it."""
import ctypes

import numpy as np
import pytest

from paper_2012_15667_amd import binding as B
from tests.test_dense import HALF_ULP, TINY, TYPES, assert_within, make, to64


def _torch():
    import torch
    return torch


def philox(low, high, seed):
    """Philox4x32 with ten rounds for an array of lower counter words, in Python's whole numbers."""
    out = np.zeros((len(low), 4), dtype=np.uint32)
    M = 0xffffffff
    for i, at in enumerate(low):
        c = [at & M, at >> 32, high & M, high >> 32]
        k = [seed & M, seed >> 32]
        for _ in range(10):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(b >> 32) ^ c[1] ^ k[0], b & M, (a >> 32) ^ c[3] ^ k[1], a & M]
            k = [(k[0] + 0x9E3779B9) & M, (k[1] + 0xBB67AE85) & M]
        out[i] = c
    return out


def mask64(rows, cols, p, seed, offset, first_row=0):
    per = -(-cols // 8)
    words = philox([(first_row + r) * per + j for r in range(rows) for j in range(per)], offset, seed)
    halves = np.stack([words & 0xffff, words >> 16], 2).reshape(rows, per * 8)[:, :cols]
    t = round(p * 65536)
    if p < 1:
        t = min(t, 65535)
    return halves >= t, 65536 / (65536 - t) if t < 65536 else 0.0


def test_the_generator_gives_the_published_words():
    """Known answers that its authors published with the generator: counters and keys of zeros and of ones."""
    assert [hex(w) for w in philox([0], 0, 0)[0]] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
    ones = 2 ** 64 - 1
    assert [hex(w) for w in philox([ones], ones, ones)[0]] == ["0x408f276d", "0x41c83b0e", "0xa20bc7c6", "0x6d5451fd"]


def check(rng, rows, cols, dtype, p, seed, offset, residual=False, gap=0, lead=0, counter=None):
    torch = _torch()

    def wide():
        return make(rng, (rows, cols + gap + lead), dtype)[0][:, lead:lead + cols]
    x, r = wide(), wide() if residual else None
    extra = counter or (0, 0)
    keep, scale = mask64(rows, cols, p, (seed + extra[0]) % 2 ** 64, (offset + extra[1]) % 2 ** 64)
    device = torch.from_numpy(np.array(counter, dtype=np.uint64).view(np.int64)).cuda() if counter else None
    got, c = B.dropout(x, p, seed, offset, counter=device, residual=r, checkpoint=True)
    want = np.where(keep, to64(x) * scale, 0.0)
    off = 2.0 ** -23 * np.abs(want)                 # the scale's rounding and the product's
    if residual:
        want = want + to64(r)
        off = off + 2.0 ** -24 * (np.abs(want) + off)
    assert_within(got, want, off + HALF_ULP[dtype] * (np.abs(want) + off) + TINY[dtype])
    if not residual:
        assert np.array_equal(to64(got) != 0, keep & (to64(x) != 0))
    packed = B.checkpoint_pack(got)
    assert torch.equal(c.q, packed.q) and torch.equal(c.e, packed.e)
    assert torch.equal(B.dropout(x, p, seed, offset, counter=device, residual=r), got)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (5, 33), (40, 100), (2, 2049), (300, 16), (1, 4096)])
@pytest.mark.parametrize("residual", [False, True])
def test_sizes(dtype, rows, cols, residual):
    check(np.random.default_rng(cols), rows, cols, dtype, 0.3, 12345678901234567890, 7, residual)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gap,lead", [(8, 0), (3, 0), (5, 1), (7, 9)])
@pytest.mark.parametrize("rows,cols", [(3, 40), (20, 301)])
def test_strides_and_alignment(dtype, gap, lead, rows, cols):
    check(np.random.default_rng(gap), rows, cols, dtype, 0.5, 99, 2 ** 64 - 1, True, gap, lead)


@pytest.mark.gpu
@pytest.mark.parametrize("p", [0.0, 1e-6, 2.0 ** -17, 0.1, 0.999, 1 - 2.0 ** -18, 1.0])
def test_probabilities(p):
    check(np.random.default_rng(1), 30, 200, "float32", p, 5, 6)


@pytest.mark.gpu
@pytest.mark.parametrize("seed,offset,counter", [(0, 0, None), (2 ** 64 - 1, 2 ** 64 - 1, None), (1, 2, (3, 4)), (2 ** 64 - 1, 2 ** 63, (1, 2 ** 63)), (0, 0, (2 ** 64 - 1, 5))])
def test_seeds_offsets_and_counters_on_the_device(seed, offset, counter):
    check(np.random.default_rng(1), 9, 70, "bfloat16", 0.4, seed, offset, counter=counter)


@pytest.mark.gpu
def test_share_of_dropped_values_and_masks_of_other_offsets():
    """2^22 values at p = 0.25: the share's standard deviation is sqrt(0.1875 / 2^22) = 2.1e-4, six of them 1.3e-3; two masks agree on
    0.0625 + 0.5625 of the values to the same width (2.4e-4 each)."""
    torch = _torch()
    x = torch.ones((1024, 4096), device="cuda")
    masks = [B.dropout(x, 0.25, s, o) != 0 for s, o in ((1, 0), (1, 1), (2, 0))]
    for m in masks:
        assert abs(float((~m).float().mean()) - 0.25) < 1.3e-3
        assert float((~m).float().mean(0).max()) < 0.25 + 6 * (0.1875 / 1024) ** 0.5
    for a, b in ((0, 1), (0, 2), (1, 2)):
        assert abs(float((masks[a] == masks[b]).float().mean()) - 0.625) < 1.5e-3


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_backward_is_the_same_call_and_dropped_values_are_not_looked_at(dtype):
    torch = _torch()
    rng = np.random.default_rng(3)
    x, dy = make(rng, (50, 77), dtype)[0], make(rng, (50, 77), dtype)[0]
    x = torch.where(x == 0, torch.ones_like(x), x)
    keep = B.dropout(x, 0.5, 11, 3) != 0
    dx = B.dropout(dy, 0.5, 11, 3)
    assert torch.equal(dx, torch.where(keep, 2 * dy, torch.zeros_like(dy)))
    for bad in (float("nan"), float("inf")):
        t = torch.where(keep, x, torch.full_like(x, bad))
        assert torch.equal(B.dropout(t, 0.5, 11, 3), B.dropout(x, 0.5, 11, 3))
        t = torch.where(keep, torch.full_like(x, bad), x)
        got = B.dropout(t, 0.5, 11, 3)
        assert bool((got[~keep] == 0).all()) and not bool(torch.isfinite(got[keep]).any())


@pytest.mark.gpu
def test_gradients_against_differences():
    """The call is linear in x: a difference with step 1 is its slope to the rounding of values of order 1 in 32 bits."""
    torch = _torch()
    rng = np.random.default_rng(4)
    x, dy = make(rng, (6, 40), "float32")[0], make(rng, (6, 40), "float32")[0]
    dx = to64(B.dropout(dy, 0.3, 8, 9))
    base = to64(B.dropout(x, 0.3, 8, 9))
    for i in rng.integers(0, 240, 12):
        t = x.clone()
        t.view(-1)[int(i)] += 1
        slope = ((to64(B.dropout(t, 0.3, 8, 9)) - base) * to64(dy)).sum()
        assert abs(slope - dx.flat[i]) <= 2.0 ** -20 * (np.abs(dx).max() + 1)
    del torch


@pytest.mark.gpu
def test_in_place_and_into_wider_rows():
    torch = _torch()
    rng = np.random.default_rng(5)
    x, r = make(rng, (33, 50), "bfloat16")[0], make(rng, (33, 50), "bfloat16")[0]
    want = B.dropout(x, 0.2, 1, 2, residual=r)
    wide = torch.full((33, 70), 7.0, dtype=torch.bfloat16, device="cuda")
    B.dropout(x, 0.2, 1, 2, residual=r, y=wide[:, 9:59])
    assert torch.equal(wide[:, 9:59], want) and bool((wide[:, :9] == 7).all()) and bool((wide[:, 59:] == 7).all())
    a, b = x.clone(), r.clone()
    assert B.dropout(a, 0.2, 1, 2, residual=r, y=a) is a and torch.equal(a, want)
    assert B.dropout(x, 0.2, 1, 2, residual=b, y=b) is b and torch.equal(b, want)


@pytest.mark.gpu
def test_replays_of_a_graph_take_their_masks_from_the_counter():
    torch = _torch()
    x = torch.ones((70, 300), dtype=torch.bfloat16, device="cuda")
    counter = torch.zeros(2, dtype=torch.int64, device="cuda")
    one = torch.tensor([0, 1], device="cuda")
    B.dropout(x, 0.5, 17, 40, counter=counter)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, c = B.dropout(x, 0.5, 17, 40, counter=counter, checkpoint=True)
        counter.add_(one)
    seen = []
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = B.dropout(x, 0.5, 17, 40 + step)
        assert torch.equal(y, want) and torch.equal(B.checkpoint_unpack(c, torch.bfloat16), want)
        seen.append(y.clone())
    assert not any(torch.equal(seen[0], t) for t in seen[1:])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = B.dropout(x, 0.5, 17, 41)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(other, seen[1])


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """Rows 2^21 values apart: the last ones start beyond 2^31 values; and 70000 rows, more than a grid's second axis has workgroups for one by one."""
    torch = _torch()
    rng = np.random.default_rng(6)
    rows, gap = 1100, 1 << 21
    big = torch.empty(rows * gap, dtype=torch.bfloat16, device="cuda").view(rows, gap)
    x = make(rng, (rows, 64), "bfloat16")[0]
    big[:, 128:192].copy_(x)
    B.dropout(big[:, 128:192], 0.3, 4, 5, y=big[:, 256:320])
    assert torch.equal(big[:, 256:320], B.dropout(x, 0.3, 4, 5))
    rows = 70000
    y = B.dropout(torch.ones((rows, 2100), device="cuda"), 0.5, 4, 5)
    for r in (0, 65534, 65535, 65536, rows - 1):
        assert np.array_equal(to64(y[r:r + 1]) != 0, mask64(1, 2100, 0.5, 4, 5, r)[0])


@pytest.mark.gpu
def test_tensors_larger_than_the_caches():
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x, r = (torch.randn((9001, 8200), generator=g, device="cuda").bfloat16() for _ in range(2))
    y, c = B.dropout(x, 0.5, 4, 5, residual=r, checkpoint=True)
    plain = B.dropout(x, 0.5, 4, 5)
    packed = B.checkpoint_pack(y)
    assert torch.equal(c.q, packed.q) and torch.equal(c.e, packed.e)
    for at in (0, 4500, 9000):
        keep = torch.from_numpy(mask64(1, 8200, 0.5, 4, 5, at)[0]).cuda()
        want = torch.where(keep, 2 * x[at:at + 1], torch.zeros_like(x[:1]))
        assert torch.equal(plain[at:at + 1], want) and torch.equal(y[at:at + 1], want + r[at:at + 1])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(0, 5), (5, 0), (0, 0)])
def test_empty(rows, cols):
    y, c = B.dropout(_torch().empty((rows, cols), device="cuda"), 0.5, 1, checkpoint=True)
    assert y.shape == (rows, cols) and c.q.shape == (rows, cols)


@pytest.mark.gpu
def test_a_backward_pass_through_the_result_is_refused():
    torch = _torch()
    x = torch.ones((4, 8), device="cuda", requires_grad=True)
    for kind in (False, True):
        y = B.dropout(x, 0.5, 1, checkpoint=kind)
        y = y[0] if kind else y
        with pytest.raises(RuntimeError, match="dropout"):
            y.sum().backward()
    with torch.no_grad():
        assert not B.dropout(x, 0.5, 1).requires_grad
    with pytest.raises(RuntimeError):
        B.dropout(x, 0.5, 1, y=x)


# ---- refusals ---------------------------------------------------------------------------------------------

P = 4096


@pytest.mark.parametrize("change,code", [
    (dict(rows=-1), -1), (dict(cols=-1), -1), (dict(rows=1 << 31), -2), (dict(cols=1 << 31), -2), (dict(dtype=3), -2), (dict(p=-0.1), -1), (dict(p=1.1), -1),
    (dict(p=float("nan")), -1), (dict(x=None), -1), (dict(y=None), -1), (dict(zq=P), -1), (dict(ze=P), -1), (dict(ldx=7), -1), (dict(ldy=7), -1),
    (dict(residual=P, ldr=7), -1), (dict(x=P + 2), -1), (dict(y=P + 1), -1), (dict(counter=P + 4), -1)])
def test_c_call_refuses_without_touching_the_gpu(change, code):
    a = dict(rows=4, cols=8, dtype=0, p=0.5, seed=1, offset=2, counter=None, x=P, residual=None, y=P, ldx=8, ldr=8, ldy=8, zq=None, ze=None)
    a.update(change)
    assert B.lib().iolb_dropout(ctypes.byref(B.DropoutArgs(*[a[n] for n, _ in B.DropoutArgs._fields_]))) == code
    assert B.lib().iolb_dropout(None) == -1


@pytest.mark.gpu
def test_python_refusals():
    torch = _torch()
    x = torch.zeros((4, 8), device="cuda")
    for error, call in (
            (ValueError, lambda: B.dropout(x, 1.5, 1)), (ValueError, lambda: B.dropout(x, float("nan"), 1)), (ValueError, lambda: B.dropout(x, 0.5, -1)),
            (ValueError, lambda: B.dropout(x, 0.5, 2 ** 64)), (TypeError, lambda: B.dropout(x, 0.5, 1.5)), (TypeError, lambda: B.dropout(x, 0.5, 1, offset="2")),
            (TypeError, lambda: B.dropout(x, 0.5, 1, counter=torch.zeros(2, device="cuda"))), (ValueError, lambda: B.dropout(x, 0.5, 1, counter=torch.zeros(3, dtype=torch.int64, device="cuda"))),
            (TypeError, lambda: B.dropout(x, 0.5, 1, counter=torch.zeros(2, dtype=torch.int64))), (ValueError, lambda: B.dropout(x, 0.5, 1, residual=x[:2])),
            (TypeError, lambda: B.dropout(x.cpu(), 0.5, 1)), (TypeError, lambda: B.dropout(x.double(), 0.5, 1)), (ValueError, lambda: B.dropout(x, 0.5, 1, y=x[:2]))):
        with pytest.raises(error):
            call()
