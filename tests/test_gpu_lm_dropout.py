"""Dropout without a stored mask (asi_dropout) against the generator in numpy: equal bits."""
import numpy as np
import pytest
import torch
from torch.autograd import forward_ad

import paper_2505_05086_amd as asi
from oracle import asi_oracle as O

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def kept(first, count, p, seed, offset):
    """Which of the elements first .. first + count - 1 dropout keeps."""
    group = np.arange(first // 8, (first + count + 7) // 8, dtype=np.uint64)
    word = lambda v: np.full_like(group, v % 2 ** 32)  # noqa: E731
    w = O.philox4x32_10([group & np.uint64(0xFFFFFFFF), group >> np.uint64(32), word(offset), word((offset % 2 ** 64) >> 32)],
                        (seed % 2 ** 32, (seed % 2 ** 64) >> 32))
    halves = np.stack([np.asarray(x, dtype=np.uint64) for x in w], -1)
    halves = np.stack((halves & np.uint64(0xFFFF), halves >> np.uint64(16)), -1).reshape(-1)
    return halves[first % 8:first % 8 + count] >= round(p * 65536)


def definition(x, p, seed, offset):
    """One product in fp32 and one rounding."""
    keep = torch.from_numpy(kept(0, x.numel(), p, seed, offset)).to(x.device).view(x.shape)
    factor = torch.tensor(65536 / (65536 - round(p * 65536)), dtype=torch.float32, device=x.device)
    return torch.where(keep, x.float() * factor, 0.0).to(x.dtype)


def _x(shape, dtype, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", [(), (1,), (7,), (8,), (9,), (64,), (4095,), (4096,), (4097,), (3, 5), (17, 129), (5, 3, 1001), (2, 40, 512), (300000,)])
def test_dropout(shape, dtype):
    x = _x(shape, DTYPES[dtype])
    for p, seed, offset in ((0.0, 1, 2), (0.1, 123456789012345, 7), (0.5, -5, 2 ** 40 + 3), (0.999, 2 ** 64 - 1, -1)):
        want = definition(x, p, seed, offset)
        assert torch.equal(asi.dropout(x, p, seed, offset), want)
        on_gpu = torch.tensor([seed - 2 ** 64 if seed >= 2 ** 63 else seed], device="cuda")
        assert torch.equal(asi.dropout(x, p, on_gpu, offset), want)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_rows_that_begin_anywhere(dtype):
    for rows, dim, apart, shift in ((9, 33, 40, 0), (9, 33, 41, 3), (700, 1, 9, 1), (50, 1000, 1008, 8), (3, 4999, 5001, 1), (1000, 7, 8, 0)):
        base = _x((rows * apart + shift,), DTYPES[dtype], rows)
        x = base[shift:].as_strided((rows, dim), (apart, 1))
        assert torch.equal(asi.dropout(x, 0.3, 11, 1), definition(x, 0.3, 11, 1))
    flat = _x((5001,), DTYPES[dtype])[1:]                                 # an address that is no multiple of 16
    assert torch.equal(asi.dropout(flat, 0.3, 11), definition(flat, 0.3, 11, 0))
    x = _x((6, 5, 4), DTYPES[dtype]).permute(2, 0, 1)                     # entries that are not next to each other: by their place in x
    assert torch.equal(asi.dropout(x, 0.3, 11), definition(x, 0.3, 11, 0))
    x = _x((1, 40), DTYPES[dtype]).expand(30, 40)
    assert torch.equal(asi.dropout(x, 0.3, 11), definition(x, 0.3, 11, 0))
    assert asi.dropout(_x((0, 5), DTYPES[dtype]), 0.3, 11).shape == (0, 5)


def test_elements_past_32_bits():
    n = 2 ** 32 + 4099
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    y = asi.dropout(x, 0.5, 99, 3)
    for first in (0, 2 ** 31 - 8, 2 ** 32 - 2048, n - 4000):
        part = y[first:first + 4000].float().cpu().numpy()
        assert np.array_equal(part, np.where(kept(first, len(part), 0.5, 99, 3), 2.0, 0.0))
    rows = x[:2 ** 32 - 1024].view(2 ** 22 - 1, 1024)[:, :1000]           # 4.19e9 elements in rows apart from each other
    y = asi.dropout(rows, 0.5, 99, 3)
    first = (rows.shape[0] - 3) * 1000
    assert np.array_equal(y[-3:].float().cpu().numpy().reshape(-1), np.where(kept(first, 3000, 0.5, 99, 3), 2.0, 0.0))


def test_what_is_dropped_may_hold_anything():
    x = torch.full((4096,), float("nan"), device="cuda")
    keep = torch.from_numpy(kept(0, 4096, 0.4, 21, 0)).cuda()
    x[keep] = 3.0
    y = asi.dropout(x, 0.4, 21)
    assert torch.isfinite(y).all() and not y[~keep].any()
    x[keep] = float("inf")
    assert torch.equal(torch.isinf(asi.dropout(x, 0.4, 21)), keep)


def test_shares_and_independence():
    """Shares of a binomial count, each within 6 of its standard deviations; two offsets agree as often as independent ones do."""
    n = 1 << 20
    one = torch.ones(n, device="cuda")
    for p in (0.05, 0.1, 0.5, 0.9):
        a, b = asi.dropout(one, p, 5, 0) > 0, asi.dropout(one, p, 5, 1) > 0
        for share, q in ((a.double().mean(), 1 - p), (b.double().mean(), 1 - p), ((a & b).double().mean(), (1 - p) ** 2)):
            assert abs(float(share) - q) < 6 * (q * (1 - q) / n) ** 0.5 + 2.0 ** -16
        mean = asi.dropout(one, p, 5, 0).double().mean()
        assert abs(float(mean) - 1) < 6 * (p / (1 - p) / n) ** 0.5


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_gradient(dtype):
    x = _x((33, 65), DTYPES[dtype]).requires_grad_()
    seed = torch.tensor([77], device="cuda")
    grad = _x((33, 65), DTYPES[dtype], 3)
    y = asi.dropout(x, 0.2, seed, 4)
    y.backward(grad)
    assert torch.equal(y.detach(), definition(x.detach(), 0.2, 77, 4)) and torch.equal(x.grad, definition(grad, 0.2, 77, 4))
    x.grad = None
    asi.dropout(x, 0.2, 77, 4).sum().backward()                           # the gradient of a sum: one value spread over all
    assert torch.equal(x.grad, definition(torch.ones_like(grad), 0.2, 77, 4))
    y = asi.dropout(x, 0.2, seed, 4)
    seed += 1                                                             # other numbers than the forward pass had
    with pytest.raises(RuntimeError):
        y.backward(grad)
    # linear in x: differences are exact where the steps are
    d = torch.ones_like(grad)
    up = asi.dropout(torch.zeros_like(grad) + d, 0.5, 9).float() - asi.dropout(torch.zeros_like(grad), 0.5, 9).float()
    assert torch.equal(up, definition(d, 0.5, 9, 0).float())


def test_a_graph_takes_the_numbers_of_each_replay():
    x, seed = _x((1000, 257), torch.bfloat16), torch.zeros(1, dtype=torch.int64, device="cuda")
    asi.dropout(x, 0.1, seed, 1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = asi.dropout(x, 0.1, seed, 1)
        z = asi.dropout(x, 0.1, seed, 2)
        seed.add_(1)
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, definition(x, 0.1, step, 1)) and torch.equal(z, asi.dropout(x, 0.1, step, 2))


def test_another_stream():
    x = _x((100, 100), torch.float32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = asi.dropout(x, 0.1, 3)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, definition(x, 0.1, 3, 0))


def test_refusals():
    x = _x((4, 4), torch.float32)
    for p in (-0.1, 1.0, 1.5, float("nan"), 0.999999):
        with pytest.raises(ValueError):
            asi.dropout(x, p, 1)
    for seed in (None, 2 ** 64, -2 ** 63 - 1, torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64)):
        with pytest.raises(ValueError):
            asi.dropout(x, 0.1, seed)
    with pytest.raises(ValueError):
        asi.dropout(x.cpu(), 0.1, 1)
    with pytest.raises(ValueError):
        asi.dropout(x, 0.1, 1, 2 ** 63)
    for bad in (lambda: asi.dropout(x.half(), 0.1, 1), lambda: asi.dropout(x, 0.1, 1.5)):
        with pytest.raises(TypeError):
            bad()
    with forward_ad.dual_level(), pytest.raises(NotImplementedError):
        asi.dropout(forward_ad.make_dual(x, x), 0.1, 1)
