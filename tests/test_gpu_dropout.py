"""GPU: surgeon_dropout against its definition, the generator made again on the host in 64-bit integers."""
import numpy as np
import pytest
import torch

from paper_2503_20354_b200 import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def bits(n, seed, offset):
    """16 bits for each of n elements, as the header defines them."""
    low = 0xFFFFFFFF
    m = np.uint64(low)
    i = np.arange((n + 7) // 8, dtype=np.uint64)
    c = [i & m, i >> np.uint64(32), np.full_like(i, offset & low), np.full_like(i, offset >> 32 & low)]
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), q & m, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p & m]
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    w = np.stack(c, 1)
    return torch.from_numpy(np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 2).reshape(-1)[:n].astype(np.int64))


def want(x, p, seed, offset, residual):
    t = int(np.floor(p * 65536 + 0.5))
    keep = bits(x.numel(), seed & (1 << 64) - 1, offset & (1 << 64) - 1).view(x.shape) >= t
    scale = np.float32(65536.0 / (65536 - t)) if t < 65536 else np.float32(0)
    y = torch.where(keep, x.float().cpu() * float(scale), torch.zeros(()))             # (a product of fp32 numbers, rounded once)
    if residual is not None:
        y = y + residual.float().cpu()
    return y.to(x.dtype), keep


def test_the_generator_itself():
    """Published answers of the generator for counters and keys of zeros and of ones."""
    words = bits(8, 0, 0)
    assert [int(words[2 * i] + (words[2 * i + 1] << 16)) for i in range(4)] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]


@pytest.mark.parametrize("dt", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 1000, 2049, 4096, 100003])
def test_matches_the_definition(n, dt):
    g = torch.Generator().manual_seed(n)
    x, res = torch.randn(n, generator=g).to(dt).cuda(), torch.randn(n, generator=g).to(dt).cuda()
    for p, seed, offset, r in ((0.1, 1, 0, None), (0.5, (1 << 63) + 5, (1 << 40) + 3, res), (0.0, 2, 1, res), (1.0, 3, 1, res), (0.999, -1, -1, None)):
        pad = torch.full((n + 64,), 7.0, dtype=dt, device="cuda")
        y = B.surgeon_dropout(x, p, seed, offset, residual=r, out=pad[:n])
        expected, _ = want(x, p, seed, offset, r)
        assert torch.equal(y.cpu(), expected) and bool((pad[n:] == 7.0).all())
        assert torch.equal(B.surgeon_dropout(x, p, seed, offset, residual=r), y)
        place = x.clone()
        assert torch.equal(B.surgeon_dropout(place, p, seed, offset, residual=r, out=place), y)
        if r is not None:
            place = r.clone()
            assert torch.equal(B.surgeon_dropout(x, p, seed, offset, residual=place, out=place), y)


def test_the_gradient_drops_the_same_elements():
    x, dy = torch.randn(3, 700, device="cuda").to(BF16), torch.randn(3, 700, device="cuda")
    y, dx = B.surgeon_dropout(x, 0.3, 11, 5), B.surgeon_dropout(dy, 0.3, 11, 5)
    _, keep = want(x, 0.3, 11, 5, None)
    assert torch.equal((y != 0).cpu() & keep, (x != 0).cpu() & keep) and torch.equal((dx != 0).cpu(), keep & (dy != 0).cpu())
    scale = np.float32(65536.0 / (65536 - int(0.3 * 65536 + 0.5)))
    assert torch.equal(dx.cpu(), torch.where(keep, dy.cpu() * float(scale), torch.zeros(())))


def test_a_dropped_nan_is_gone():
    x = torch.full((1000,), float("nan"), device="cuda")
    y = B.surgeon_dropout(x, 0.5, 1)
    _, keep = want(torch.zeros(1000), 0.5, 1, 0, None)
    assert torch.equal(torch.isnan(y).cpu(), keep) and bool((y.cpu()[~keep] == 0).all())
    assert bool((B.surgeon_dropout(x, 1.0, 1) == 0).all())


def test_share_that_is_dropped():
    """n draws: the share is off by at most 6 of its standard deviations, and so is its average of pairs of neighbours."""
    n = 1 << 22
    for p in (0.1, 0.5):
        keep = (B.surgeon_dropout(torch.ones(n, device="cuda"), p, 123, 9) != 0).double()
        t = int(p * 65536 + 0.5) / 65536
        sd = (t * (1 - t) / n) ** 0.5
        assert abs((1 - keep).mean().item() - t) <= 6 * sd
        both = ((1 - keep[::2]) * (1 - keep[1::2])).mean().item()
        assert abs(both - t * t) <= 6 * (t * t * (1 - t * t) / (n / 2)) ** 0.5
        other = (B.surgeon_dropout(torch.ones(n, device="cuda"), p, 123, 10) != 0).double()        # another offset: other bits
        assert abs((keep * other).mean().item() - (1 - t) ** 2) <= 6 * ((1 - t) ** 2 / n) ** 0.5


def test_offset_on_the_device_and_replays():
    x, y = torch.randn(5000, device="cuda"), torch.empty(5000, device="cuda")
    later = torch.zeros(1, dtype=torch.int64, device="cuda")
    B.surgeon_dropout(x, 0.4, 7, 100, out=y, device_offset=later)
    assert torch.equal(y, B.surgeon_dropout(x, 0.4, 7, 100))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.surgeon_dropout(x, 0.4, 7, 100, out=y, device_offset=later)
        later += 1
    for i in range(3):
        later.fill_(i)
        graph.replay()
        assert torch.equal(y, B.surgeon_dropout(x, 0.4, 7, 100 + i)) and later.item() == i + 1


def test_nothing():
    assert B.surgeon_dropout(torch.empty(0, device="cuda"), 0.5, 1).numel() == 0
