"""bz_dropout: the mask against the generator in numpy's 64-bit integers, bit for bit; the values exactly."""
import numpy as np
import pytest
import torch

from paper_2010_04902_b200 import binding as bz

pytestmark = pytest.mark.gpu


def philox(counter, key):
    """Ten rounds on arrays of 32-bit words held in uint64."""
    c, k = [np.asarray(w, np.uint64) for w in counter], list(key)
    m = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & m, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(rng, size, rate, first=0):
    """Truth values of elements first .. first + size - 1."""
    seed, offset = (int(r) & (2 ** 64 - 1) for r in rng)
    e = np.arange(first, first + size, dtype=np.uint64)
    g = e >> np.uint64(3)
    one = np.ones_like(g)
    w = philox([g & np.uint64(0xFFFFFFFF), g >> np.uint64(32), one * np.uint64(offset & 0xFFFFFFFF), one * np.uint64(offset >> 32)], (seed & 0xFFFFFFFF, seed >> 32))
    k = (e & np.uint64(7)).astype(np.int64)
    word = np.choose(k >> 1, w)
    bits = np.where(k & 1, word >> np.uint64(16), word & np.uint64(0xFFFF))
    return torch.from_numpy(bits >= round(rate * 65536))


def wanted(x, rng, rate):
    """Exact: one product in binary32, one rounding to the type."""
    scale = torch.tensor(65536.0 / (65536 - round(rate * 65536)), dtype=torch.float32)
    keep = kept(rng.tolist(), x.numel(), rate).view(x.shape)
    return torch.where(keep, x.cpu().float() * scale, torch.zeros(())).to(x.dtype)


def state(seed, offset=5):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def same(a, b):
    kind = torch.int32 if a.dtype == torch.float32 else torch.int16
    return torch.equal(a.cpu().contiguous().view(kind), b.contiguous().view(kind))


def test_generator_gives_the_published_numbers():
    """Known answers of the authors' own tests: counter and key all zeros, all ones, digits of pi."""
    ones = 0xFFFFFFFF
    for counter, key, want in [((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
                               ((ones,) * 4, (ones,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
                               ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))]:
        assert tuple(int(w) for w in philox(counter, key)) == want


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (1, 4096), (3, 5, 17), (33, 515), (64, 2048), (2, 4, 33, 37), (100003,)])
def test_matches(shape, dtype):
    x = torch.randn(shape, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    for rate, seed, offset in ((0.1, 12345, 0), (0.5, -1, -1), (0.0, 1, 2), (65535 / 65536, 2 ** 62 + 11, 2 ** 40 + 3)):
        rng = state(seed, offset)
        assert same(bz.dropout(x, rate, rng), wanted(x, rng, rate))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 3, 8, 13, 64, 515, 520, 2048])
def test_strides(n, dtype):
    """Padded rows, rows off the 16-byte grid, inputs and outputs that sit differently: the same elements by number."""
    rng, rate = state(7), 0.3
    for m, pad, where in ((1, 0, 1), (5, 3, 0), (5, 8, 0), (37, 8, 8), (37, 1, 1)):
        full = torch.randn(m, n + pad + where, device="cuda").to(dtype)
        x = full[:, where:where + n]
        want = wanted(x, rng, rate)
        assert same(bz.dropout(x, rate, rng), want)
        assert same(bz.dropout(x.contiguous(), rate, rng), want)
        out = torch.full((m, n + 5), 7.0, dtype=dtype, device="cuda")
        bz.dropout(x, rate, rng, out=out[:, 2:2 + n])
        assert same(out[:, 2:2 + n], want) and (out[:, :2] == 7).all() and (out[:, 2 + n:] == 7).all()
        got = torch.empty(m, n, dtype=dtype, device="cuda")
        assert same(bz.dropout(x, rate, rng, out=got), want)
        assert same(bz.dropout(x.contiguous(), rate, rng, out=x), want)
        rest = torch.cat([full[:, :where], full[:, where + n:]], 1)
        bz.dropout(x, rate, rng, out=x)          # in place
        assert torch.equal(rest, torch.cat([full[:, :where], full[:, where + n:]], 1))


def test_attention_probabilities():
    """[b][h][tq][tk] with padded rows: rows one distance apart count as a matrix."""
    full = torch.rand(2, 3, 40, 72, device="cuda")
    x = full[..., :65]
    rng = state(3)
    assert same(bz.dropout(x, 0.2, rng), wanted(x, rng, 0.2))
    with pytest.raises(ValueError, match="contiguous"):
        bz.dropout(full[:, :, ::2, :65][:, :2], 0.2, rng)
    with pytest.raises(ValueError, match="contiguous"):
        bz.dropout(torch.rand(5, 1, device="cuda").expand(5, 9), 0.2, rng)


def test_what_is_dropped_becomes_zero_and_nothing_else_does():
    x = torch.full((4096,), float("nan"), device="cuda")
    x[::2] = float("inf")
    rng = state(1)
    got, keep = bz.dropout(x, 0.5, rng), kept(rng.tolist(), 4096, 0.5)
    assert (got.cpu()[~keep] == 0).all() and not (got.cpu()[keep] == 0).any()


def test_elements_beyond_32_bits():
    """2^32 + 4096 binary16 elements: the ends of some rows by number."""
    n = (1 << 23) + 8
    m = 512
    x = torch.ones(m, n, dtype=torch.float16, device="cuda")
    rng = state(99)
    bz.dropout(x, 0.25, rng, out=x)
    for row in (0, 1, m - 1):
        assert torch.equal(x[row, -1000:].cpu() != 0, kept(rng.tolist(), 1000, 0.25, first=row * n + n - 1000))


def test_rate_and_independence():
    """Share of the kept among 2^22 elements: mean 0.75, deviation 2e-4, six of them; masks of neighbouring seeds and offsets agree
    on 0.75^2 + 0.25^2 of the elements."""
    x = torch.ones(1 << 22, device="cuda")
    masks = [bz.dropout(x, 0.25, state(s, o)) != 0 for s, o in ((1, 0), (2, 0), (1, 1))]
    for m in masks:
        assert abs(float(m.float().mean()) - 0.75) < 6 * 2.2e-4
    for a, b in ((0, 1), (0, 2), (1, 2)):
        assert abs(float((masks[a] == masks[b]).float().mean()) - 0.625) < 6 * 2.4e-4


def test_graph_takes_new_numbers_and_streams_do_not_matter():
    x, rng = torch.randn(3000, device="cuda"), state(1)
    graph = torch.cuda.CUDAGraph()
    bz.dropout(x, 0.1, rng)
    with torch.cuda.graph(graph):
        out = bz.dropout(x, 0.1, rng)
    for k in (1, 2):
        rng.copy_(state(k))
        graph.replay()
        assert same(out, wanted(x, rng, 0.1))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = bz.dropout(x, 0.1, rng)
    s.synchronize()
    assert torch.equal(got, out)


def test_gradient_is_the_same_call():
    """out is linear in x: <dout, drop(x)> = <drop(dout), x>, exactly so for small whole numbers and rate 1/2."""
    x, dout = (torch.randint(-8, 8, (999,), device="cuda").float() for _ in range(2))
    rng = state(17)
    assert float((dout * bz.dropout(x, 0.5, rng)).sum()) == float((bz.dropout(dout, 0.5, rng) * x).sum())
    assert bz.dropout(torch.empty(0, device="cuda"), 0.5, rng).numel() == 0 and bz.dropout(torch.empty(3, 0, 4, device="cuda"), 0.5, rng).numel() == 0
