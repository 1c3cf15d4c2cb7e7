"""The embedding and its gradient against plain references.

A row of the lookup is one fp32 product and one rounding: it has to be equal.
A sum of n fp32 values is off by at most n 2^-24 times the sum of their
magnitudes, and the product with the scale by half a step more.
"""

import numpy as np
import pytest
import torch

from oracle import layers_oracle as orc
from paper_2608_11519_amd import flarepp as fp

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _ids(kind, T, V, seed=0):
    rng = np.random.default_rng(seed)
    if kind == "one":
        ids = np.full(T, V // 2)
    elif kind == "skewed":
        ids = np.minimum((np.exp(rng.random(T) * np.log(V + 1)) - 1).astype(np.int64), V - 1)
    elif kind == "sorted":
        ids = np.sort(rng.integers(0, V, T))
    else:
        ids = rng.integers(0, V, T)
    if kind == "padded":
        ids[rng.random(T) < 0.3] = -1
        ids[T // 2] = V  # one past the table
    if kind == "empty":
        ids[:] = -5
    return torch.from_numpy(ids.astype(np.int64)).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,C", [(1, 1, 1), (1, 300, 128), (7, 3, 5), (1000, 256, 128), (333, 5000, 130), (50, 9, 2100),
                                   (4097, 77, 64), (90, 30, 289), (70, 30, 11)])
@pytest.mark.parametrize("scale", [1.0, 11.3137])
def test_forward(T, V, C, scale, dtype):
    ids = _ids("padded" if T > 5 else "uniform", T, V)
    table = torch.randn(V, C, device="cuda").to(DT[dtype])
    got = fp.flarepp_embedding_forward(ids, table, scale=scale)
    want = (table.float()[ids.clamp(0, V - 1)] * torch.tensor(scale, dtype=torch.float32, device="cuda")).to(DT[dtype])
    want[ids < 0] = 0
    inside = ids < V
    assert torch.equal(got[inside], want[inside])
    assert torch.isnan(got[~inside].float()).all()


def _backward(ids, d, V, scale, dtype):
    got = fp.flarepp_embedding_backward(ids, d, V=V, scale=scale)
    torch.cuda.synchronize()
    i, x = ids.cpu().numpy(), d.double().cpu().numpy()
    s = float(np.float32(scale))
    ref, size = orc.embedding_backward(i, x, V, s), orc.embedding_backward(i, np.abs(x), V, abs(s))
    count = np.bincount(i[(i >= 0) & (i < V)], minlength=V)[:, None]
    err = np.abs(got.double().cpu().numpy() - ref)
    assert np.all(err <= (count + 2) * 2.0 ** -24 * size), np.max(err - (count + 2) * 2.0 ** -24 * size)
    assert torch.equal(got, fp.flarepp_embedding_backward(ids, d, V=V, scale=scale))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,C", [(1, 1, 1), (2, 1, 3), (5, 700, 16), (63, 9, 128), (64, 9, 128), (65, 9, 128), (129, 2, 8),
                                   (2047, 256, 128), (2049, 1023, 40), (5000, 1024, 9), (3000, 70000, 4), (9000, 31, 520),
                                   (20011, 256, 128), (700, 1 << 21, 1), (2048, 40, 210), (2048, 5, 35),
                                   (300000, 300, 12), (2500, 60, 210), (4000, 17, 7)])
@pytest.mark.parametrize("kind", ["uniform", "padded", "one", "skewed"])
def test_backward(T, V, C, kind, dtype):
    g = torch.Generator().manual_seed(T)
    _backward(_ids(kind, T, V), torch.randn(T, C, generator=g).to(DT[dtype]).cuda(), V, 2.5, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,C", [(210, 5, 65536), (1500, 3000, 1300), (2048, 9, 640), (2048, 9, 644), (2049, 70001, 36)])
def test_backward_of_few_positions_and_many_channels(T, V, C, dtype):
    """Both sides of the bound up to which no sort is done; few positions sorted, a large table cleared."""
    g = torch.Generator().manual_seed(T)
    _backward(_ids("padded", T, V), torch.randn(T, C, generator=g).to(DT[dtype]).cuda(), V, 0.5, dtype)


@pytest.mark.parametrize("kind", ["empty", "sorted"])
@pytest.mark.parametrize("T", [3, 300, 5000])
def test_backward_without_symbols_and_in_order(kind, T):
    _backward(_ids(kind, T, 40), torch.randn(T, 12, device="cuda"), 40, 1.0, "f32")


def test_symbols_of_any_64_bits():
    ids = torch.tensor([0, 1 << 32, -(1 << 63), (1 << 63) - 1, (1 << 32) + 1, 1], dtype=torch.int64, device="cuda")
    table = torch.ones(2, 4, device="cuda")
    out = fp.flarepp_embedding_forward(ids, table)
    assert out[0].eq(1).all() and out[5].eq(1).all() and out[2].eq(0).all() and torch.isnan(out[[1, 3, 4]]).all()
    d = torch.ones(6, 4, device="cuda")
    assert torch.equal(fp.flarepp_embedding_backward(ids, d, V=2), torch.ones(2, 4, device="cuda"))


def test_not_finite_gradients_stay_in_their_rows():
    ids = _ids("uniform", 3000, 50)
    d = torch.randn(3000, 8, device="cuda")
    ref = fp.flarepp_embedding_backward(ids, d, V=50)
    d[1234, 3] = float("nan")
    got = fp.flarepp_embedding_backward(ids, d, V=50)
    row = int(ids[1234])
    assert torch.isnan(got[row, 3])
    got[row, 3] = ref[row, 3]
    assert torch.equal(got, ref)
    pad = ids.clone()
    pad[1234] = -1  # padding is not read into any sum
    assert torch.isfinite(fp.flarepp_embedding_backward(pad, d, V=50)).all()


def test_shapes_graph_and_stream():
    ids = _ids("padded", 6000, 300).view(2, 3, 1000)
    table = torch.randn(300, 64, device="cuda", dtype=torch.bfloat16)
    out = fp.flarepp_embedding_forward(ids, table, scale=2.0)
    assert out.shape == (2, 3, 1000, 64)
    d = torch.randn(2, 3, 1000, 64, device="cuda")
    ref = fp.flarepp_embedding_backward(ids, d, V=300)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = fp.flarepp_embedding_backward(ids, d, V=300)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, ref)
    o, gr = torch.empty_like(out), torch.empty_like(ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fp.flarepp_embedding_forward(ids, table, scale=2.0, out=o)
        fp.flarepp_embedding_backward(ids, d, V=300, out=gr)
    for k in range(3):
        new = ids.roll(k + 1, 2).contiguous()
        ids.copy_(new)
        gr.fill_(float("nan"))
        want = fp.flarepp_embedding_backward(ids, d, V=300)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(gr, want)
        assert torch.equal(o.view(torch.int16), fp.flarepp_embedding_forward(ids, table, scale=2.0).view(torch.int16))


def test_offsets_past_32_bits():
    """A table, a lookup and gradients of more than 2^32 elements."""
    V, T, C = (1 << 22) + 9, (1 << 22) + 3, 1032
    ids = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    ids[:2], ids[-3:] = torch.tensor([V - 1, 5], device="cuda"), torch.tensor([V - 2, V - 1, 0], device="cuda")
    table = torch.zeros(V, C, dtype=torch.bfloat16, device="cuda")
    table[-2:] = torch.randn(2, C, device="cuda").bfloat16()
    table[5], table[0] = 3.0, -2.0
    out = fp.flarepp_embedding_forward(ids, table, scale=2.0)
    for t in (0, 1, 2, T // 2, T - 3, T - 2, T - 1):
        want = table[ids[t]] * 2 if int(ids[t]) >= 0 else torch.zeros_like(table[0])
        assert torch.equal(out[t], want)
    out.zero_()
    out[:2], out[-3:] = torch.randn(2, C, device="cuda").bfloat16(), torch.randn(3, C, device="cuda").bfloat16()
    dT = fp.flarepp_embedding_backward(ids, out, V=V)
    f = [out[i].float() for i in (0, 1, T - 3, T - 2, T - 1)]
    assert torch.equal(dT[V - 1], f[0] + f[3]) and torch.equal(dT[5], f[1]) and torch.equal(dT[V - 2], f[2])
    assert torch.equal(dT[0], f[4]) and not dT[6:V - 2].any() and not dT[1:5].any()
