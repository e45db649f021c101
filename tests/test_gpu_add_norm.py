"""w4a8_add_rmsnorm_quantize_act against the oracle (bit for bit) and against
the separate addition followed by w4a8_rmsnorm_quantize_act.

Every step is one IEEE fp32 operation on both sides, except the sum of
squares, which is fp64 on both: codes, scales and sums have to be equal."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_12932_amd as w
from paper_2608_12932_amd import inputs as I
from helpers import bf16_dev, dev, to_np_bits

pytestmark = pytest.mark.gpu

EPS = 1e-6


def inputs(M, K, seed):
    return I.activations(M, K, 900 + seed), I.activations(M, K, 950 + seed), I.activations(1, K, 980 + seed, outliers=False)[0]


def check(x, r, g, label, eps=EPS):
    print(f"[case] add+rmsnorm {label} {x.shape}", flush=True)
    q, s, t = w.w4a8_add_rmsnorm_quantize_act(bf16_dev(x), bf16_dev(r), bf16_dev(g), eps)
    torch.cuda.synchronize()
    qo, so, to = oracle.add_rmsnorm_quantize(x, r, g, eps)
    np.testing.assert_array_equal(to_np_bits(t), to, err_msg=f"{label}: sum")
    np.testing.assert_array_equal(s.cpu().numpy().view(np.uint32), so.view(np.uint32), err_msg=f"{label}: scales")
    np.testing.assert_array_equal(q.cpu().numpy(), qo, err_msg=f"{label}: codes")


# every number of threads per row and chunks per thread, rows that are read
# again from memory (K above 32768), ragged rows
@pytest.mark.parametrize("M,K", [(1, 128), (3, 128), (1, 4096), (16, 4096), (65, 4096), (301, 4096), (1, 12288), (70, 12288), (5, 640),
                                 (200, 1024), (130, 2048), (100, 8192), (66, 384), (2, 32768), (2, 33024), (2, 65536), (65, 65536),
                                 (2047, 1024), (2048, 1024), (2049, 4096), (2500, 2560)])
def test_bit_exact(M, K):
    check(*inputs(M, K, M + K), f"M={M} K={K}")


def test_special_rows():
    K = 1024
    x, r, g = inputs(6, K, 7)
    r[0] = x[0] ^ 0x8000  # the sum is zero everywhere
    x[1] = 0
    r[1] = 0
    r[1, 5] = 0x3F80  # one nonzero element
    x[2], r[2] = 0x0001, 0x8002  # subnormals
    x[3, ::2] = 0x7F00  # large: 2^127, its square past fp32 but not its mean with the rest at 0
    x[3], r[3] = 0, 0
    x[3, 0] = 0x5F00
    x[4] = r[4]  # doubling is exact
    check(x, r, g, "special rows")
    g[:] = 0
    check(x, r, g, "zero gain")


@pytest.mark.parametrize("which", ["x", "residual"])
@pytest.mark.parametrize("M,K", [(1, 4096), (70, 4096), (2, 65536)])
def test_in_place(M, K, which):
    x, r, g = inputs(M, K, 11)
    want = w.w4a8_add_rmsnorm_quantize_act(bf16_dev(x), bf16_dev(r), bf16_dev(g), EPS)
    xd, rd = bf16_dev(x), bf16_dev(r)
    out = xd if which == "x" else rd
    q, s, t = w.w4a8_add_rmsnorm_quantize_act(xd, rd, bf16_dev(g), EPS, out=out)
    assert t is out
    for a, b in zip((q, s, t), want):
        assert torch.equal(a.view(torch.int8), b.view(torch.int8))
    other = rd if which == "x" else xd  # the other input is as it was
    np.testing.assert_array_equal(to_np_bits(other), r if which == "x" else x)


def test_is_addition_then_norm():
    x, r, g = (bf16_dev(t) for t in inputs(777, 4096, 12))
    q, s, t = w.w4a8_add_rmsnorm_quantize_act(x, r, g, 1e-5)
    assert torch.equal(t, x + r)
    q2, s2 = w.w4a8_rmsnorm_quantize_act(t, g, 1e-5)
    assert torch.equal(q, q2) and torch.equal(s, s2)


def test_same_tensor_twice_and_no_rows():
    x, _, g = (bf16_dev(t) for t in inputs(3, 512, 13))
    q, s, t = w.w4a8_add_rmsnorm_quantize_act(x, x, g, EPS)
    assert torch.equal(t, x + x)
    q, s, t = w.w4a8_add_rmsnorm_quantize_act(x[:0], x[:0], g, EPS)
    assert q.shape == (0, 512) and s.shape == (0,) and t.shape == (0, 512)


def test_side_stream_and_graph():
    x, r, g = (bf16_dev(t) for t in inputs(40, 4096, 14))
    want = w.w4a8_add_rmsnorm_quantize_act(x, r, g, EPS)
    side = torch.cuda.Stream(dev())
    side.wait_stream(torch.cuda.current_stream())
    got = w.w4a8_add_rmsnorm_quantize_act(x, r, g, EPS, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.int8), b.view(torch.int8))
    res = r.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        q, s, t = w.w4a8_add_rmsnorm_quantize_act(x, res, g, EPS, out=res)  # the stream grows by x at each replay
    for rep in range(4):
        before = res.clone()
        graph.replay()
        torch.cuda.synchronize()
        q2, s2, t2 = w.w4a8_add_rmsnorm_quantize_act(x, before, g, EPS)
        assert torch.equal(res, t2) and torch.equal(q, q2) and torch.equal(s, s2), rep


def test_refusals():
    x, r, g = (bf16_dev(t) for t in inputs(4, 256, 15))
    with pytest.raises(ValueError):
        w.w4a8_add_rmsnorm_quantize_act(x, r[:3], g, EPS)
    with pytest.raises(ValueError):
        w.w4a8_add_rmsnorm_quantize_act(x, r, g[:128], EPS)
    with pytest.raises(ValueError):
        w.w4a8_add_rmsnorm_quantize_act(x, r, g, EPS, out=r[:3])
    with pytest.raises(TypeError):
        w.w4a8_add_rmsnorm_quantize_act(x, r.float(), g, EPS)
    with pytest.raises(TypeError):
        w.w4a8_add_rmsnorm_quantize_act(x, r.cpu(), g, EPS)
    big = torch.empty(8, 256, dtype=torch.bfloat16, device=dev())
    with pytest.raises(w.W4A8Error) as e:  # the sum overlaps the input without being it
        w.w4a8_add_rmsnorm_quantize_act(big[:4], r, g, EPS, out=big[1:5])
    assert e.value.status == w.W4A8_EINVAL
    with pytest.raises(w.W4A8Error):
        w.w4a8_add_rmsnorm_quantize_act(x, r, g, 0.0)
