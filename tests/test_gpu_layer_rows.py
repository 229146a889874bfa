"""Residual norm and gated activation to int8 codes (include/qqq_layer.h) against the definitions in 64 bits.

Tolerances.  The sum of two fp16 values is exact in fp32 wherever its rounding to fp16 could depend on it, so sums are compared bit
for bit.  The sum of squares goes through chains of at most 8 * 16 fused additions and 22 more, so rho is within (150 / 2 + 6) * 2^-24 < 1e-5
of its value.  A code is the nearest integer to a quotient that is within 127 * 1e-5 of the exact one (norm: 127 * 2^-22, since its
codes do not depend on rho), so |code - quotient| <= 1/2 + that; the exponential, its argument's rounding (|argument| <= 60 where
the result counts) and the reciprocal keep the gated product within 1e-5.
"""
import numpy as np
import pytest
import torch

from oracle import qqq_layer_oracle as ref
from paper_2406_09904_amd import binding as qqq

pytestmark = pytest.mark.gpu

REL = 1e-5


def _rows(rng, M, K, scale=1.0):
    x = rng.standard_normal((M, K)) * np.where(rng.random(K) < 0.02, 20.0, 1.0) * scale
    return x.astype(np.float16)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _padded(a, pad):
    """The same values in rows of a wider tensor."""
    wide = torch.full((a.shape[0], a.shape[1] + pad), 7.0, dtype=_dev(a).dtype, device="cuda")
    wide[:, :a.shape[1]] = _dev(a)
    return wide[:, :a.shape[1]]


def _check_codes(y, a_q, s_a, slack):
    a_q, s_a = a_q.cpu().numpy(), s_a.cpu().numpy().astype(np.float64)
    s = np.abs(y).max(1) / 127
    assert np.all(np.abs(s_a - s) <= REL * s), "scales"
    assert np.abs(a_q.astype(int)).max(initial=0) <= 127
    quotient = np.divide(y, s[:, None], out=np.zeros_like(y), where=s[:, None] > 0)
    assert np.abs(a_q - quotient).max(initial=0) <= 0.5 + slack, "codes"
    assert not a_q[s == 0].any() and not s_a[s == 0].any()


# M on both sides of the number of CUs; K: one vector, a wave's, odd counts, each row length class and the one that reads twice
SHAPES = [(1, 8), (3, 512), (1, 520), (2, 2048), (5, 2056), (777, 1352), (300, 4096), (2, 5120), (9, 8200), (3, 16384), (2, 16392), (2, 32768),
          (2, 32776), (1, 131072)]


@pytest.mark.parametrize("residual", ["none", "fp16", "fp32"])
@pytest.mark.parametrize("M,K", SHAPES)
def test_norm(M, K, residual):
    rng = np.random.default_rng(M * 131 + K)
    x, gain = _rows(rng, M, K), (1 + 0.3 * rng.standard_normal(K)).astype(np.float16)
    r = None if residual == "none" else (3 * rng.standard_normal((M, K))).astype(np.float16 if residual == "fp16" else np.float32)
    total, y = ref.add_rmsnorm(x, gain, r, 1e-6)
    d_x, d_r, d_g = _padded(x, 24), None if r is None else _padded(r, 8), _dev(gain)
    got_sum, a_q, s_a = qqq.qqq_add_rmsnorm_quant(d_x, d_g, d_r, 1e-6)
    got_sum2, got_y = qqq.qqq_add_rmsnorm(d_x, d_g, d_r, 1e-6)
    torch.cuda.synchronize()
    if r is None:
        assert got_sum is None and got_sum2 is None
    else:
        want = total if residual == "fp16" else (x.astype(np.float32) + r)
        assert np.array_equal(got_sum.cpu().numpy(), want) and np.array_equal(got_sum2.cpu().numpy(), want)
    _check_codes(y, a_q, s_a, 127 * (2 ** -22 if residual != "fp32" else 2 ** -21))
    got = got_y.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - y) <= np.abs(y) * (2 ** -11 + REL) + 2 ** -25)


@pytest.mark.parametrize("residual", ["none", "fp16", "fp32"])
@pytest.mark.parametrize("M,K", [(300, 5128), (300, 8192), (280, 12296), (280, 16384)])
def test_norm_of_more_rows_than_compute_units(M, K, residual):
    """Rows of more than 4096 values, four vectors a thread: prompts of the larger models."""
    test_norm(M, K, residual)


def test_norm_sum_in_the_residuals_place():
    rng = np.random.default_rng(5)
    for K in (1024, 40000):
        x, r, gain = _rows(rng, 7, K), rng.standard_normal((7, K)).astype(np.float32), np.ones(K, np.float16)
        d_x, d_r, d_g = _dev(x), _dev(r), _dev(gain)
        apart = qqq.qqq_add_rmsnorm_quant(d_x, d_g, d_r)
        same = qqq.qqq_add_rmsnorm_quant(d_x, d_g, d_r, sum_out=d_r)
        torch.cuda.synchronize()
        assert same[0] is d_r
        for a, b in zip(apart, same):
            assert torch.equal(a, b)


def test_norm_rows_of_zeros_and_of_tiny_and_large_values():
    rng = np.random.default_rng(6)
    x = _rows(rng, 6, 1000)
    x[1] = 0
    x[2] = 6e-8                                   # the least fp16 value
    x[3] = 65504                                  # the largest
    x[4, 1:] = 0                                  # a single value
    gain = np.ones(1000, np.float16)
    gain[::7] = 0
    for eps in (0.0, 1e-6):
        total, y = ref.add_rmsnorm(x, gain, None, eps)
        _, a_q, s_a = qqq.qqq_add_rmsnorm_quant(_dev(x), _dev(gain), eps=eps)
        _, got = qqq.qqq_add_rmsnorm(_dev(x), _dev(gain), eps=eps)
        torch.cuda.synchronize()
        _check_codes(y, a_q, s_a, 127 * 2 ** -22)
        assert np.all(np.abs(got.cpu().numpy() - y) <= np.abs(y) * (2 ** -11 + REL) + 2 ** -25)


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("M,F", [(1, 8), (4, 504), (1, 2048), (300, 1368), (16, 11008), (5, 13824), (3, 28672), (2, 32768), (2, 40000), (1, 131072)])
def test_gated(M, F, act):
    rng = np.random.default_rng(M * 17 + F)
    both = _rows(rng, M, 2 * F, 1.5)
    y = ref.gated_act(both[:, :F], both[:, F:], act)
    d = _dev(both)
    a_q, s_a = qqq.qqq_gated_act_quant(d[:, :F], d[:, F:], act)
    torch.cuda.synchronize()
    _check_codes(y, a_q, s_a, 127 * REL)


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("M,F", [(7, 2056), (300, 4096), (5, 4104), (300, 8192), (3, 8200)])
def test_gated_rows_of_every_length_class(M, F, act):
    test_gated(M, F, act)


def test_gated_products_past_fp16_and_rows_of_nothing():
    g = np.array([[300.0, -300.0, 1.0, 0, 0, 0, 0, 0], [0] * 8, [-65504.0] * 8, [-60.0] * 8], np.float16)
    u = np.array([[400.0, 400.0, 1.0, 0, 0, 0, 0, 0], [5] * 8, [65504.0] * 8, [6e-8] * 8], np.float16)
    for act in ("silu", "gelu_tanh"):
        y = ref.gated_act(g, u, act)
        y[np.abs(y).max(1) / 127 < 2.0 ** -120] = 0              # rows that count as zero
        a_q, s_a = qqq.qqq_gated_act_quant(_dev(g), _dev(u), act)
        torch.cuda.synchronize()
        assert float(s_a[0]) * 127 > 65504
        _check_codes(y, a_q, s_a, 127 * REL)


def test_codes_feed_the_gemm():
    """The codes and scales are what the W4A8 GEMM takes: its accumulators are those of the codes, in integers."""
    rng = np.random.default_rng(9)
    M, K, N = 5, 1024, 256
    x = _dev(_rows(rng, M, K))
    _, a_q, s_a = qqq.qqq_add_rmsnorm_quant(x, torch.ones(K, dtype=torch.float16, device="cuda"))
    w_nat, s_w = qqq.qqq_quantize_w4_perchannel(torch.randn(N, K, device="cuda").half())
    acc = torch.empty(M, N, dtype=torch.int32, device="cuda")
    y = qqq.qqq_gemm_w4a8_perchannel(a_q, s_a, qqq.qqq_pack_w4(w_nat, K), s_w, qqq.new_workspace(M, N, K), acc_out=acc)
    nibbles = torch.stack([(w_nat >> (4 * i)) & 15 for i in range(8)], -1).reshape(N, K)
    w = torch.where(nibbles > 7, nibbles - 16, nibbles).double()
    want = a_q.double().cpu() @ w.cpu().t()
    assert torch.equal(acc.cpu().double(), want)
    assert torch.isfinite(y).all()


def test_another_stream_and_graph_replays():
    """On a stream of its own, and captured: every replay gives what a call of its own gives."""
    x, r = torch.randn(33, 4096, device="cuda").half(), torch.randn(33, 4096, device="cuda").half()
    gain = torch.ones(4096, dtype=torch.float16, device="cuda")
    a_q, s_a, total = torch.empty(33, 4096, dtype=torch.int8, device="cuda"), torch.empty(33, device="cuda"), torch.empty_like(r)
    a_q2, s_a2 = torch.empty(33, 2048, dtype=torch.int8, device="cuda"), torch.empty(33, device="cuda")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        qqq.qqq_add_rmsnorm_quant(x, gain, r, a_q=a_q, s_a=s_a, sum_out=total)
        qqq.qqq_gated_act_quant(total[:, :2048], total[:, 2048:], a_q=a_q2, s_a=s_a2)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qqq.qqq_add_rmsnorm_quant(x, gain, r, a_q=a_q, s_a=s_a, sum_out=total)
        qqq.qqq_gated_act_quant(total[:, :2048], total[:, 2048:], a_q=a_q2, s_a=s_a2)
    for _ in range(3):
        x.copy_(torch.randn(33, 4096, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (total, a_q, s_a, a_q2, s_a2)]
        want = qqq.qqq_add_rmsnorm_quant(x, gain, r)
        want2 = qqq.qqq_gated_act_quant(want[0][:, :2048], want[0][:, 2048:])
        torch.cuda.synchronize()
        for a, b in zip(got, (*want, *want2)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("residual", [None, torch.float16, torch.float32])
def test_more_rows_than_the_last_level_cache_holds(residual):
    """Calls that read past the caches: the same bits as calls of a thousand rows, which do not."""
    M, K = 17000, 5120
    x, gain = torch.randn(M, K, device="cuda").half(), torch.randn(K, device="cuda").half()
    r = None if residual is None else torch.randn(M, K, device="cuda", dtype=residual)
    h, a, s = qqq.qqq_add_rmsnorm_quant(x, gain, r)
    h2, y = qqq.qqq_add_rmsnorm(x, gain, r)
    for at in range(0, M, 1000):
        part = slice(at, at + 1000)
        ph, pa, ps = qqq.qqq_add_rmsnorm_quant(x[part], gain, None if r is None else r[part])
        _, py = qqq.qqq_add_rmsnorm(x[part], gain, None if r is None else r[part])
        assert torch.equal(pa, a[part]) and torch.equal(ps, s[part]) and torch.equal(py, y[part]), at
        assert r is None or (torch.equal(ph, h[part]) and torch.equal(ph, h2[part])), at


@pytest.mark.parametrize("F", [8200, 28672])
def test_more_gated_rows_than_the_last_level_cache_holds(F):
    M = 7000
    x = torch.randn(M, 2 * F, device="cuda").half()
    a, s = qqq.qqq_gated_act_quant(x[:, :F], x[:, F:])
    for at in range(0, M, 1000):
        pa, ps = qqq.qqq_gated_act_quant(x[at:at + 1000, :F], x[at:at + 1000, F:])
        assert torch.equal(pa, a[at:at + 1000]) and torch.equal(ps, s[at:at + 1000]), at
