"""The int8 product (include/qqq_serve.h).  Sums are whole numbers below 2^53: compared with the products in 64 bits, equal; outputs are the formula's roundings, bit for bit:
fp32(acc) and its product with s_a are one rounding each, the product of that and s_w is exact in 64 bits and rounded once."""
import numpy as np
import pytest
import torch

from paper_2406_09904_amd import binding as qqq

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def automatic():
    yield
    qqq.set_w8a8_tuning(0, 0)


def _codes(gen, *shape):
    return torch.randint(-127, 128, shape, generator=gen, device="cuda").to(torch.int8)


def _want(a_q, s_a, w_q, s_w, dtype):
    acc = a_q.double() @ w_q.double().t()
    t = acc.float() * s_a[:, None]                      # two roundings to fp32
    y = t.double() * s_w.double()[None, :]
    return acc.to(torch.int64), torch.from_numpy(y.cpu().numpy().astype(np.float16 if dtype == torch.float16 else np.float32)).cuda()


def _check(M, N, K, seed=0, dtypes=(torch.float16, torch.float32), ldy=None, offset=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + M * 7 + N)
    a_q, w_q = _codes(gen, M, K), _codes(gen, N, K)
    s_a, s_w = 1e-3 + torch.rand(M, generator=gen, device="cuda"), 1e-3 * (1e-3 + torch.rand(N, generator=gen, device="cuda"))
    packed = qqq.qqq_pack_w8(w_q)
    for dtype in dtypes:
        acc, y = _want(a_q, s_a, w_q, s_w, dtype)
        wide = torch.full((M + 2, (ldy or N) + offset), 9.0, dtype=dtype, device="cuda")
        view = wide[1:M + 1, offset:offset + N]
        got_acc = torch.full((M, N), 7, dtype=torch.int32, device="cuda")
        assert qqq.qqq_gemm_w8a8(a_q, s_a, packed, s_w, y=view, acc_out=got_acc) is view
        assert torch.equal(got_acc.to(torch.int64), acc), (qqq.last_route(), M, N, K)
        assert torch.equal(view, y), (qqq.last_route(), M, N, K)
        view.fill_(9.0)
        assert (wide == 9).all(), "written beside the output"
        assert torch.equal(qqq.qqq_gemm_w8a8(a_q, s_a, packed, s_w, dtype=dtype), y)


# one row, operand order's last and the next, every row tile's ends, past them; one channel, less and more than a tile's, a wave's, a workgroup's
@pytest.mark.parametrize("M", [1, 2, 8, 9, 16, 17, 33, 48, 49, 64, 65, 130, 257])
@pytest.mark.parametrize("N,K", [(1, 128), (15, 256), (16, 1152), (130, 384), (515, 2176), (5003, 256)])
def test_sizes(M, N, K):
    _check(M, N, K)


# many rows of few channels: the few-rows kernel by 16, 32, 48 and 64 rows, and where it is not considered any more
@pytest.mark.parametrize("M,N,K", [(70, 40, 1024), (500, 100, 640), (1000, 33, 2048), (1333, 70, 256), (4096, 17, 384), (4097, 16, 384), (3000, 300, 128)])
def test_many_rows_of_few_channels(M, N, K):
    for shape in (0, 1):
        qqq.set_w8a8_tuning(shape, 0)
        _check(M, N, K)


@pytest.mark.parametrize("shape", range(1, 7))
@pytest.mark.parametrize("M", [1, 63, 64, 65, 300, 513])
def test_every_kernel(shape, M):
    for N, K in ((48, 128), (257, 256), (1000, 384), (511, 1024)):
        qqq.set_w8a8_tuning(shape, 0)
        _check(M, N, K, seed=shape)


@pytest.mark.parametrize("shape", range(1, 7))
@pytest.mark.parametrize("k_splits", [2, 3, 7, 100])
def test_parts_of_k(shape, k_splits):
    """Parts of one block of 128 among them."""
    for M, N, K in ((5, 77, 1024), (64, 300, 896), (270, 520, 384)):
        qqq.set_w8a8_tuning(shape, k_splits)
        _check(M, N, K, seed=k_splits)


TILES = {1: "w8a8 few rows ", 2: "w8a8 tile=256x256 ", 3: "w8a8 tile=192x256 ", 4: "w8a8 tile=128x256 ", 5: "w8a8 tile=128x128 ", 6: "w8a8 tile=64x128 "}


@pytest.mark.parametrize("shape", range(1, 7))
@pytest.mark.parametrize("k_splits", [0, 2, 7, 100])
def test_the_kernel_that_is_asked_for_runs(shape, k_splits):
    for M, N, K in ((1, 48, 1024), (270, 520, 384), (4097, 130, 256)):
        qqq.set_w8a8_tuning(shape, k_splits)
        _check(M, N, K, seed=shape, dtypes=(torch.float16,))
        route = qqq.last_route()
        if shape > 1 or M <= 4096:             # (the few-rows kernel is considered up to there)
            assert route.startswith(TILES[shape]), route
        assert ("ksplit=%d" % min(max(k_splits, 1), K // 128)) in route and route.endswith(" + sum") == (k_splits > 0), route


# (one row of short K over many channels is near the cost model's border: 3.7 us by the few-rows kernel, 4.6 by the smallest tile)
@pytest.mark.parametrize("M,N,K,shapes", [(1, 32000, 512, (1, 6)), (1, 32000, 4096, (1,)), (48, 5001, 1024, (1,)), (64, 130, 4096, (1,)), (3000, 9000, 512, (2,))])
def test_the_kernel_that_is_chosen(M, N, K, shapes):
    _check(M, N, K)
    assert any(qqq.last_route().startswith(TILES[s]) for s in shapes), qqq.last_route()


@pytest.mark.parametrize("M", [3, 100, 300])
@pytest.mark.parametrize("N,ldy,offset", [(64, 64, 0), (64, 67, 0), (64, 72, 3), (96, 104, 8), (333, 333, 1), (336, 344, 0)])
def test_output_rows_apart_and_unaligned(M, N, ldy, offset):
    _check(M, N, 256, ldy=ldy, offset=offset)


def test_the_ends_of_the_codes():
    """The largest sums: 127 * 127 * 131072 = 2^31 - 2^24 + ..; and weights of -128."""
    for M in (2, 80):
        for N, K in ((40, 131072),):
            a_q, w_q = torch.full((M, K), 127, dtype=torch.int8, device="cuda"), torch.full((N, K), 127, dtype=torch.int8, device="cuda")
            a_q[1], w_q[1::2] = -127, -127
            w_q[2] = -128
            a_q[0, 0] = 126
            s = torch.full((max(M, N),), 2.0 ** -16, device="cuda")
            acc = torch.empty(M, N, dtype=torch.int32, device="cuda")
            want_acc, y = _want(a_q, s[:M], w_q, s[:N], torch.float32)
            for shape in range(7):
                qqq.set_w8a8_tuning(shape, 0)
                got = qqq.qqq_gemm_w8a8(a_q, s[:M], qqq.qqq_pack_w8(w_q), s[:N], acc_out=acc, dtype=torch.float32)
                assert torch.equal(acc.to(torch.int64), want_acc) and torch.equal(got, y)


@pytest.mark.parametrize("N,K,pad", [(1, 128, 0), (16, 256, 16), (33, 384, 128), (1000, 1024, 0)])
def test_packing(N, K, pad):
    w = torch.randint(-128, 128, (N, K + pad), device="cuda").to(torch.int8)
    packed = qqq.qqq_pack_w8(w[:, :K])
    assert packed.numel() == (N + 15) // 16 * 16 * K and torch.equal(qqq.qqq_unpack_w8(packed, N, K), w[:, :K])


def test_a_linear_layer_of_fp16_weights():
    """Weights and activations through the library's own quantiser: each code is off by half a step, amax / 254, at most."""
    M, N, K = 70, 300, 512
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, w = torch.randn(M, K, generator=gen, device="cuda").half(), (torch.randn(N, K, generator=gen, device="cuda") * K ** -0.5).half()
    (a_q, s_a), (w_q, s_w) = qqq.qqq_quant_act(x), qqq.qqq_quant_act(w)
    y = qqq.qqq_gemm_w8a8(a_q, s_a, qqq.qqq_pack_w8(w_q), s_w, dtype=torch.float32).double()
    dx, dw = x.double().abs().amax(1) / 254, w.double().abs().amax(1) / 254
    bound = (dx[:, None] * w.double().abs().sum(1)[None, :] + dw[None, :] * x.double().abs().sum(1)[:, None] + K * dx[:, None] * dw[None, :]) * (1 + 1e-5)
    assert ((y - x.double() @ w.double().t()).abs() <= bound).all()


def test_sums_past_32_bit_places():
    """More than 2^31 bytes of weights and 2^31 outputs' bytes."""
    N, K, M = 140001, 16384, 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    w_q = torch.empty(N, K, dtype=torch.int8, device="cuda").random_(-127, 128, generator=gen)
    a_q, s = _codes(gen, M, K), torch.full((N,), 2.0 ** -20, device="cuda")
    packed = qqq.qqq_pack_w8(w_q)
    for rows in (3, 65):
        a = a_q[:1].expand(rows, K).contiguous() if rows > 3 else a_q
        y = qqq.qqq_gemm_w8a8(a, s[:rows], packed, s, dtype=torch.float32)
        part = slice(N - 300, N)
        assert torch.equal(y[:, part], _want(a, s[:rows], w_q[part], s[part], torch.float32)[1])


def test_wide_output_past_32_bits():
    M, N, K = 40000, 60000, 128
    gen = torch.Generator(device="cuda").manual_seed(2)
    a_q, w_q, s = _codes(gen, M, K), _codes(gen, N, K), torch.full((N,), 2.0 ** -10, device="cuda")
    y = qqq.qqq_gemm_w8a8(a_q, s[:M], qqq.qqq_pack_w8(w_q), s)
    for rows in (slice(0, 3), slice(M - 300, M)):
        assert torch.equal(y[rows], _want(a_q[rows], s[rows], w_q, s, torch.float16)[1])


def test_no_rows():
    w = qqq.qqq_pack_w8(torch.zeros(10, 128, dtype=torch.int8, device="cuda"))
    assert qqq.qqq_gemm_w8a8(torch.zeros(0, 128, dtype=torch.int8, device="cuda"), torch.zeros(0, device="cuda"), w, torch.zeros(10, device="cuda")).shape == (0, 10)


@pytest.mark.parametrize("M,shape,k_splits", [(1, 0, 0), (8, 1, 3), (200, 0, 0), (200, 4, 2)])
def test_captured(M, shape, k_splits):
    N, K = 777, 1024
    qqq.set_w8a8_tuning(shape, k_splits)
    gen = torch.Generator(device="cuda").manual_seed(3)
    a_q, w_q, s_a, s_w = _codes(gen, M, K), _codes(gen, N, K), torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    packed, work, y = qqq.qqq_pack_w8(w_q), qqq.new_w8a8_workspace(M, N, K), torch.empty(M, N, dtype=torch.float32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qqq.qqq_gemm_w8a8(a_q, s_a, packed, s_w, work, y=y)
    for turn in range(3):
        a_q.copy_(_codes(gen, M, K))
        work.fill_(0x55)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, _want(a_q, s_a, w_q, s_w, torch.float32)[1])


def test_refusals_on_the_device():
    """What neither path of the binding takes."""
    a_q, s_a, w, s_w = torch.zeros(2, 128, dtype=torch.int8, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(2048, dtype=torch.uint8, device="cuda"), torch.zeros(16, device="cuda")
    for call in (lambda: qqq.qqq_gemm_w8a8(a_q, s_a, w, s_w, dtype=torch.bfloat16), lambda: qqq.qqq_gemm_w8a8(a_q, s_a, w[:1024], s_w), lambda: qqq.qqq_gemm_w8a8(a_q, s_a[:1], w, s_w),
                 lambda: qqq.qqq_gemm_w8a8(a_q, s_a, w, s_w.half()), lambda: qqq.qqq_gemm_w8a8(a_q, s_a, w, s_w, y=torch.zeros(2, 15, device="cuda")),
                 lambda: qqq.qqq_gemm_w8a8(a_q, s_a, w, s_w, acc_out=torch.zeros(16, 2, dtype=torch.int32, device="cuda").t()), lambda: qqq.qqq_gemm_w8a8(a_q.cpu(), s_a, w, s_w),
                 lambda: qqq.qqq_gemm_w8a8(a_q, s_a, w.cpu(), s_w)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(qqq.QQQError):
        qqq.qqq_pack_w8(a_q[:, :112])


def test_tensors_of_another_device_than_the_current_one(monkeypatch):
    """As if the current device were another: refused, by the native marshalling's fall-back too."""
    a_q, s_a, w, s_w = torch.zeros(2, 128, dtype=torch.int8, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(2048, dtype=torch.uint8, device="cuda"), torch.zeros(16, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    monkeypatch.setattr(qqq, "_device", lambda: 1)
    monkeypatch.setattr(qqq, "_raw_stream", lambda device: stream)
    logits = torch.zeros(3, 40, device="cuda")
    sessions, batch = qqq.new_kv8_sessions(2, 3, 9), qqq.new_kv8_batch(2, 3, 1, 20)
    for call in (lambda: qqq.qqq_gemm_w8a8(a_q, s_a, w, s_w), lambda: qqq.qqq_logprobs(logits), lambda: qqq.qqq_kv8_plan(sessions, batch, batch.kv_len, 16),
                 lambda: qqq.qqq_kv8_release(sessions, 16), lambda: qqq.qqq_pack_w8(a_q)):
        with pytest.raises(ValueError, match="current device"):
            call()


def test_packing_one_channel_of_a_tensor_whose_rows_lie_anywhere():
    """One row's stride is used by nobody; of more rows it has to be a multiple of 16."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    wide = _codes(gen, 3, 265)
    assert torch.equal(qqq.qqq_unpack_w8(qqq.qqq_pack_w8(wide[:1, :256]), 1, 256), wide[:1, :256])
    with pytest.raises(qqq.QQQError):
        qqq.qqq_pack_w8(wide[:2, :256])
