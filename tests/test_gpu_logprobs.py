"""Log probabilities, entropies and largest logits (include/qqq_serve.h) against the definitions in 64 bits.

Tolerances.  u = 2^-24, a rounding to fp32.  An exponential e^d: d is one rounding, d log2(e) another and the constant's, the instruction an ulp: relative |d| 3 u + 2 u.  Weighted with the
exponentials themselves |d| is |t| / z <= log V on average.  A thread adds at most V / 256 of them, then come 4 or fewer rescalings a batch of 16 at least (two
roundings and an exponential each, counted below as 6 u for every 16) and some 60 additions.  So z is within r = (V / 256 (1 + 6 / 16) + 100 + 3 log V) u of its value,
t within that of sum |d| e <= z log V, and
    |lse - exact| <= r + 2 u (|lse| + |m| + log V),   |logprob - exact| <= r + 2 u (|logprob| + |m - x| + log V),   |entropy - exact| <= r (1 + 2 log V) + 4 u log V.
Places are whole numbers and equal.
"""
import numpy as np
import pytest
import torch

from oracle import qqq_serve_oracle as ref
from paper_2406_09904_amd import binding as qqq

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _device(x, pad=0, offset=0):
    """x in rows that are `pad` values further apart, the first `offset` values behind an aligned place."""
    wide = torch.full((x.shape[0], x.shape[1] + pad + offset), 3.0, dtype=torch.float16 if x.dtype == np.float16 else torch.float32, device="cuda")
    wide[:, offset:offset + x.shape[1]] = torch.from_numpy(x).cuda()
    return wide[:, offset:offset + x.shape[1]]


def _close(got, want, tolerance, what):
    got = got.cpu().numpy().astype(np.float64)
    want = np.where(np.abs(want) > np.finfo(np.float32).max, np.copysign(np.inf, want), want)   # (differences of the type's two ends are past fp32)
    odd = ~np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[odd & ~np.isnan(want)], want[odd & ~np.isnan(want)]), what
    bad = np.abs(got - np.where(odd, 0, want)) > tolerance
    assert not (bad & ~odd).any(), (what, np.abs(got - want)[bad & ~odd].max(), np.argwhere(bad & ~odd)[:3])


def _check(x, top, tokens=None, pad=0, offset=0, rng=None):
    M, V = x.shape
    if tokens is None:
        tokens = (rng or np.random.default_rng(V)).integers(0, V, M).astype(np.int32)
    want = ref.logprobs(x, tokens, top)
    out = qqq.qqq_logprobs(_device(x, pad, offset), torch.from_numpy(tokens).cuda(), top)
    log_v = np.log(V) + 1e-30
    r = (V / 256 * (1 + 6 / 16) + 100 + 3 * log_v) * U
    with np.errstate(invalid="ignore"):
        largest = np.abs(np.where(np.isfinite(x), x.astype(np.float64), -1e300).max(1))
        largest = np.where(largest == 1e300, 0, largest)
        _close(out.lse, want[2], r + 2 * U * (np.abs(want[2]) + largest + log_v), "lse")
        _close(out.logprob, want[0], r + 2 * U * (2 * np.abs(want[0]) + 2 * log_v), "logprob")
        _close(out.entropy, want[1], r * (1 + 2 * log_v) + 4 * U * log_v, "entropy")
        if top:
            assert np.array_equal(out.top_tokens.cpu().numpy(), want[3]), "top tokens"
            _close(out.top_logprobs, want[4], r + 2 * U * (2 * np.abs(want[4]) + 2 * log_v), "top logprobs")
    return out


def _logits(rng, M, V, dtype):
    x = 2.5 * rng.standard_normal((M, V))
    x[np.arange(M)[:, None], rng.integers(0, V, (M, 5))] += 10 * rng.random((M, 5))
    return x.astype(dtype)


# one value, less and more than 16 bytes, a thread's, a wave's, both workgroup sizes, split rows and whole ones, several turns of a thread
SIZES = [(1, 1), (3, 2), (2, 7), (5, 9), (4, 63), (600, 65), (3, 511), (7, 1000), (1, 8192), (2, 8193), (513, 4099), (1, 16385), (30, 16391), (1, 32000), (3, 50001), (2, 131071),
         (520, 20011), (100, 700), (90, 40013), (70, 70001), (1, 600011)]


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("M,V", SIZES)
def test_sizes(M, V, dtype):
    rng = np.random.default_rng(M * 31 + V)
    x = _logits(rng, M, V, dtype)
    for top, pad, offset in ((0, 0, 0), (1, 1, 0), (20, 8, 3), (64, 5, 1)):
        _check(x, top, pad=pad, offset=offset, rng=rng)


# rows of a workgroup of 256, of 1024, split rows (and their joining)
WAYS = [(530, 3001), (530, 17001), (4, 12000), (2, 70000)]


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("M,V", WAYS)
def test_masks_and_what_is_no_number(M, V, dtype):
    rng = np.random.default_rng(V)
    M0, M = M, max(M, 12)
    x = _logits(rng, M, V, dtype)
    lowest = np.finfo(dtype).min
    x[0, :] = -np.inf                                   # nothing
    x[1, rng.random(V) < 0.999] = -np.inf               # little
    x[2, :] = -np.inf
    x[2, V // 3] = 1.5                                  # one, the probability 1
    x[3, rng.random(V) < 0.99] = lowest
    x[4, :] = lowest                                    # all equal, at the type's end
    x[5, 17], x[5, V - 1] = np.nan, np.nan
    x[6, V // 2] = np.inf
    x[7, ::2], x[7, 1::2] = lowest, -np.inf
    x[8, :] = -lowest                                   # the other end
    x[9, 5] = -lowest
    x[9, 6:] = lowest
    x[10, :] = 0.0
    x[10, ::3] = -0.0                                   # equal
    x[11, :] = np.nan
    tokens = rng.integers(0, V, M).astype(np.int32)
    tokens[[1, 6]], tokens[2] = V, V // 3
    for top in (0, 3, 64):
        for rows in ([slice(0, M)] if M0 == M else [slice(i, i + M0) for i in range(0, M, M0)]):    # (few at a time where few rows are what is tested)
            _check(x[rows], top, tokens[rows], pad=3)


@pytest.mark.parametrize("M,V", WAYS)
@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "few values", "one thread's"])
def test_orders(M, V, kind):
    """Equal values go by their place; values that come in the worst order."""
    rng = np.random.default_rng(V)
    if M > 4:
        M = 513 if V > 10000 else 530
    x = np.zeros((M, V), np.float32)
    if kind == "rising":
        x[:] = np.arange(V) * 1e-3
    elif kind == "falling":
        x[:] = -np.arange(V) * 1e-3
    elif kind == "few values":
        x[:] = rng.integers(0, 4, (M, V))
    elif kind == "one thread's":
        x[:, 1024:1024 + 8] = 5 + np.arange(8) % 3
        x[:, V - 9:] = 5
    for dtype in (np.float16, np.float32):
        for top in (1, 40, 64):
            _check(x.astype(dtype)[:3 if kind in ("rising", "falling") and M > 4 else M], top) if M <= 4 else _check_some(x.astype(dtype), top)


def _check_some(x, top):
    """All rows on the device, where they are whole; the host's check of some."""
    out = qqq.qqq_logprobs(_device(x), None, top)
    some = [0, 1, len(x) // 2, len(x) - 1]
    want = ref.logprobs(x[some], None, top)
    assert out.logprob is None
    assert np.array_equal(out.top_tokens.cpu().numpy()[some], want[3])
    r = (x.shape[1] / 256 * (1 + 6 / 16) + 100 + 3 * np.log(x.shape[1])) * U
    _close(out.lse[some], want[2], r + 2 * U * (np.abs(want[2]) + np.abs(x[some]).max(1) + np.log(x.shape[1])), "lse")


# rows of 256 threads value by value and by blocks, of 512, of 1024, in registers or not, split ones
@pytest.mark.parametrize("M,V", [(300, 700), (600, 30011), (100, 700), (100, 3001), (100, 9001), (100, 40013), (70, 70001), (70, 200003), (2100, 40013), (2, 70000), (1, 12000)])
@pytest.mark.parametrize("dtype", [np.float16, np.float32])
def test_more_candidates_than_there_is_room_for(M, V, dtype):
    """Values in great number that are the last of the largest, or are more than that: only the first of them count, wherever in the row they lie."""
    rng = np.random.default_rng(M + V)
    lowest, inf = np.finfo(dtype).min, np.inf
    rows = []
    for masked in (-inf, lowest):                                           # few allowed
        for allowed in (1, 5, 63):
            r = np.full(V, masked)
            r[rng.permutation(V)[:allowed]] = 3 * rng.standard_normal(allowed)
            rows.append(r)
    r = np.full(V, -inf)                                                    # few allowed, some at the type's end, nothing else
    r[rng.permutation(V)[:13]] = lowest
    r[rng.permutation(V)[:3]] = [1, 2, 1]
    rows.append(r)
    for value in (2.0, 0.0, inf, np.nan):                                   # the last quarter, and the same with three above and a tail that is not
        r = rng.uniform(-5, -1, V)
        r[V - V // 4:] = value
        if value == 0:
            r[V - V // 4:][rng.random(V // 4) < 0.5] = -0.0
        rows.append(r)
        rows.append(np.where(np.arange(V) > V - 9, -7.0, r))
        rows[-1][[V // 2, 1, V - 1]] = 4.0
    r = np.floor(rng.uniform(0, 3, V))                                      # three values, the largest rare at first
    r[:V // 2] = np.minimum(r[:V // 2], 1)
    rows.append(r)
    rows.append(np.sort(rng.uniform(-8, 8, V)))                             # rising
    rows.append(np.where(np.arange(V) % 2, np.nan, inf))
    rows = np.stack(rows).astype(dtype)
    for top in (1, 2, 20, 64):
        for offset in (0, 1):
            want = ref.logprobs(rows, None, top)
            for begin in range(0, len(rows), M):                            # (few rows at a time where that is what is tested)
                some = rows[begin:begin + M]
                n = len(some)
                out = qqq.qqq_logprobs(_device(some[np.arange(M) % n], offset=offset, pad=1), None, top)    # the rows again and again, until it is M
                for i in {0, max(0, (M - n) // n * n)}:
                    assert np.array_equal(out.top_tokens[i:i + n].cpu().numpy(), want[3][begin:begin + n]), (top, offset)
                    r = (V / 256 * (1 + 6 / 16) + 100 + 3 * np.log(V)) * U
                    with np.errstate(invalid="ignore"):
                        _close(out.top_logprobs[i:i + n], want[4][begin:begin + n], r + 2 * U * (2 * np.abs(want[4][begin:begin + n]) + 2 * np.log(V)), "top logprobs")


def test_rows_that_are_past_the_last_cache():
    """Logits of more than the last level of cache holds, in both sizes of workgroup."""
    for M, V, dtype in ((2100, 80001, np.float16), (3000, 50001, np.float32), (9000, 20001, np.float16)):
        rng = np.random.default_rng(V)
        some = _logits(rng, 7, V, dtype)
        dev = torch.from_numpy(some).cuda().repeat((M + 6) // 7, 1)[:M].contiguous()
        assert dev.numel() * dev.element_size() > 256 << 20
        for top in (0, 7):
            out = qqq.qqq_logprobs(dev, None, top)
            want = ref.logprobs(some, None, top)
            last = (M - 7) // 7 * 7
            for i in (0, last):
                r = (V / 256 * (1 + 6 / 16) + 100 + 3 * np.log(V)) * U
                _close(out.lse[i:i + 7], want[2], r + 2 * U * (np.abs(want[2]) + np.abs(some).max(1) + np.log(V)), "lse")
                if top:
                    assert np.array_equal(out.top_tokens[i:i + 7].cpu().numpy(), want[3])
            # equal rows, equal numbers, where they begin at as many bytes behind 16 (which threads have which values goes by that): every 56th of these odd rows
            assert torch.equal(out.lse, out.lse[:56].repeat((M + 55) // 56)[:M])


# (rows, values, how many of the largest) for each kernel, of fp16; fp32's rows are half as long
KERNELS = [(3, 3000, 5, "in registers threads=512 blocks=1"), (3, 7001, 5, "in registers threads=512 blocks=2"), (400, 16001, 5, "in registers threads=512 blocks=4"),
           (3, 32003, 5, "in registers threads=512 blocks=8"), (3, 48001, 20, "in registers threads=512 blocks=16"), (3, 48001, 64, "in registers threads=1024 blocks=8"),
           (80, 128003, 7, "in registers threads=1024 blocks=16"), (80, 140003, 7, "in turns threads=1024 past=false tracked=false"),
           (530, 30011, 5, "in turns threads=256 past=false tracked=false"), (9000, 20001, 5, "in turns threads=256 past=true tracked=false"),
           (530, 40013, 5, "in turns threads=512 past=false tracked=false"), (2100, 80001, 5, "in turns threads=512 past=true tracked=false"),
           (600, 60001, 64, "in turns threads=512 past=false tracked=true"), (2100, 80001, 20, "in turns threads=512 past=true tracked=true"), (2, 100001, 5, "in parts")]


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("M,V,top,kernel", KERNELS)
def test_every_kernel(M, V, top, kernel, dtype):
    """By the kernels' names, so that a limit that moves is seen: ordinary rows, masked ones, equal, rising and falling ones and what is no number."""
    V = V if dtype == np.float16 else (V + 1) // 2
    rng = np.random.default_rng(V + top)
    some = _logits(rng, 11, V, dtype)
    some[1, rng.random(V) < 0.99] = -np.inf
    some[2, :] = -np.inf
    some[3, rng.random(V) < 0.999] = np.finfo(dtype).min
    some[4, :] = 1.25
    some[5] = np.sort(rng.uniform(-8, 8, V))
    some[6] = np.sort(rng.uniform(-8, 8, V))[::-1]
    some[7, V // 2] = np.nan
    some[8, [V - 1, 3]] = np.inf
    some[9, V // 3:] = 2.0
    tokens = rng.integers(0, V, 11).astype(np.int32)
    want = ref.logprobs(some, tokens, top)
    log_v = np.log(V)
    r = (V / 256 * (1 + 6 / 16) + 100 + 3 * log_v) * U
    for begin in range(0, 11, M):              # (few rows at a time where that is what is tested)
        rows = np.arange(begin, min(begin + M, 11))
        of = torch.from_numpy(rows[np.arange(M) % len(rows)]).cuda()
        dev = torch.from_numpy(some).cuda()[of]
        out = qqq.qqq_logprobs(dev, torch.from_numpy(tokens).cuda()[of], top)
        assert qqq.last_route().startswith("logprobs " + kernel), qqq.last_route()
        for at in {0, (M - 1) // len(rows) * len(rows)}:
            n = min(len(rows), M - at)
            x, got, w = some[rows[:n]], [o[at:at + n] for o in out], [o[rows[:n]] for o in want]
            with np.errstate(invalid="ignore"):
                largest = np.abs(np.where(np.isfinite(x), x.astype(np.float64), -1e300).max(1))
                largest = np.where(largest == 1e300, 0, largest)
                _close(got[2], w[2], r + 2 * U * (np.abs(w[2]) + largest + log_v), "lse")
                _close(got[0], w[0], r + 2 * U * (2 * np.abs(w[0]) + 2 * log_v), "logprob")
                _close(got[1], w[1], r * (1 + 2 * log_v) + 4 * U * log_v, "entropy")
                assert np.array_equal(got[3].cpu().numpy(), w[3]), "top tokens"
                _close(got[4], w[4], r + 2 * U * (2 * np.abs(w[4]) + 2 * log_v), "top logprobs")


def test_no_token_and_a_short_vocabulary():
    x = _logits(np.random.default_rng(1), 6, 5, np.float16)
    out = _check(x, 9, np.array([-1, 0, 4, 5, -2 ** 31, 2 ** 31 - 1], np.int32))
    assert (out.top_tokens[:, 5:] == -1).all() and (out.top_logprobs[:, 5:] == -np.inf).all()


def test_outputs_that_are_not_wanted_and_rows_beside():
    rng = np.random.default_rng(2)
    x = _device(_logits(rng, 40, 9001, np.float32))
    whole = qqq.qqq_logprobs(x, None, 4)
    lse = torch.full((42,), 7.0, device="cuda")
    out = qqq.qqq_logprobs(x, None, 0, out=qqq.LogProbs(None, None, lse[1:41], None, None))
    assert torch.equal(out.lse, whole.lse) and lse[0] == 7 and lse[41] == 7
    assert qqq.qqq_logprobs(x[:0], None, 3).top_tokens.shape == (0, 3)


def test_the_same_twice_and_in_any_company():
    """A row's results do not depend on the run; parts of a row meet in one order."""
    x = _device(_logits(np.random.default_rng(3), 3, 100003, np.float16))
    a, b = qqq.qqq_logprobs(x, None, 64), qqq.qqq_logprobs(x, None, 64)
    for p, q in zip(a[1:], b[1:]):
        assert torch.equal(p, q)


def test_offsets_past_32_bits():
    """Rows that begin more than 2^31 values, and 2^32 bytes, behind the first."""
    V, rows = 4099, 3
    big = torch.empty((1 << 31) + 4 * V, dtype=torch.float16, device="cuda")
    x = big.as_strided((rows, V), (1 << 30, 1))
    host = _logits(np.random.default_rng(4), rows, V, np.float16)
    x.copy_(torch.from_numpy(host))
    out = qqq.qqq_logprobs(x, None, 5)
    assert np.array_equal(out.top_tokens.cpu().numpy(), ref.logprobs(host, None, 5)[3])
    del big, x


@pytest.mark.parametrize("M,V", [(1, 40000), (600, 5000)])
def test_captured(M, V):
    rng = np.random.default_rng(5)
    x, tokens = _device(_logits(rng, M, V, np.float16)), torch.zeros(M, dtype=torch.int32, device="cuda")
    out = qqq.qqq_logprobs(x, tokens, 10)
    work = torch.empty(max(16, qqq.qqq_logprobs_workspace_bytes(M, V)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qqq.qqq_logprobs(x, tokens, 10, out=out, workspace=work)
    for turn in range(3):
        x.copy_(torch.from_numpy(_logits(rng, M, V, np.float16)))
        tokens.random_(0, V)
        graph.replay()
        torch.cuda.synchronize()
        eager = qqq.qqq_logprobs(x, tokens, 10)
        for p, q in zip(out, eager):
            assert torch.equal(p, q)
