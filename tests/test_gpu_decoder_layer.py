"""The layer's calls together (paper_2406_09904_amd/decoder_layer.py).

Tolerance of the whole layer against 64 bits with the same int4 weights: a code is off by at most half a step of amax / 127, for rows of normal
values (amax about 4 of their deviation) 4 / 127 / sqrt(12) = 0.9 % of it, in each of the four products, and keys and values likewise: 2 % of the
output's norm at most where they add up as independent errors, 6 % is asked.
"""
import numpy as np
import pytest
import torch

from oracle import qqq_oracle as orc
from paper_2406_09904_amd import binding as qqq
from paper_2406_09904_amd import decoder_layer as dl

pytestmark = pytest.mark.gpu

HIDDEN, HQ, HK, D, FFN = 512, 8, 2, 64, 1024


def _weights(linear):
    w_nat = qqq.qqq_unpack_w4(linear.packed, linear.N, linear.K).cpu().numpy().view(np.uint32)
    return orc.w8_perchannel(w_nat, linear.K).astype(np.float64) * linear.scale.cpu().numpy().astype(np.float64)[:, None]


def _reference(layer, x, lengths):
    """The layer in 64 bits on whole sequences, no cache."""
    norm = lambda h, g: h / np.sqrt((h * h).mean(-1, keepdims=True) + layer.eps) * g.cpu().numpy().astype(np.float64)  # noqa: E731
    w = [_weights(m) for m in (layer.qkv, layer.o, layer.gate_up, layer.down)]
    outs, streams, at = [], [], 0
    for n in lengths:
        h = x[at:at + n].astype(np.float64)
        at += n
        qkv = (norm(h, layer.gain_attention) @ w[0].T).reshape(n, HQ + 2 * HK, D)
        angle = np.arange(n)[:, None, None] * 10000.0 ** (-np.arange(0, D, 2) / D)
        a, b = qkv[:, :HQ + HK, :D // 2], qkv[:, :HQ + HK, D // 2:]
        rot = np.concatenate([a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)], -1)
        o = np.zeros((n, HQ, D))
        for head in range(HQ):
            s = rot[:, head] @ rot[:, HQ + head // (HQ // HK)].T * D ** -0.5
            s[np.triu_indices(n, 1)] = -np.inf
            p = np.exp(s - s.max(-1, keepdims=True))
            o[:, head] = p / p.sum(-1, keepdims=True) @ qkv[:, HQ + HK + head // (HQ // HK)]
        h = h + o.reshape(n, -1) @ w[1].T
        gu = norm(h, layer.gain_ffn) @ w[2].T
        g = gu[:, :FFN]
        outs.append((g / (1 + np.exp(-g)) * gu[:, FFN:]) @ w[3].T)
        streams.append(h)
    return np.concatenate(outs), np.concatenate(streams)


def _serve(layer, x, lengths, pieces, page):
    """x in pieces: how many tokens of each sequence a call takes."""
    B = len(lengths)
    table, pages = dl.pages_in_order(B, max(lengths), page)
    cache = qqq.new_kv8_cache(pages, HK, D, page, B)
    starts = np.concatenate([[0], np.cumsum(lengths)])
    done = np.zeros(B, int)
    y = torch.zeros(len(x), HIDDEN, dtype=torch.float16, device="cuda")
    stream = torch.zeros_like(y)
    for new in pieces:
        new = np.minimum(new, np.array(lengths) - done)
        rows = torch.from_numpy(np.concatenate([starts[b] + done[b] + np.arange(n) for b, n in enumerate(new)])).cuda()
        positions = torch.from_numpy(np.concatenate([done[b] + np.arange(n) for b, n in enumerate(new)])).cuda()
        done += new
        i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
        batch = qqq.KV8Batch(table, i32(done), i32(np.concatenate([[0], np.cumsum(new)])), None, int(new.max()), max(lengths))
        out, res = layer(x[rows], None, cache, batch, positions)
        y[rows], stream[rows] = out, res
    torch.cuda.synchronize()
    return y.cpu().numpy(), stream.cpu().numpy(), cache


def test_layer_against_64_bits_and_in_pieces():
    layer = dl.random_layer(HIDDEN, HQ, HK, D, FFN, seed=3)
    lengths = [70, 1, 33, 100]
    x = torch.randn(sum(lengths), HIDDEN, generator=torch.Generator().manual_seed(4)).half()
    want, want_stream = _reference(layer, x.numpy(), lengths)
    x = x.cuda()
    whole, stream, cache = _serve(layer, x, lengths, [[100] * 4], 32)
    for got, ref in ((whole, want), (stream, want_stream)):
        assert np.linalg.norm(got - ref) <= 0.06 * np.linalg.norm(ref)
    # a few tokens at a time, single tokens among them: keys and values do not depend on attention, so the cache is the same, bit for bit
    pieces = [[20, 1, 1, 40], [1, 1, 1, 1], [30, 1, 20, 30], [1, 1, 1, 1], [100] * 4]
    parts, _, cache2 = _serve(layer, x, lengths, pieces, 32)
    for name in ("k_codes", "k_scale", "v_codes", "v_scale"):
        assert torch.equal(getattr(cache, name), getattr(cache2, name)), name
    assert np.linalg.norm(parts.astype(np.float64) - want) <= 0.06 * np.linalg.norm(want)


def test_residual_in_place_over_two_layers():
    a, b = (dl.random_layer(HIDDEN, HQ, HK, D, FFN, seed=s) for s in (5, 6))
    n = 48
    table, pages = dl.pages_in_order(1, n, 16)
    caches = [qqq.new_kv8_cache(pages, HK, D, 16, 1) for _ in range(2)]
    batch = qqq.KV8Batch(table, torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda"), None, n, n)
    x = torch.randn(n, HIDDEN, device="cuda").half()
    positions = torch.arange(n, device="cuda")
    y, r = a(x.clone(), None, caches[0], batch, positions)
    kept = r.clone()
    y2, r2 = b(y, r, caches[1], batch, positions)
    torch.cuda.synchronize()
    assert r2.data_ptr() != r.data_ptr() and torch.equal(r, (kept.float() + y.float()).half())
    assert torch.isfinite(y2).all() and torch.isfinite(r2).all()


def _token_step(layer, sessions, seed, past=30):
    """A step of one token of each of some sessions behind a prompt -> what the layer is called with (the step can be repeated: it writes the same tokens again)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    table, pages = dl.pages_in_order(sessions, 64, 16)
    cache = qqq.new_kv8_cache(pages, HK, D, 16, sessions)
    i32 = lambda v: torch.full((sessions,), v, dtype=torch.int32, device="cuda")  # noqa: E731
    cu = torch.arange(sessions + 1, dtype=torch.int32, device="cuda")
    kv = torch.randn(sessions * past, 2, HK, D, generator=gen, device="cuda").half()
    qqq.qqq_kv8_append(cache, qqq.KV8Batch(table, i32(past), cu * past, None, past, 64), kv[:, 0], kv[:, 1])
    x, residual = (torch.randn(sessions, HIDDEN, generator=gen, device="cuda").half() for _ in range(2))
    return x, residual, cache, qqq.KV8Batch(table, i32(past + 1), cu, None, 1, 64), i32(past)


def _run(layer, step, **more):
    x, residual, cache, batch, positions = step
    return layer(x, residual.clone(), cache, batch, positions, **more)


def test_no_workspace_stays_behind():
    """Steps of ever other numbers of rows leave nothing allocated."""
    layer = dl.random_layer(HIDDEN, HQ, HK, D, FFN, seed=7)
    steps = [_token_step(layer, n, n) for n in (1, 5, 20, 70, 150)]
    _run(layer, steps[0])
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for step in steps:
        _run(layer, step)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() == before


@pytest.mark.parametrize("sessions", [3, 16, 40])
def test_steps_on_two_streams_at_once(sessions):
    layer = dl.random_layer(HIDDEN, HQ, HK, D, FFN, seed=8)
    steps = [_token_step(layer, sessions, seed) for seed in (1, 2)]
    want = [_run(layer, s) for s in steps]
    kept = [layer.new_workspaces(sessions) for _ in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    got = [[], []]
    for turn in range(10):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(_run(layer, steps[i], workspaces=kept[i] if turn % 2 else None))
    torch.cuda.synchronize()
    for i in range(2):
        for y, r in got[i]:
            assert torch.equal(y, want[i][0]) and torch.equal(r, want[i][1])


@pytest.mark.parametrize("sessions,keep", [(4, False), (4, True), (24, False), (100, False)])
def test_a_captured_step_between_eager_ones(sessions, keep):
    """A number of rows that is first met inside of a capture; eager steps of as many before the first replay and between the others."""
    layer = dl.random_layer(HIDDEN, HQ, HK, D, FFN, seed=9)
    step, other = _token_step(layer, sessions, 3), _token_step(layer, sessions + 1, 4)
    x, residual, cache, batch, positions = step
    work = layer.new_workspaces(sessions) if keep else None
    into = residual.clone()
    _run(layer, other)   # (another number of rows: torch's own libraries are ready)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        into.copy_(residual)
        y, r = layer(x, into, cache, batch, positions, work)
    want_y, want_r = _run(layer, step)
    torch.cuda.synchronize()
    for _ in range(4):
        graph.replay()
        again = _run(layer, step)
        torch.cuda.synchronize()
        assert torch.equal(y, want_y) and torch.equal(r, want_r)
        assert torch.equal(again[0], want_y) and torch.equal(again[1], want_r)


def test_workspaces_of_another_number_of_tokens_are_refused():
    layer = dl.random_layer(HIDDEN, HQ, HK, D, FFN, seed=10)
    with pytest.raises(ValueError):
        _run(layer, _token_step(layer, 3, 5), workspaces=layer.new_workspaces(4))
