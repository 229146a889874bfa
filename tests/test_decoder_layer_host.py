"""Which workspaces the decoder layer's linear calls get (paper_2406_09904_amd/decoder_layer.py), on the host, with the library's calls replaced."""
import types

import pytest
import torch

from paper_2406_09904_amd import binding
from paper_2406_09904_amd import decoder_layer as dl

HIDDEN, HQ, HK, D, FFN = 128, 2, 1, 64, 128


class Calls:
    """The binding's calls that the layer makes, without a device; keeps every workspace that a linear call was given."""

    def __init__(self):
        self.given = []
        f16 = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
        codes = lambda x: (torch.zeros(x.shape, dtype=torch.int8), torch.zeros(x.shape[0]))  # noqa: E731

        def linear(x, packed, scale, work):
            self.given.append(work)
            return f16(x.shape[0], packed.shape[0])

        self.module = types.SimpleNamespace(
            KV8Cache=binding.KV8Cache, KV8Batch=binding.KV8Batch,
            qqq_quantize_w4_perchannel=lambda w: (w, torch.ones(w.shape[0])), qqq_pack_w4=lambda w, K: w,
            new_linear_workspace=lambda M, N, K, device="cpu": torch.zeros(64, dtype=torch.uint8),
            qqq_linear_workspace_bytes=lambda M, N, K: 64, qqq_gemm_workspace_zero_bytes=lambda M, N, K: 32,
            qqq_gemm_w4a8_perchannel=lambda a_q, s_a, packed, scale, work: linear(a_q, packed, scale, work), qqq_linear_w4a8_perchannel=linear,
            qqq_add_rmsnorm_quant=lambda x, gain, residual, eps, sum_out=None: (residual, *codes(x)),
            qqq_kv8_append=lambda *a: None, qqq_attention_kv8=lambda cache, batch, q, window=0: (f16(*q.shape), None),
            qqq_gated_act_quant=lambda gate, up: codes(gate))


@pytest.fixture
def calls(monkeypatch):
    c = Calls()
    monkeypatch.setattr(dl, "qqq", c.module)
    dl._workspace_sizes.cache_clear()
    yield c
    dl._workspace_sizes.cache_clear()


def _layer():
    w = lambda n, k: torch.zeros(n, k, dtype=torch.float16)  # noqa: E731
    gain = torch.ones(HIDDEN, dtype=torch.float16)
    return dl.DecoderLayer(w((HQ + 2 * HK) * D, HIDDEN), w(HIDDEN, HQ * D), w(2 * FFN, HIDDEN), w(HIDDEN, FFN), gain, gain, HQ, HK, D)


def _step(layer, tokens, **more):
    x = torch.zeros(tokens, HIDDEN, dtype=torch.float16)
    return layer(x, x.clone(), None, None, torch.arange(tokens), **more)


def test_calls_that_may_overlap_share_no_workspace(calls):
    """Counters and partial sums lie there: two streams that run one layer with as many rows must not meet in them."""
    layer = _layer()
    _step(layer, 3)
    _step(layer, 3)
    assert len(calls.given) == 8
    assert len({w.untyped_storage().data_ptr() for w in calls.given}) == 8


def test_given_workspaces_are_used_and_their_rows_checked(calls):
    layer = _layer()
    work = layer.new_workspaces(3)
    for _ in range(2):
        _step(layer, 3, workspaces=work)
    first = [w.data_ptr() for w in calls.given[:4]]
    assert len(set(first)) == 4 and [w.data_ptr() for w in calls.given[4:]] == first
    with pytest.raises(ValueError):
        _step(layer, 4, workspaces=work)


def test_only_the_part_that_must_be_zero_is_cleared(calls, monkeypatch):
    monkeypatch.setattr(torch.Tensor, "new_empty", lambda self, n: torch.full((n,), 7, dtype=self.dtype))
    work = _layer().new_workspaces(2)
    for w in work[1:]:
        assert not w[:32].any() and w[32:].eq(7).all()
