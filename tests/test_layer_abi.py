"""CPU-only checks of include/qqq_layer.h's boundary: exports, and arguments that are refused on the host before anything is enqueued."""
import ctypes
import os
import re

import pytest
import torch

from paper_2406_09904_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD = ctypes.c_void_p(0x1000)   # never dereferenced: every call below fails validation, or has nothing to do
ODD = ctypes.c_void_p(0x1008)
NULL, SHAPE, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2406_09904_amd import build
        build.build()
    return binding.lib()


def test_header_functions_are_exported(L):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "qqq_layer.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(qqq_[a-z0-9_]+)\s*\(", src)))
    assert names == sorted(binding.LAYER_SYMBOLS)
    for n in names:
        assert hasattr(L, n), n


def test_norm_refusals(L):
    def call(x=BAD, ldx=64, res=BAD, ldr=64, kind=1, gain=BAD, eps=1e-6, M=4, K=64, out=BAD, lds=64, a_q=BAD, s_a=BAD):
        return L.qqq_add_rmsnorm_quant(x, ldx, res, ldr, kind, gain, eps, M, K, out, lds, a_q, s_a, None)
    assert call(M=0) == 0
    for bad in (dict(K=60), dict(K=0), dict(K=131080, ldx=131080, ldr=131080, lds=131080), dict(M=-1), dict(ldx=56), dict(ldx=68), dict(ldr=56), dict(lds=66),
                dict(kind=3), dict(kind=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=ODD), dict(res=ODD), dict(out=ODD), dict(a_q=ODD),
                dict(gain=ODD), dict(s_a=ctypes.c_void_p(0x1002)), dict(kind=0), dict(lds=72)):
        assert call(**bad) == SHAPE, bad    # (kind=0: a residual without its type; lds=72: in the residual's place with another stride)
    for missing in ("x", "res", "gain", "out", "a_q", "s_a"):
        assert call(**{missing: None}) == NULL, missing
    assert L.qqq_add_rmsnorm(BAD, 64, None, 0, 0, BAD, 1e-6, 4, 64, None, 0, None, None) == NULL
    assert L.qqq_add_rmsnorm(BAD, 64, None, 0, 0, BAD, 1e-6, 4, 64, None, 0, ODD, None) == SHAPE
    assert b"qqq_add_rmsnorm" in L.qqq_last_error()


def test_gated_refusals(L):
    def call(g=BAD, ldg=128, u=BAD, ldu=128, act=0, M=4, F=64, a_q=BAD, s_a=BAD):
        return L.qqq_gated_act_quant(g, ldg, u, ldu, act, M, F, a_q, s_a, None)
    assert call(M=0) == 0
    for bad in (dict(F=4), dict(F=65), dict(ldg=56), dict(ldu=130), dict(act=2), dict(act=-1), dict(g=ODD), dict(u=ODD), dict(a_q=ODD)):
        assert call(**bad) == SHAPE, bad
    for missing in ("g", "u", "a_q", "s_a"):
        assert call(**{missing: None}) == NULL, missing


def _cache(**more):
    c = dict(k_codes=0x1000, k_scale=0x1000, v_codes=0x1000, v_scale=0x1000, k_tail=0x1000, v_tail=0x1000, pages=10, slots=2, kv_heads=2, head_dim=128, page_tokens=32)
    c.update(more)
    return binding._Cache(**c)


def _batch(**more):
    b = dict(page_table=0x1000, table_stride=4, kv_len=0x1000, cu=0x1000, slots=None, columns=4, sequences=2, max_new=3, max_len=4 * 32 + 31)
    b.update(more)
    return binding._Batch(**b)


CACHE_REFUSALS = [dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=128), dict(head_dim=96), dict(head_dim=0), dict(kv_heads=0), dict(pages=0), dict(slots=0),
                  dict(pages=1 << 31), dict(pages=1 << 30, kv_heads=2)]
BATCH_REFUSALS = [dict(sequences=-1), dict(max_new=-1), dict(max_len=-1), dict(columns=-1), dict(table_stride=3), dict(max_len=5 * 32), dict(max_new=(1 << 30) + 1)]
POINTER_REFUSALS = [({n: None}, {}, NULL) for n in ("k_codes", "k_scale", "v_codes", "v_scale", "k_tail", "v_tail")] + [
    ({}, {n: None}, NULL) for n in ("page_table", "kv_len", "cu")] + [({n: 0x1008}, {}, SHAPE) for n in ("k_codes", "v_codes", "k_tail", "v_tail")] + [
    ({}, {"slots": 0x1002}, SHAPE), ({}, {"cu": 0x1001}, SHAPE)]


def _attend(L, c, b, q=BAD, qt=1024, qh=128, heads=8, T=5, scale=0.1, causal=1, window=0, out=BAD, lse=BAD, work=BAD, nbytes=1 << 30):
    return L.qqq_attention_kv8(ctypes.byref(c) if c is not None else None, ctypes.byref(b) if b is not None else None, q, qt, qh, heads, T, scale, causal, window, out, lse,
                               work, nbytes, None)


def test_cache_and_batch_refusals(L):
    calls = [lambda c, b: L.qqq_kv8_append(ctypes.byref(c), ctypes.byref(b), BAD, 256, 128, BAD, 256, 128, 5, None),
             lambda c, b: L.qqq_kv8_read(ctypes.byref(c), ctypes.byref(b), BAD, BAD, 5, None), lambda c, b: _attend(L, c, b)]
    for call in calls:
        for bad in CACHE_REFUSALS:
            assert call(_cache(**bad), _batch()) == SHAPE, bad
        for bad in BATCH_REFUSALS:
            assert call(_cache(), _batch(**bad)) == SHAPE, bad
        for cache, batch, rc in POINTER_REFUSALS:
            assert call(_cache(**cache), _batch(**batch)) == rc, (cache, batch)
        # nothing to do: no sequence, no new token
        assert call(_cache(), _batch(sequences=0)) == 0 and call(_cache(), _batch(max_new=0)) == 0
    assert L.qqq_kv8_append(None, ctypes.byref(_batch()), BAD, 256, 128, BAD, 256, 128, 5, None) == NULL
    assert L.qqq_kv8_read(ctypes.byref(_cache()), None, BAD, BAD, 5, None) == NULL


def test_append_read_and_attention_refusals(L):
    c, b = _cache(), _batch()
    r = ctypes.byref
    for args, rc in (((None, 256, 128, BAD, 256, 128, 5), NULL), ((BAD, 256, 128, None, 256, 128, 5), NULL), ((BAD, 260, 128, BAD, 256, 128, 5), SHAPE),
                     ((BAD, 256, 4, BAD, 256, 128, 5), SHAPE), ((BAD, 256, 128, BAD, -256, 128, 5), SHAPE), ((ODD, 256, 128, BAD, 256, 128, 5), SHAPE),
                     ((BAD, 256, 128, BAD, 256, 128, -1), SHAPE), ((BAD, 256, 128, BAD, 256, 128, 0), 0)):
        assert L.qqq_kv8_append(r(c), r(b), *args, None) == rc, args
    assert L.qqq_kv8_read(r(c), r(b), None, BAD, 5, None) == NULL and L.qqq_kv8_read(r(c), r(b), BAD, ODD, 5, None) == SHAPE
    for bad in (dict(heads=7), dict(heads=0), dict(qt=1020), dict(qh=4), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1),
                dict(window=5, causal=0), dict(q=ODD), dict(out=ODD), dict(work=ODD), dict(lse=ctypes.c_void_p(0x1002)), dict(T=-1)):
        assert _attend(L, c, b, **bad) == SHAPE, bad
    assert _attend(L, c, b, q=None) == NULL and _attend(L, c, b, out=None) == NULL and _attend(L, None, b) == NULL
    # a long past of few rows is split over workgroups: that needs its workspace
    long = _batch(columns=4000, table_stride=4000, max_len=4000 * 32)
    need = L.qqq_attention_kv8_workspace_bytes(r(c), r(long), 8, 5)
    assert need > 0 and need % 8 == 0
    assert _attend(L, c, long, work=None) == WORKSPACE and _attend(L, c, long, nbytes=1024) == WORKSPACE
    assert b"workspace" in L.qqq_last_error()
    assert L.qqq_attention_kv8_workspace_bytes(r(c), r(b), 8, 5) == 0            # a short one is not
    assert L.qqq_attention_kv8_workspace_bytes(r(c), r(long), 7, 5) == 0 and L.qqq_attention_kv8_workspace_bytes(r(_cache(pages=0)), r(long), 8, 5) == 0


def test_a_window_never_needs_more_workspace(L):
    """The query does not know the window: what it gives is enough for every one."""
    c = _cache(head_dim=64, page_tokens=64, pages=1000)
    for sequences in (1, 3, 20, 200):
        for max_new in (1, 5, 40, 300):
            for tiles in (1, 7, 8, 9, 63, 100, 129, 500):
                for window in (1, 100, 1000, 5000, 20000):
                    long = _batch(columns=tiles, table_stride=tiles, max_len=tiles * 64, sequences=sequences, max_new=max_new)
                    narrow = _batch(columns=tiles, table_stride=tiles, max_len=min(tiles * 64, window + max_new), sequences=sequences, max_new=max_new)
                    a, b = (L.qqq_attention_kv8_workspace_bytes(ctypes.byref(c), ctypes.byref(x), 8, 1000) for x in (long, narrow))
                    assert b <= a, (sequences, max_new, tiles, window)


def _windowed_call(L, sequences, max_new, max_len, window, kv_heads, q_heads, tokens):
    """The code of a call with a window and a workspace of the queried size.  Without a device it is never enqueued."""
    c = _cache(kv_heads=kv_heads, page_tokens=64, pages=100, slots=1000)
    b = _batch(columns=max_len // 64, table_stride=max(1, max_len // 64), max_len=max_len, sequences=sequences, max_new=max_new)
    need = L.qqq_attention_kv8_workspace_bytes(ctypes.byref(c), ctypes.byref(b), q_heads, tokens)
    return _attend(L, c, b, heads=q_heads, T=tokens, window=window, work=BAD if need else None, nbytes=need)


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="made-up pointers: only where nothing can be launched")
def test_the_queried_workspace_is_enough_for_the_call_with_any_window(L):
    """Windows a little shorter than the past among them, whose first key may lie inside a tile."""
    for sequences in (1, 2, 3, 16, 48, 300):
        for max_new in (1, 3, 40, 300):
            for kv_heads, q_heads in ((1, 1), (8, 64), (32, 32)):
                for max_len in (400, 512, 1000, 1024, 2048, 3827, 60000):
                    for less in (0, 1, 12, 28, 32, 62, 63, 64, 72, 100, 400, 2000):
                        window = max(1, max_len - less)
                        rc = _windowed_call(L, sequences, max_new, max_len, window, kv_heads, q_heads, sequences * max_new)
                        assert rc not in (NULL, SHAPE, WORKSPACE), (sequences, max_new, kv_heads, q_heads, max_len, window, L.qqq_last_error())


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="made-up pointers: only where nothing can be launched")
@pytest.mark.parametrize("sequences,max_len", [(199, 734743714), (300, 1 << 29), (3000, 50_000_000)])
def test_the_queried_workspace_is_enough_with_a_window_where_all_tiles_pass_31_bits(L, sequences, max_len):
    """Without a window the keys of such calls are not split; with one they are."""
    for window in (1000, 100_000, max_len // 2):
        for kv_heads, q_heads in ((1, 8), (7, 21)):
            rc = _windowed_call(L, sequences, 1, max_len, window, kv_heads, q_heads, sequences)
            assert rc not in (NULL, SHAPE, WORKSPACE), (window, kv_heads, L.qqq_last_error())


def test_binding_refuses_cpu_tensors_and_shapes_that_disagree():
    x = torch.zeros((2, 64), dtype=torch.float16)
    gain = torch.ones(64, dtype=torch.float16)
    cache = binding.KV8Cache(torch.zeros(2, 1, 16, 64, dtype=torch.uint8), torch.zeros(2, 1), torch.zeros(2, 1, 64, 16, dtype=torch.uint8), torch.zeros(2, 1),
                             torch.zeros(1, 1, 16, 64, dtype=torch.float16), torch.zeros(1, 1, 64, 16, dtype=torch.float16))
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    batch = binding.KV8Batch(i32(0, 1).view(1, 2), i32(3), i32(0, 3), None, 3, 30)
    kv = torch.zeros(3, 1, 64, dtype=torch.float16)
    for call in (lambda: binding.qqq_add_rmsnorm(x, gain), lambda: binding.qqq_add_rmsnorm_quant(x, gain), lambda: binding.qqq_gated_act_quant(x, x),
                 lambda: binding.qqq_gated_act_quant(x, x, "relu"), lambda: binding.qqq_kv8_append(cache, batch, kv, kv), lambda: binding.qqq_kv8_read(cache, batch, kv, kv),
                 lambda: binding.qqq_kv8_read(cache, batch), lambda: binding.qqq_attention_kv8(cache, batch, kv)):
        with pytest.raises(ValueError):
            call()
