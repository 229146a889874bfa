"""CPU-only checks of include/qqq_serve.h's boundary: exports, and arguments that are refused on the host before anything is enqueued."""
import ctypes
import os
import re

import pytest
import torch

from paper_2406_09904_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD = ctypes.c_void_p(0x1000)   # never dereferenced: every call below fails validation, or has nothing to do
NULL, SHAPE, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2406_09904_amd import build
        build.build()
    return binding.lib()


def test_header_functions_are_exported(L):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "qqq_serve.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(qqq_[a-z0-9_]+)\s*\(", src)))
    assert names == sorted(binding.SERVE_SYMBOLS)
    for n in names:
        assert hasattr(L, n), n


def _sessions(**more):
    s = dict(pages=0x1000, pages_stride=4, held=0x1000, held_after=0x1000, free_pages=0x1000, free_count=0x1000, free_count_after=0x1000, pool=10, sessions=3, columns=4,
             page_tokens=32)
    s.update(more)
    return binding._Sessions(**s)


def _batch(**more):
    b = dict(page_table=0x2000, table_stride=4, kv_len=0x1000, cu=0x1000, slots=None, columns=4, sequences=2, max_new=3, max_len=4 * 32 + 31)
    b.update(more)
    return binding._Batch(**b)


def _plan(L, s, b, new=BAD, tokens=6, sequence=BAD, positions=BAD, lacking=BAD, work=BAD, nbytes=1 << 20):
    return L.qqq_kv8_plan(ctypes.byref(s) if s is not None else None, ctypes.byref(b) if b is not None else None, new, tokens, sequence, positions, lacking, work, nbytes, None)


SESSION_REFUSALS = [dict(page_tokens=8), dict(page_tokens=48), dict(sessions=0), dict(columns=-1), dict(pages_stride=3), dict(pool=-1), dict(pool=(1 << 30) + 1)]


def test_plan_refusals(L):
    for bad in SESSION_REFUSALS + [dict(columns=3), dict(sessions=1), dict(pages=0x1002), dict(held=0x1001), dict(held_after=0x1002), dict(free_pages=0x1002), dict(free_count=0x1002),
                                   dict(free_count_after=0x1002)]:
        assert _plan(L, _sessions(**bad), _batch()) == SHAPE, bad
    for missing in ("pages", "held", "held_after", "free_pages", "free_count", "free_count_after"):
        assert _plan(L, _sessions(**{missing: None}), _batch()) == NULL, missing
    for bad in (dict(sequences=-1), dict(max_new=-1), dict(max_new=(1 << 30) + 1), dict(max_len=-1), dict(max_len=5 * 32), dict(columns=-1), dict(table_stride=3), dict(columns=3),
                dict(sequences=4), dict(sequences=1 << 24, slots=0x1000), dict(page_table=0x2002), dict(kv_len=0x1001), dict(cu=0x1002), dict(slots=0x1002),
                dict(page_table=0x1000, slots=0x1000), dict(page_table=0x1000, table_stride=5)):    # the last two: the sessions' own table with slots, with another stride
        assert _plan(L, _sessions(), _batch(**bad)) == SHAPE, bad
    for missing in ("page_table", "kv_len", "cu"):
        assert _plan(L, _sessions(), _batch(**{missing: None})) == NULL, missing
    for bad in (dict(tokens=-1), dict(tokens=(1 << 30) + 1), dict(new=ctypes.c_void_p(0x1001)), dict(sequence=ctypes.c_void_p(0x1002)), dict(positions=ctypes.c_void_p(0x1002)),
                dict(lacking=ctypes.c_void_p(0x1002)), dict(work=ctypes.c_void_p(0x1002))):
        assert _plan(L, _sessions(), _batch(), **bad) == SHAPE, bad
    assert _plan(L, None, _batch()) == NULL and _plan(L, _sessions(), None) == NULL and _plan(L, _sessions(), _batch(), new=None) == NULL
    # large tables are made in two launches, which need a workspace
    s, b = _sessions(sessions=3000, columns=4000, pages_stride=4000), _batch(sequences=3000, columns=4000, table_stride=4000, max_len=4000 * 32)
    need = L.qqq_kv8_plan_workspace_bytes(ctypes.byref(s), ctypes.byref(b))
    assert need == 3000 * 4
    assert _plan(L, s, b, work=None) == WORKSPACE and _plan(L, s, b, nbytes=need - 1) == WORKSPACE
    assert b"workspace" in L.qqq_last_error()
    assert L.qqq_kv8_plan_workspace_bytes(ctypes.byref(_sessions()), ctypes.byref(_batch())) == 0
    assert L.qqq_kv8_plan_workspace_bytes(ctypes.byref(_sessions(page_tokens=7)), ctypes.byref(b)) == 0


def test_release_refusals(L):
    def call(ids=BAD, count=2, **more):
        return L.qqq_kv8_release(ctypes.byref(_sessions(**more)), ids, count, None)
    for bad in SESSION_REFUSALS + [dict(held_after=0x1004), dict(free_count_after=0x1004), dict(count=-1), dict(count=4, ids=None), dict(ids=ctypes.c_void_p(0x1002)), dict(held=0x1002, held_after=0x1002)]:
        assert call(**bad) == SHAPE, bad
    assert call(held=None) == NULL and call(free_pages=None) == NULL and call(pages=None) == NULL
    assert L.qqq_kv8_release(None, BAD, 1, None) == NULL
    assert call(count=0) == 0


def test_binding_refuses_cpu_tensors_and_shapes_that_disagree():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    sessions = binding.KV8Sessions(i32(2, 3), i32(2), i32(9), i32(1))
    batch = binding.KV8Batch(i32(2, 3), i32(2), i32(3), None, 4, 50)
    for call in (lambda: binding.qqq_kv8_plan(sessions, batch, i32(2), 16), lambda: binding.qqq_kv8_release(sessions, 16), lambda: binding.qqq_kv8_plan_workspace_bytes(sessions, batch, 16)):
        with pytest.raises(ValueError):
            call()


def test_logprobs_refusals(L):
    def call(x=BAD, ld=100, kind=0, M=3, V=100, tokens=BAD, top=5, logprob=BAD, entropy=BAD, lse=BAD, top_tokens=BAD, top_logprobs=BAD, work=BAD, nbytes=1 << 20):
        return L.qqq_logprobs(x, ld, kind, M, V, tokens, top, logprob, entropy, lse, top_tokens, top_logprobs, work, nbytes, None)
    odd = ctypes.c_void_p(0x1002)
    assert call(M=0) == 0
    for bad in (dict(M=-1), dict(M=1 << 24), dict(V=0), dict(V=1 << 30, ld=1 << 30), dict(ld=99), dict(kind=2), dict(kind=-1), dict(top=-1), dict(top=65), dict(x=ctypes.c_void_p(0x1001)),
                dict(x=odd, kind=1), dict(tokens=odd), dict(logprob=odd), dict(entropy=odd), dict(lse=odd), dict(top_tokens=odd), dict(top_logprobs=odd), dict(work=ctypes.c_void_p(0x1008))):
        assert call(**bad) == SHAPE, bad
    for missing in ("x", "tokens", "logprob", "top_tokens", "top_logprobs"):
        assert call(**{missing: None}) == NULL, missing
    need = L.qqq_logprobs_workspace_bytes(1, 100000, 0)
    assert need > 0 and need % 4 == 0
    assert call(M=1, V=100000, ld=100000, nbytes=need - 1) == WORKSPACE and call(M=1, V=100000, ld=100000, work=None) == WORKSPACE
    assert b"workspace" in L.qqq_last_error()
    assert L.qqq_logprobs_workspace_bytes(5000, 100000, 0) == 0 and L.qqq_logprobs_workspace_bytes(1, 100, 0) == 0 and L.qqq_logprobs_workspace_bytes(1, 0, 0) == 0


def test_logprobs_binding_refusals():
    x = torch.zeros(2, 30, dtype=torch.float16)
    for call in (lambda: binding.qqq_logprobs(x), lambda: binding.qqq_logprobs(x.double()), lambda: binding.qqq_logprobs(x[0]), lambda: binding.qqq_logprobs(x.t())):
        with pytest.raises(ValueError):
            call()


def test_product_refusals(L):
    def call(a=BAD, s_a=BAD, w=BAD, s_w=BAD, y=BAD, kind=0, ldy=100, acc=None, M=3, N=100, K=256, work=BAD, nbytes=1 << 30):
        return L.qqq_gemm_w8a8(a, s_a, w, s_w, y, kind, ldy, acc, M, N, K, work, nbytes, None)
    odd = ctypes.c_void_p(0x1002)
    assert call(M=0) == 0
    for bad in (dict(M=-1), dict(M=(1 << 30) + 1), dict(N=0), dict(N=1 << 24, K=2176, ldy=1 << 25), dict(N=(1 << 24) + 1, ldy=1 << 25), dict(K=200), dict(K=0), dict(K=131072 + 128), dict(kind=2), dict(kind=-1), dict(ldy=99), dict(a=ctypes.c_void_p(0x1008)),
                dict(w=ctypes.c_void_p(0x1008)), dict(s_a=odd), dict(s_w=odd), dict(y=ctypes.c_void_p(0x1001)), dict(y=odd, kind=1), dict(acc=odd), dict(work=ctypes.c_void_p(0x1008))):
        assert call(**bad) == SHAPE, bad
    for missing in ("a", "s_a", "w", "s_w", "y"):
        assert call(**{missing: None}) == NULL, missing
    assert L.qqq_set_w8a8_tuning(9, 0) == -1 and L.qqq_set_w8a8_tuning(0, -1) == -1
    assert L.qqq_set_w8a8_tuning(0, 2) == 0
    try:
        need = L.qqq_gemm_w8a8_workspace_bytes(3, 100, 256)
        assert need == 2 * 3 * 100 * 4 and call(nbytes=need - 1) == WORKSPACE and call(work=None) == WORKSPACE
    finally:
        L.qqq_set_w8a8_tuning(0, 0)
    assert L.qqq_gemm_w8a8_workspace_bytes(3, 100, 200) == 0 and L.qqq_gemm_w8a8_workspace_bytes(0, 100, 256) == 0


def test_packing_refusals(L):
    assert L.qqq_packed_w8_bytes(17, 256) == 32 * 256 and L.qqq_packed_w8_bytes(0, 256) == 0 and L.qqq_packed_w8_bytes(1 << 24, 2176) == 0 and L.qqq_packed_w8_bytes(16, 200) == 0
    other = ctypes.c_void_p(0x2000)
    assert L.qqq_pack_w8(BAD, 16, 256, 255, other, None) == SHAPE and L.qqq_pack_w8(BAD, 16, 256, 264, other, None) == SHAPE and L.qqq_pack_w8(BAD, 16, 256, 256, BAD, None) == SHAPE
    assert L.qqq_pack_w8(None, 16, 256, 256, other, None) == NULL and L.qqq_pack_w8(BAD, 16, 256, 256, None, None) == NULL
    assert L.qqq_pack_w8(ctypes.c_void_p(0x1008), 16, 256, 256, other, None) == SHAPE and L.qqq_pack_w8(BAD, 16, 100, 112, other, None) == SHAPE
    assert L.qqq_unpack_w8(None, 16, 256, other, None) == NULL and L.qqq_unpack_w8(BAD, 16, 256, BAD, None) == SHAPE and L.qqq_unpack_w8(BAD, 16, 100, other, None) == SHAPE


def test_product_binding_refusals():
    i8 = lambda *s: torch.zeros(s, dtype=torch.int8)  # noqa: E731
    f32 = lambda *s: torch.zeros(s)  # noqa: E731
    for call in (lambda: binding.qqq_pack_w8(i8(16, 128)), lambda: binding.qqq_pack_w8(f32(16, 128)), lambda: binding.qqq_unpack_w8(torch.zeros(2048, dtype=torch.uint8), 16, 128),
                 lambda: binding.qqq_gemm_w8a8(i8(2, 128), f32(2), torch.zeros(2048, dtype=torch.uint8), f32(16))):
        with pytest.raises(ValueError):
            call()
