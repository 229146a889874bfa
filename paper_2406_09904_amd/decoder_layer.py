"""A decoder layer served in W4A8 with its keys and values in 8 bits: the calls of ``binding`` in the order a program makes them.

    x, residual --qqq_add_rmsnorm_quant--> codes --GEMM--> queries, keys, values --rotary positions-->
        qqq_kv8_append, qqq_attention_kv8 --linear--> --qqq_add_rmsnorm_quant--> codes --GEMM--> gate, up --qqq_gated_act_quant--> codes --GEMM--> x

Run as a program it serves a few sessions on random weights: prompts in pieces, then single tokens from a captured graph.
"""
from __future__ import annotations

import functools
import typing

import torch

from . import binding as qqq


@functools.lru_cache(maxsize=4096)
def _workspace_sizes(rows, N, K):
    """(bytes of a linear call's workspace, those of its part that is to be zero)"""
    return max(qqq.qqq_linear_workspace_bytes(rows, N, K), 16), qqq.qqq_gemm_workspace_zero_bytes(rows, N, K)


class _Linear:
    """Per-channel W4A8 weights [N, K] from fp16."""

    def __init__(self, weight):
        self.N, self.K = weight.shape
        w_nat, self.scale = qqq.qqq_quantize_w4_perchannel(weight)
        self.packed = qqq.qqq_pack_w4(w_nat, self.K)
        self.empty = torch.empty((0,), dtype=torch.uint8, device=self.packed.device)

    def workspace(self, rows):
        """Of a call with that many rows.  Its first part is to be zero, and every call leaves it so."""
        nbytes, zero = _workspace_sizes(rows, self.N, self.K)
        work = self.empty.new_empty(nbytes)
        work[:zero].zero_()
        return work

    def of_codes(self, a_q, s_a, workspace=None):
        return qqq.qqq_gemm_w4a8_perchannel(a_q, s_a, self.packed, self.scale, self.workspace(a_q.shape[0]) if workspace is None else workspace)

    def __call__(self, x, workspace=None):
        return qqq.qqq_linear_w4a8_perchannel(x, self.packed, self.scale, self.workspace(x.shape[0]) if workspace is None else workspace)


class Workspaces(typing.NamedTuple):
    """The linear calls' workspaces of steps of so many tokens (DecoderLayer.new_workspaces)."""
    tokens: int
    qkv: torch.Tensor
    o: torch.Tensor
    gate_up: torch.Tensor
    down: torch.Tensor


class DecoderLayer:
    """w_qkv [(q_heads + 2 kv_heads) * head_dim, hidden], w_o [hidden, q_heads * head_dim], w_gate_up [2 * ffn, hidden], w_down [hidden, ffn] and the
    two norms' gains [hidden], all fp16 on the GPU."""

    def __init__(self, w_qkv, w_o, w_gate_up, w_down, gain_attention, gain_ffn, q_heads, kv_heads, head_dim, eps=1e-6, window=0, rope_base=10000.0):
        self.qkv, self.o, self.gate_up, self.down = _Linear(w_qkv), _Linear(w_o), _Linear(w_gate_up), _Linear(w_down)
        self.gain_attention, self.gain_ffn, self.eps, self.window = gain_attention, gain_ffn, eps, window
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.frequency = rope_base ** (-torch.arange(0, head_dim, 2, device=w_qkv.device, dtype=torch.float32) / head_dim)

    def rotate(self, x, positions):
        """Rotary positions on x [tokens, heads, head_dim] fp16: channel i and channel i + head_dim / 2 are a pair."""
        angle = positions.to(torch.float32)[:, None, None] * self.frequency
        cos, sin = angle.cos(), angle.sin()
        a, b = x.float().chunk(2, dim=-1)
        return torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1).half()

    def new_workspaces(self, tokens) -> Workspaces:
        """For a program that keeps them over steps of `tokens` tokens, which saves each step their clearing.  They hold counters and partial sums: steps that may
        run at the same time, on other streams or in other graphs, need workspaces of their own, and those of a graph are made outside of its capture."""
        return Workspaces(tokens, *(m.workspace(tokens) for m in (self.qkv, self.o, self.gate_up, self.down)))

    def __call__(self, x, residual, cache: qqq.KV8Cache, batch: qqq.KV8Batch, positions, workspaces: typing.Optional[Workspaces] = None):
        """x [tokens, hidden] fp16, the layer before's output, residual the stream that it is to be added to (None: x is the stream), positions [tokens]
        -> (x, residual) for the next layer, the residual a new tensor; the one that was given holds its sum with x then, without what attention adds.
        Without workspaces torch's allocator lends them for the call."""
        H, Hk, D = self.q_heads, self.kv_heads, self.head_dim
        if workspaces is not None and workspaces.tokens != x.shape[0]:
            raise ValueError("workspaces of %d tokens for %d" % (workspaces.tokens, x.shape[0]))
        work = workspaces or Workspaces(x.shape[0], None, None, None, None)
        total, a_q, s_a = qqq.qqq_add_rmsnorm_quant(x, self.gain_attention, residual, self.eps, sum_out=residual)
        residual = x if total is None else total
        qkv = self.qkv.of_codes(a_q, s_a, work.qkv).view(-1, H + 2 * Hk, D)
        q, k = self.rotate(qkv[:, :H], positions), self.rotate(qkv[:, H:H + Hk], positions)
        qqq.qqq_kv8_append(cache, batch, k, qkv[:, H + Hk:])
        attended, _ = qqq.qqq_attention_kv8(cache, batch, q, window=self.window)
        y = self.o(attended.view(-1, H * D), work.o)
        residual, a_q, s_a = qqq.qqq_add_rmsnorm_quant(y, self.gain_ffn, residual, self.eps)
        gate_up = self.gate_up.of_codes(a_q, s_a, work.gate_up)
        ffn = self.down.K
        a_q, s_a = qqq.qqq_gated_act_quant(gate_up[:, :ffn], gate_up[:, ffn:])
        return self.down.of_codes(a_q, s_a, work.down), residual


def random_layer(hidden=4096, q_heads=32, kv_heads=8, head_dim=128, ffn=11008, seed=0, device="cuda", **more) -> DecoderLayer:
    g = torch.Generator(device=device).manual_seed(seed)
    w = lambda n, k: (torch.randn(n, k, generator=g, device=device) * k ** -0.5).half()  # noqa: E731
    gain = lambda: (1 + 0.1 * torch.randn(hidden, generator=g, device=device)).half()  # noqa: E731
    return DecoderLayer(w((q_heads + 2 * kv_heads) * head_dim, hidden), w(hidden, q_heads * head_dim), w(2 * ffn, hidden), w(hidden, ffn), gain(), gain(),
                        q_heads, kv_heads, head_dim, **more)


def pages_in_order(sequences, max_len, page_tokens, device="cuda"):
    """A page table that gives every sequence its own pages, one after the other -> (table, pages)."""
    per = max(1, max_len // page_tokens)
    return torch.arange(sequences * per, dtype=torch.int32, device=device).view(sequences, per), sequences * per


def main():
    sessions, prompt, steps, page = 8, 500, 20, 64
    max_len = prompt + steps
    layer = random_layer()
    columns = max_len // page
    held = qqq.new_kv8_sessions(sessions, columns, sessions * columns)
    cache = qqq.new_kv8_cache(sessions * columns, layer.kv_heads, layer.head_dim, page, sessions)
    new = torch.zeros(sessions, dtype=torch.int32, device="cuda")
    # prompts, in two pieces
    for n in (300, prompt - 300):
        batch = qqq.new_kv8_batch(sessions, columns, n, max_len)
        positions = torch.zeros(sessions * n, dtype=torch.int32, device="cuda")
        qqq.qqq_kv8_plan(held, batch, new.fill_(n), page, positions=positions)
        x, residual = layer(torch.randn(sessions * n, 4096, device="cuda").half(), None, cache, batch, positions)
    # single tokens: one captured step, replayed
    x, residual = torch.randn(sessions, 4096, device="cuda").half(), torch.zeros(sessions, 4096, device="cuda").half()
    batch, positions = qqq.new_kv8_batch(sessions, columns, 1, max_len), torch.zeros(sessions, dtype=torch.int32, device="cuda")
    work = layer.new_workspaces(sessions)   # (the graph's own)

    def step(residual):
        qqq.qqq_kv8_plan(held, batch, new, page, positions=positions)
        return layer(x, residual, cache, batch, positions, work)

    new.zero_()
    step(residual.clone())   # (once outside of the capture; it brings no token)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, stream = step(residual)
    new.fill_(1)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    print("one layer, hidden 4096, %d sessions past %d tokens: %.1f us a step" % (sessions, prompt, start.elapsed_time(end) / steps * 1e3))


if __name__ == "__main__":
    main()
