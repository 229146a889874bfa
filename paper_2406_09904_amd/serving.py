"""Sessions served through decoder layers, from token ids to the likeliest next ones, with no number that the host has to wait for:

    how many tokens each session brings --qqq_kv8_plan--> page table, lengths, rows' positions
    ids --embedding--> x --layers (decoder_layer.py)--> --qqq_add_rmsnorm_quant--> codes --qqq_gemm_w8a8--> logits --qqq_logprobs--> next ids

Run as a program it serves a few sessions on random weights: prompts of different lengths, scored, in one step, then single tokens from a captured graph,
while sessions end and others begin in their pages.
"""
from __future__ import annotations

import typing

import torch

from . import binding as qqq
from .decoder_layer import DecoderLayer, Workspaces, random_layer


class Head:
    """The vocabulary's product, weights [V, hidden] fp16: 8 bits, a scale a token.  The layers' 4 bits would show here, where no later layer evens them out."""

    def __init__(self, weight):
        self.V, self.K = weight.shape
        codes, self.scale = qqq.qqq_quant_act(weight)
        self.packed = qqq.qqq_pack_w8(codes)

    def __call__(self, a_q, s_a, workspace=None):
        return qqq.qqq_gemm_w8a8(a_q, s_a, self.packed, self.scale, workspace)


class Step(typing.NamedTuple):
    """A step's tensors (Server.new_step).  The program writes ids and new (and batch.slots); the rest is filled by the step.  A graph's are its own.

    A sequence brings fewer tokens than new says where max_new, max_len or the rows end, and none where a page that it needs is not there: batch.cu and batch.kv_len
    say what it brought and holds then.  The others are none the worse for it: ids, targets and the results of rows stay where new puts them."""
    ids: torch.Tensor        # int32 [rows]: the sequences' tokens, one sequence after the other (one outside of the vocabulary is its nearest end); rows behind the last one's hold any
    new: torch.Tensor        # int32 [sequences]: tokens that each has there, none for one that rests (written in place: it lies in starts)
    batch: qqq.KV8Batch
    positions: torch.Tensor  # int32 [rows], of the rows that are brought, one sequence after the other
    lacking: torch.Tensor    # int32 [1]: pages that were not there.  What is free goes to the first sequences; the first that wants more than is left, and those behind it that
                             # want any, bring nothing and hold what they held
    workspaces: typing.Optional[typing.List[Workspaces]]
    starts: torch.Tensor     # int32 [1 + sequences]: 0, then new
    sequence: torch.Tensor   # int32 [rows]: of the rows that are brought
    places: torch.Tensor     # int32 [rows]: 0, 1, 2, ..


class Server:
    """embedding [V, hidden] fp16, the layers, the last norm's gain [hidden] and head weights [V, hidden] fp16; a cache of `pages` pages that `sessions` sessions of
    up to max_len tokens share (pages: as many as all need at their longest)."""

    def __init__(self, embedding, layers: typing.Sequence[DecoderLayer], gain, head, sessions, max_len, page_tokens=64, pages=None):
        if not layers or embedding.shape != head.shape:
            raise ValueError("a server takes layers, and a head of the embedding's shape")
        self.embedding, self.layers, self.gain, self.head = embedding, list(layers), gain, Head(head)
        self.max_len, self.page_tokens = max_len, page_tokens
        columns = max(1, max_len // page_tokens)
        self.scarce = pages is not None and pages < sessions * (max_len // page_tokens)   # (else every session has its pages at its longest)
        pages = sessions * columns if pages is None else pages
        self.sessions = qqq.new_kv8_sessions(sessions, columns, pages, embedding.device)
        self.caches = [qqq.new_kv8_cache(pages, m.kv_heads, m.head_dim, page_tokens, sessions, embedding.device) for m in self.layers]

    def new_step(self, rows, max_new, slots=None, keep=False) -> Step:
        """Of up to `rows` rows, at most max_new of a sequence, of the sessions slots (int32 [sequences]; None: all in order).  keep: with workspaces of its own,
        for a graph."""
        if rows < 1:
            raise ValueError("a step of %d rows" % rows)
        sequences, device = self.sessions.held.numel() if slots is None else slots.numel(), self.embedding.device
        i32 = lambda n: torch.zeros((n,), dtype=torch.int32, device=device)  # noqa: E731
        batch = qqq.new_kv8_batch(sequences, self.sessions.pages.shape[1], max_new, self.max_len, slots, device)
        starts = i32(1 + sequences)
        return Step(i32(rows), starts[1:], batch, i32(rows), i32(1), [m.new_workspaces(rows) for m in self.layers] if keep else None, starts, i32(rows),
                    torch.arange(rows, dtype=torch.int32, device=device))

    def _affordable(self, step: Step, new):
        """new, or none for a sequence whose pages are not all there; counts those pages.  The plan itself would give such a sequence entries without a page: what append puts
        there is lost, and attention reads another session's page in its place."""
        held, slots, P = self.sessions.held, step.batch.slots, self.page_tokens
        if slots is None:
            held = held[:new.numel()]
        else:
            there = (slots >= 0) & (slots < held.numel())
            held, new = held.index_select(0, slots.clamp(0, held.numel() - 1)), new * there
        new = torch.minimum(new.clamp(0, step.batch.max_new), self.max_len - held)
        fresh = torch.div(held + new, P, rounding_mode="floor") - torch.div(held, P, rounding_mode="floor")
        wanted = fresh.cumsum(0)
        step.lacking.copy_((wanted[-1:] - self.sessions.free_count).clamp(min=0))
        return new * ((fresh == 0) | (wanted <= self.sessions.free_count))

    def __call__(self, step: Step, targets=None, top=1) -> qqq.LogProbs:
        """The step -> the `top` likeliest tokens behind each sequence's last row [sequences, top] and their log probabilities, or, given targets (int32 [rows]; below 0: none),
        those of every row and of its target.  A sequence that brings no token has every token equally likely (nothing of another's is in its results), a row that is not brought NaN."""
        rows, sequences, cu = step.ids.numel(), step.new.numel(), step.batch.cu
        starts = step.starts.clamp(0, rows).cumsum(0, dtype=torch.int32)
        new = torch.minimum(step.new, rows - starts[:-1])     # (what has no row brings nothing)
        scarce = self.scarce and sequences > 0
        if scarce:
            new = self._affordable(step, new)
        qqq.qqq_kv8_plan(self.sessions, step.batch, new, self.page_tokens, step.sequence, step.positions, None if scarce else step.lacking)
        # The rows that are brought lie one after the other; in ids those that are not stand between them
        of_row = ((starts - cu).index_select(0, step.sequence) + step.places).clamp_(0, rows - 1)
        x, residual = self.embedding.index_select(0, step.ids.index_select(0, of_row).clamp_(0, self.embedding.shape[0] - 1)), None
        for i, layer in enumerate(self.layers):
            x, residual = layer(x, residual, self.caches[i], step.batch, step.positions, step.workspaces and step.workspaces[i])
        if targets is None:
            at, none = (cu[1:] - 1).clamp_(min=0), cu[1:] == cu[:-1]
        else:
            sequence = torch.searchsorted(starts[1:], step.places, right=True, out_int32=True)
            at = (cu - starts).index_select(0, sequence) + step.places
            none = at >= cu.index_select(0, (sequence + 1).clamp_(max=sequences))
            at.clamp_(0, rows - 1)
        x, residual = x.index_select(0, at), residual.index_select(0, at)
        _, a_q, s_a = qqq.qqq_add_rmsnorm_quant(x, self.gain, residual, self.layers[-1].eps, sum_out=residual)
        s_a.masked_fill_(none, 0.0 if targets is None else float("nan"))
        return qqq.qqq_logprobs(self.head(a_q, s_a), targets, top)

    def release(self, ids=None):
        """Sessions ids (int32 on the device; None: all) end; their pages are free for others."""
        qqq.qqq_kv8_release(self.sessions, self.page_tokens, ids)


def random_server(layers=2, vocabulary=32000, hidden=4096, sessions=8, max_len=1024, page_tokens=64, pages=None, seed=0, device="cuda", **layer) -> Server:
    g = torch.Generator(device=device).manual_seed(seed + 1000)
    w = lambda scale: (torch.randn(vocabulary, hidden, generator=g, device=device) * scale).half()  # noqa: E731
    return Server(w(1.0), [random_layer(hidden, seed=seed + i, device=device, **layer) for i in range(layers)],
                  (1 + 0.1 * torch.randn(hidden, generator=g, device=device)).half(), w(2 * hidden ** -0.5), sessions, max_len, page_tokens, pages)


def main():
    sessions, steps, vocabulary = 8, 20, 32000
    server = random_server(vocabulary=vocabulary, sessions=sessions, max_len=1024)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    # prompts: all in one step, each row's token scored by the row before
    lengths = [500, 17, 1, 300, 64, 129, 250, 450]
    prompts = server.new_step(sum(lengths), max(lengths))
    prompts.ids.random_(0, vocabulary)
    prompts.new.copy_(i32(lengths))
    ends = i32(lengths).cumsum(0)
    targets = prompts.ids.roll(-1).index_fill_(0, ends - 1, -1)
    scored = server(prompts, targets)
    print("log probability of the prompts' tokens: %.3f on average" % (scored.logprob.sum() / (sum(lengths) - sessions)).item())
    # single tokens: one captured step, replayed
    step = server.new_step(sessions, 1, keep=True)
    server(step)                     # (once outside of the capture; it brings no token)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.ids.copy_(server(step).top_tokens[:, 0])
    step.ids.copy_(scored.top_tokens[ends - 1, 0])
    step.new.fill_(1)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    print("%d layers, hidden %d, %d tokens: %d sessions, %.1f us a step" % (len(server.layers), server.head.K, vocabulary, sessions, start.elapsed_time(end) / steps * 1e3))
    # two end, and two more begin in their pages
    server.release(i32([0, 3]))
    begin = server.new_step(96, 64, slots=i32([3, 0]))
    begin.ids.random_(0, vocabulary)
    begin.new.copy_(i32([32, 64]))
    first = server(begin)
    step.ids[[3, 0]] = first.top_tokens[:, 0]
    for _ in range(steps):
        graph.replay()
    print("held now: %s tokens, %d pages free" % (server.sessions.held.tolist(), server.sessions.free_count.item()))


if __name__ == "__main__":
    main()
