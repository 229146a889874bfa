"""The two ends of a serving step, as cases that can be timed and checked.

Three pieces of work, each through the calls that a serving program makes:
  plan      page tables, lengths and the place of every token row of a step, made on the GPU from how much each session holds and how many
            tokens it brings; pages come from a stack of free ones
  product   the output head, or a layer too sensitive for 4 bits: int8 codes with a scale a token times int8 weights with a scale a channel
  logprobs  of the logits: log probabilities of given tokens, entropies, the likeliest alternatives

Layer sizes are those of this repository's benchmark and tests (hidden 4096, 5120, 8192; 13824 and 28672 channels); vocabularies are generic.
"""
import collections
import math

import torch

own = False

# what a program keeps of its sessions, and what a step is given of them
Sessions = collections.namedtuple("Sessions", "pages held free free_count")


# ---- the cases ----------------------------------------------------------------------------------------------------------------------

def _product(name, M, N, K, out):
    return dict(name=name, op="product", M=M, N=N, K=K, out=out)


def _logprobs(name, M, V, dtype, top, masked=0, pad=0):
    """masked: columns at the end that hold -infinity; pad: values between the rows."""
    return dict(name=name, op="logprobs", M=M, V=V, dtype=dtype, top=top, masked=masked, pad=pad)


def _plan(name, B, sessions, new_lo, new_hi, held_lo, held_hi, page, spare_rows=0):
    """B of the sessions bring tokens; spare_rows: rows of the step's tensors that belong to no sequence."""
    return dict(name=name, op="plan", B=B, sessions=sessions, new_lo=new_lo, new_hi=new_hi, held_lo=held_lo, held_hi=held_hi, page=page,
                spare_rows=spare_rows)


def listed():
    return [
        # the output head of one interactive session: every weight is read for one row
        _product("product_m1_n32000_k4096", 1, 32000, 4096, "fp16"),
        # 48 sessions, a vocabulary of odd size, logits in 32 bits
        _product("product_m48_n50001_k5120", 48, 50001, 5120, "fp32"),
        # a piece of a prompt through a projection kept in 8 bits
        _product("product_m333_n13824_k5120", 333, 13824, 5120, "fp16"),
        # a long prompt through the widest layer
        _product("product_m4096_n28672_k8192", 4096, 28672, 8192, "fp16"),
        # one session's next token with its alternatives: latency
        _logprobs("logprobs_m1_v32000_top20", 1, 32000, "fp16", 20),
        # 48 sessions, logits in 32 bits as the head above gives them
        _logprobs("logprobs_m48_v50001_top5", 48, 50001, "fp32", 5),
        # a prompt is scored: log probabilities only, a vocabulary that was padded to a rounder size
        _logprobs("logprobs_m777_v65600_scored", 777, 65600, "fp16", 0, masked=63),
        # many prompts are scored, with the choice that greedy decoding would have made
        _logprobs("logprobs_m4096_v128000_top1", 4096, 128000, "fp16", 1),
        # one session takes a token
        _plan("plan_step_b1", 1, 8, 1, 1, 500, 500, 64),
        # 64 of 100 sessions take a token each
        _plan("plan_step_b64", 64, 100, 1, 1, 17, 8000, 64),
        # ragged prompts, small pages, a few rows to spare
        _plan("plan_prompts_b37", 37, 37, 1, 3000, 0, 40, 16, spare_rows=13),
        # as many long sessions as the cache of a large GPU holds take up to four tokens each
        _plan("plan_step_b2048", 2048, 2500, 1, 4, 1000, 32000, 16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["product", "product", "logprobs", "logprobs", "plan"])
    if op == "product":
        K = 128 * _log_int(rng, 2, 90)                        # 256 .. 11520
        N = _log_int(rng, 40, 60000)
        if rng.random() < 0.5:
            N = max(16, N // 16 * 16)
        return dict(op=op, M=max(1, min(_log_int(rng, 1, 4096), 900_000_000_000 // (N * K))), N=N, K=K, out=rng.choice(["fp16", "fp16", "fp32"]))
    if op == "logprobs":
        V, top, dtype = _log_int(rng, 70, 150_000), rng.choice([0, 1, 3, 20, 64]), rng.choice(["fp16", "fp16", "fp32"])
        most = (400_000_000 if dtype == "fp16" else 200_000_000) // (1 + top // 4)
        return dict(op=op, M=max(1, min(_log_int(rng, 1, 8000), most // V)), V=V, dtype=dtype, top=top, masked=rng.choice([0, V // 100]),
                    pad=rng.choice([0, 0, 1, 24]))
    B = _log_int(rng, 1, 1500)
    held_hi = min(_log_int(rng, 1, 60_000), 30_000_000 // B)
    new_hi = rng.choice([1, 1, 3, min(_log_int(rng, 2, 4000), max(2, 500_000 // B))])
    return dict(op=op, B=B, sessions=B + rng.choice([0, 0, B // 3 + 1]), new_lo=rng.choice([0, 1, new_hi]), new_hi=new_hi,
                held_lo=held_hi // rng.choice([1, 3, 100]), held_hi=held_hi, page=rng.choice([16, 32, 64, 64]), spare_rows=rng.choice([0, 0, 100]))


def _spread(lo, hi, n, turn):
    """n whole numbers from lo to hi, the largest among them, in no order."""
    return [hi if i == n // 2 else lo + int((hi - lo + 1) * ((i * 0.6180339887498949 + turn) % 1.0)) for i in range(n)]


def _lengths(case):
    """(new tokens, tokens held before them) of each sequence of the step."""
    return _spread(case["new_lo"], case["new_hi"], case["B"], 0.3), _spread(case["held_lo"], case["held_hi"], case["B"], 0.7)


def work(case):
    if case["op"] == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": N * K + M * K + 4 * (M + N) + M * N * (2 if case["out"] == "fp16" else 4), "flops": 2 * M * N * K}
    if case["op"] == "logprobs":
        M, V = case["M"], case["V"]
        return {"bytes": M * V * (2 if case["dtype"] == "fp16" else 4) + M * (16 + 8 * case["top"]), "flops": 6 * M * V}
    new, held = _lengths(case)
    P = case["page"]
    closed = sum((n + h) // P for n, h in zip(new, held))
    fresh = closed - sum(h // P for h in held)
    # lengths and numbers of the sequences, two numbers a row, table entries read and written, fresh pages written to both tables
    return {"bytes": 24 * case["B"] + 8 * sum(new) + 8 * closed + 4 * fresh, "flops": 4 * case["B"] + 2 * sum(new) + closed}


# ---- inputs -------------------------------------------------------------------------------------------------------------------------

def _codes(gen, rows, cols, scale):
    """int8 codes of normal rows, the largest near 127, and their scales."""
    codes = torch.empty(rows, cols, dtype=torch.int8, device="cuda")
    step = max(1, (1 << 26) // cols)
    for at in range(0, rows, step):
        n = min(step, rows - at)
        codes[at:at + n] = (32.0 * torch.randn(n, cols, generator=gen, device="cuda")).round_().clamp_(-127, 127).to(torch.int8)
    return codes, scale * (0.5 + torch.rand(rows, generator=gen, device="cuda"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "product":
        M, N, K = case["M"], case["N"], case["K"]
        a_q, s_a = _codes(gen, M, K, 0.03)
        w_q, s_w = _codes(gen, N, K, 0.03 / math.sqrt(K))
        st = dict(case=case, a_q=a_q, s_a=s_a, w_q=w_q, s_w=s_w,
                  y=torch.empty(M, N, dtype=torch.float16 if case["out"] == "fp16" else torch.float32, device="cuda"))
        if own:
            from paper_2406_09904_amd import binding as qqq
            st["w_packed"], st["workspace"] = qqq.qqq_pack_w8(w_q), qqq.new_w8a8_workspace(M, N, K)
        return st
    if case["op"] == "logprobs":
        M, V, k = case["M"], case["V"], case["top"]
        dtype = torch.float16 if case["dtype"] == "fp16" else torch.float32
        wide = torch.zeros(M, V + case["pad"], dtype=dtype, device="cuda")
        step = max(1, (1 << 26) // V)
        for at in range(0, M, step):
            n = min(step, M - at)
            x = 2.5 * torch.randn(n, V, generator=gen, device="cuda")
            # a handful of likely tokens in every row, more or less so
            likely = (torch.randint(0, V, (n, 1), generator=gen, device="cuda") + torch.arange(5, device="cuda") * (V // 7)) % V
            x.scatter_(1, likely, 6.0 + 10.0 * torch.rand(n, 5, generator=gen, device="cuda"))
            wide[at:at + n, :V] = x
        logits = wide[:, :V]
        if case["masked"]:
            logits[:, V - case["masked"]:] = -math.inf
        tokens = torch.randint(0, V - case["masked"], (M,), generator=gen, device="cuda").int()
        if M > 1:
            tokens[-1] = -1                                   # behind a prompt's last row nothing is given
        f32 = lambda *s: torch.empty(*s, dtype=torch.float32, device="cuda")  # noqa: E731
        return dict(case=case, logits=logits, tokens=tokens, logprob=f32(M), entropy=f32(M), lse=f32(M),
                    top_tokens=torch.empty(M, k, dtype=torch.int32, device="cuda"), top_logprobs=f32(M, k))

    B, S, P = case["B"], case["sessions"], case["page"]
    new, held = _lengths(case)
    max_len = max(n + h for n, h in zip(new, held))
    columns = max(1, max_len // P)
    ids = torch.randperm(S, generator=gen, device="cuda").int()[:B].contiguous()
    all_held = torch.randint(0, max_len + 1, (S,), generator=gen, device="cuda").int()
    all_held[ids.long()] = torch.tensor(held, dtype=torch.int32, device="cuda")
    # pages in no order, as they are after some hours of serving
    has = (all_held // P).long()
    spare = sum((n + h) // P - h // P for n, h in zip(new, held)) + 50
    total = int(has.sum()) + spare
    order = torch.randperm(total, generator=gen, device="cuda").int()
    first = torch.cumsum(has, 0) - has
    nth = torch.arange(columns, device="cuda")[None, :]
    pages = torch.where(nth < has[:, None], order[(first[:, None] + nth).clamp(max=total - 1)], 0).int().contiguous()
    free = torch.zeros(total, dtype=torch.int32, device="cuda")
    free[:spare] = order[total - spare:]
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    rows = sum(new) + case["spare_rows"]
    # the numbers after the step go to places of their own, so that a pass can be repeated
    return dict(case=case, sessions=Sessions(pages, all_held, free, torch.tensor([spare], dtype=torch.int32, device="cuda")), ids=ids,
                new=torch.tensor(new, dtype=torch.int32, device="cuda"), max_new=max(new), max_len=max_len, held_after=all_held.clone(),
                free_after=i32(1), page_table=i32(B, columns), kv_len=i32(B), cu=i32(B + 1), sequence=i32(rows), positions=i32(rows), lacking=i32(1))


# ---- one pass -----------------------------------------------------------------------------------------------------------------------

def run(st):
    case = st["case"]
    if not own:
        return {"product": _plain_product, "logprobs": _plain_logprobs, "plan": _plain_plan}[case["op"]](st)
    from paper_2406_09904_amd import binding as qqq
    if case["op"] == "product":
        return {"y": qqq.qqq_gemm_w8a8(st["a_q"], st["s_a"], st["w_packed"], st["s_w"], st["workspace"], y=st["y"])}
    if case["op"] == "logprobs":
        out = qqq.qqq_logprobs(st["logits"], st["tokens"], case["top"], out=qqq.LogProbs(st["logprob"], st["entropy"], st["lse"], st["top_tokens"], st["top_logprobs"]))
        return {"logprob": out.logprob, "entropy": out.entropy, "lse": out.lse, "top_tokens": out.top_tokens, "top_logprobs": out.top_logprobs}
    sessions = qqq.KV8Sessions(*st["sessions"])
    batch = qqq.KV8Batch(st["page_table"], st["kv_len"], st["cu"], st["ids"], st["max_new"], st["max_len"])
    qqq.qqq_kv8_plan(sessions, batch, st["new"], case["page"], st["sequence"], st["positions"], st["lacking"], after=(st["held_after"], st["free_after"]))
    return _plan_outputs(st)


def _plan_outputs(st):
    return {"page_table": st["page_table"], "kv_len": st["kv_len"], "cu": st["cu"], "sequence": st["sequence"], "positions": st["positions"],
            "pages": st["sessions"].pages, "held": st["held_after"], "free_count": st["free_after"], "lacking": st["lacking"]}


def _plain_product(st):
    acc = torch.matmul(st["a_q"].float(), st["w_q"].float().t())
    st["y"].copy_(acc * st["s_a"][:, None] * st["s_w"][None, :])
    return {"y": st["y"]}


def _plain_logprobs(st):
    x, k = st["logits"].float(), st["case"]["top"]
    V = x.shape[1]
    m = x.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    t = x - m
    e = t.exp()
    z = e.sum(1, keepdim=True)
    log_z = z.log()
    st["lse"].copy_((m + log_z)[:, 0])
    st["entropy"].copy_((log_z - torch.where(e == 0, 0.0, e * t).sum(1, keepdim=True) / z)[:, 0])
    given = st["tokens"].long()
    own_t = t.gather(1, given.clamp(min=0)[:, None])
    st["logprob"].copy_(torch.where(given[:, None] < 0, 0.0, own_t - log_z)[:, 0])
    column = torch.arange(V, device="cuda")[None, :]
    left = torch.ones_like(t, dtype=torch.bool) if k else None
    for i in range(k):                                        # the largest of those left, the first of equal ones
        best = torch.where(left, t, -math.inf).amax(1, keepdim=True)
        at = torch.where(left & (t == best), column, V).amin(1, keepdim=True)
        st["top_tokens"][:, i] = at[:, 0].int()
        st["top_logprobs"][:, i] = (best - log_z)[:, 0]
        left.scatter_(1, at, False)
    return {"logprob": st["logprob"], "entropy": st["entropy"], "lse": st["lse"], "top_tokens": st["top_tokens"], "top_logprobs": st["top_logprobs"]}


def _plain_plan(st):
    s, P, ids, new = st["sessions"], st["case"]["page"], st["ids"].long(), st["new"].long()
    held = s.held.long()[ids]
    length = held + new
    ends = torch.cumsum(new, 0)
    st["kv_len"].copy_(length)
    st["cu"][0] = 0
    st["cu"][1:] = ends
    # fresh pages come from the stack's top, the first sequence's first
    need = length // P - held // P
    before = torch.cumsum(need, 0) - need
    columns = st["page_table"].shape[1]
    column = torch.arange(columns, device="cuda")[None, :]
    nth = column - (held // P)[:, None]
    fresh, kept = (nth >= 0) & (nth < need[:, None]), nth < 0
    count = s.free_count.long()
    place = count - 1 - before[:, None] - nth
    page = torch.where(place >= 0, s.free.long()[place.clamp(min=0, max=s.free.shape[0] - 1)], -1)
    table = s.pages[ids, :columns].long()
    s.pages[ids, :columns] = torch.where(fresh, page, table).int()
    st["page_table"].copy_(torch.where(fresh, page, torch.where(kept, table, st["page_table"].long())))
    row = torch.arange(st["sequence"].shape[0], device="cuda")
    seq = (row[:, None] >= ends[None, :]).sum(1) if row.numel() * ends.numel() <= 1 << 22 else torch.searchsorted(ends, row, right=True)
    of = seq.clamp(max=ends.shape[0] - 1)
    used = row < ends[-1]
    st["sequence"].copy_(torch.where(used, seq, st["sequence"].long()))
    st["positions"].copy_(torch.where(used, length[of] - ends[of] + row, st["positions"].long()))
    st["held_after"].copy_(s.held)
    st["held_after"][ids] = length.int()
    wanted = need.sum()
    st["free_after"].copy_((count - wanted).clamp(min=0))
    st["lacking"].copy_((wanted - count).clamp(min=0))
    return _plan_outputs(st)


# ---- what run() returns, from the definitions in 64 bits ----------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    f8 = torch.float64
    if case["op"] == "product":
        a = st["a_q"].to(f8) * st["s_a"].to(f8)[:, None]
        y = torch.empty(case["M"], case["N"], dtype=f8, device="cuda")
        for n in range(0, case["N"], 8192):
            y[:, n:n + 8192] = a @ (st["w_q"][n:n + 8192].to(f8) * st["s_w"][n:n + 8192].to(f8)[:, None]).t()
        return {"y": y}
    if case["op"] == "logprobs":
        M, V, k = case["M"], case["V"], case["top"]
        outs = collections.defaultdict(list)
        for rows in torch.arange(M, device="cuda").split(max(1, (1 << 26) // V)):
            x = st["logits"][rows].to(f8)
            lse = torch.logsumexp(x, 1)
            p = torch.softmax(x, 1)
            outs["lse"].append(lse)
            outs["entropy"].append(torch.special.entr(p).sum(1))
            given = st["tokens"][rows].long()
            outs["logprob"].append(torch.where(given < 0, 0.0, x[torch.arange(len(rows), device="cuda"), given.clamp(min=0)] - lse))
            values, at = torch.sort(x, dim=1, descending=True, stable=True) if k else (x, x)
            outs["top_tokens"].append(at[:, :k].int())
            outs["top_logprobs"].append(values[:, :k] - lse[:, None])
        return {n: torch.cat(outs[n]) for n in ("logprob", "entropy", "lse", "top_tokens", "top_logprobs")}
    P, new, held = case["page"], *_lengths(case)
    ids, free, count = st["ids"].tolist(), st["sessions"].free.tolist(), int(st["sessions"].free_count)
    pages, table = st["sessions"].pages.cpu().numpy(), st["page_table"].cpu().numpy()
    after, sequence, positions, cu = st["sessions"].held.tolist(), st["sequence"].tolist(), st["positions"].tolist(), [0]
    for b, (n, h) in enumerate(zip(new, held)):
        for j in range(h // P, (h + n) // P):
            count -= 1
            pages[ids[b], j] = free[count]
        closed = (h + n) // P
        table[b, :closed] = pages[ids[b], :closed]
        sequence[cu[-1]:cu[-1] + n] = [b] * n
        positions[cu[-1]:cu[-1] + n] = range(h, h + n)
        cu.append(cu[-1] + n)
        after[ids[b]] = h + n
    i32 = lambda a: torch.as_tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"page_table": i32(table), "kv_len": i32([n + h for n, h in zip(new, held)]), "cu": i32(cu), "sequence": i32(sequence), "positions": i32(positions),
            "pages": i32(pages), "held": i32(after), "free_count": i32([count]), "lacking": i32([0])}
