"""Performance cases of the attention operators over packed sequences and a paged cache.

A language model's hidden states are the rows that the detectors score; these operators
turn token sequences into such rows: the map of a paged key / value cache from request
lengths (``page_map``), the write of new keys and values into it (``page_write``),
attention over whole packed prompts (``prompt``) and attention of each request's newest
tokens over its pages (``paged``).

A case is a dict of plain values.  ``own`` picks the side: False computes the operators
from their definitions with elementary torch operations in 32 bits, True calls this
library.  Lengths are part of what a serving program knows, so a state holds them on the
host and on the GPU.
"""
import math

import torch

own = False

_DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # One decode step's bookkeeping: 48 requests, a new token each; latency.
        {"name": "map_step", "op": "page_map", "seqs": 48, "cached_lo": 1, "cached_hi": 6000,
         "fresh_lo": 1, "fresh_hi": 1, "idle": 0.0, "page": 16, "cols": 512},
        # A large mixed step: 2,000 requests, prompts, chunks and single tokens, some idle.
        {"name": "map_mixed", "op": "page_map", "seqs": 2000, "cached_lo": 0, "cached_hi": 9000,
         "fresh_lo": 1, "fresh_hi": 60, "idle": 0.1, "page": 16, "cols": 600},
        # The keys and values of one decode step.
        {"name": "write_step", "op": "page_write", "tokens": 48, "kv_heads": 8, "dim": 128,
         "dtype": "bf16", "page": 16, "pages": 4000, "missing": 0.0},
        # The keys and values of a batch of prompts, out of a fused projection's rows.
        {"name": "write_prompts", "op": "page_write", "tokens": 20011, "kv_heads": 8, "dim": 128,
         "dtype": "fp16", "page": 64, "pages": 500, "missing": 0.01},
        # A few short texts through an encoder (all tokens see each other); latency.
        {"name": "prompt_short", "op": "prompt", "seqs": 6, "length_lo": 1, "length_hi": 190,
         "heads": 12, "kv_heads": 12, "dim": 64, "causal": False, "dtype": "fp16"},
        # A packed batch of prompts of very different lengths.
        {"name": "prompt_pack", "op": "prompt", "seqs": 24, "length_lo": 1, "length_hi": 2500,
         "heads": 32, "kv_heads": 8, "dim": 128, "causal": True, "dtype": "bf16"},
        # One long document.
        {"name": "prompt_long", "op": "prompt", "seqs": 1, "length_lo": 16001,
         "length_hi": 16001, "heads": 32, "kv_heads": 8, "dim": 128, "causal": True,
         "dtype": "bf16"},
        # The next token of one request: latency.
        {"name": "token_one", "op": "paged", "seqs": 1, "cached_lo": 900, "cached_hi": 900,
         "fresh_lo": 1, "fresh_hi": 1, "chunks": 0, "chunk_lo": 1, "chunk_hi": 1, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 16, "dtype": "bf16"},
        # The next token of many requests of different lengths.
        {"name": "token_batch", "op": "paged", "seqs": 96, "cached_lo": 100, "cached_hi": 6000,
         "fresh_lo": 1, "fresh_hi": 1, "chunks": 0, "chunk_lo": 1, "chunk_hi": 1, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 16, "dtype": "bf16"},
        # The next token of few requests over very long caches.
        {"name": "token_long", "op": "paged", "seqs": 3, "cached_lo": 120000,
         "cached_hi": 131071, "fresh_lo": 1, "fresh_hi": 1, "chunks": 0, "chunk_lo": 1,
         "chunk_hi": 1, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "fp16"},
        # One chunk of a long document's prompt.
        {"name": "chunk_long", "op": "paged", "seqs": 1, "cached_lo": 60007, "cached_hi": 60007,
         "fresh_lo": 1, "fresh_hi": 1, "chunks": 1, "chunk_lo": 512, "chunk_hi": 512,
         "heads": 16, "kv_heads": 2, "dim": 128, "page": 32, "dtype": "fp16"},
        # A serving step that mixes single tokens with chunks of prompts.
        {"name": "step_mixed", "op": "paged", "seqs": 44, "cached_lo": 0, "cached_hi": 8000,
         "fresh_lo": 1, "fresh_hi": 1, "chunks": 4, "chunk_lo": 250, "chunk_hi": 700,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 16, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    """(query heads, key / value heads): shared by 1 to 8 query heads each."""
    kv = rng.choice([1, 2, 4, 8, 12])
    group = rng.choice([1, 2, 4, 6, 8]) if kv < 12 else 1
    return kv * group, kv


def draw(rng):
    op = rng.choice(["page_map", "page_write", "prompt", "prompt", "paged", "paged", "paged"])
    dtype = rng.choice(["fp16", "bf16"])
    page = rng.choice([8, 16, 32, 64, 128])
    if op == "page_map":
        cached, fresh = _log(rng, 10, 16000), _log(rng, 1, 250)
        return {"op": op, "seqs": _log(rng, 1, 2000), "cached_lo": 0, "cached_hi": cached,
                "fresh_lo": 1, "fresh_hi": fresh, "idle": rng.choice([0.0, 0.2]), "page": page,
                "cols": (cached + fresh) // page + rng.randint(1, 40)}
    heads, kv = _heads(rng)
    dim = rng.choice([64, 64, 128, 128, 128, 72, 80, 96, 256])
    if op == "page_write":
        tokens = _log(rng, 1, 20000)
        return {"op": op, "tokens": tokens, "kv_heads": kv, "dim": dim, "dtype": dtype,
                "page": page, "pages": tokens // page + rng.randint(1, 500),
                "missing": rng.choice([0.0, 0.05])}
    if op == "prompt":
        # No more products and no more query elements than the longest listed prompt.
        causal = rng.random() < 0.7
        cap = 16001 ** 2 * 32 * 128 // (heads * dim) // (1 if causal else 2)
        top = _log(rng, 2, min(16000, math.isqrt(cap)))
        seqs = max(1, min(_log(rng, 1, 64), 16001 * 32 * 128 // (heads * dim * top),
                          cap // top ** 2))
        return {"op": op, "seqs": seqs, "length_lo": rng.randint(1, max(1, top // 2)),
                "length_hi": top, "heads": heads, "kv_heads": kv, "dim": dim, "causal": causal,
                "dtype": dtype}
    # Cached tokens of all requests: 1 GiB of keys and values at most.
    rows = (1 << 30) // (4 * kv * dim)
    seqs = _log(rng, 1, 128)
    top = max(1, min(_log(rng, 16, 131000), rows // seqs))
    chunks = rng.choice([0, 0, 0, min(seqs, rng.randint(1, 4))])
    # Chunks of no more products than the longest listed prompt.
    chunk_top = max(2, min(_log(rng, 2, 1000), 16001 ** 2 * 16 * 128 // (heads * dim * top * 4)))
    return {"op": op, "seqs": seqs, "cached_lo": rng.randint(0, top), "cached_hi": top,
            "fresh_lo": 1, "fresh_hi": rng.choice([1, 1, 1, 4]), "chunks": chunks,
            "chunk_lo": rng.randint(1, chunk_top), "chunk_hi": chunk_top, "heads": heads,
            "kv_heads": kv, "dim": dim, "page": page, "dtype": dtype}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _between(case, what, n, part):
    """n lengths of [what_lo, what_hi], spread evenly over it (the same for every seed, so that
    work() can count them) in an order that mixes short and long."""
    lo, hi = case[what + "_lo"], case[what + "_hi"]
    vals = [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]
    step = next(s for s in (7, 11, 13, 17, 19, 23) if n % s or n == 1)
    return [vals[(i * step + part) % n] for i in range(n)]


def _lengths(case):
    """(cached, fresh) lengths of the case's requests."""
    n = case["seqs"]
    if case["op"] == "prompt":
        return [0] * n, _between(case, "length", n, 0)
    cached, fresh = _between(case, "cached", n, 0), _between(case, "fresh", n, 3)
    if case["op"] == "paged" and case["chunks"]:
        for i, c in enumerate(_between(case, "chunk", case["chunks"], 0)):
            fresh[i * (n // case["chunks"])] = c
    if case["op"] == "page_map" and case["idle"]:
        every = int(round(1.0 / case["idle"]))
        fresh = [0 if i % every == every - 1 else f for i, f in enumerate(fresh)]
    return cached, fresh


def _int(values, dev):
    return torch.tensor(values, dtype=torch.int32, device=dev)


def _starts(fresh):
    out = [0]
    for n in fresh:
        out.append(out[-1] + n)
    return out


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 1000003 + 29)
    op = case["op"]
    state = {"case": case}

    def normal(*shape, spread=1.0):
        return (spread * torch.randn(*shape, generator=g, device=dev)).to(_DTYPES[case["dtype"]])

    def perm(n):
        return torch.randperm(n, generator=g, device=dev)

    if op == "page_map":
        cached, fresh = _lengths(case)
        page, cols = case["page"], case["cols"]
        have = [-(-c // page) for c in cached]
        need = [-(-(c + f) // page) - h for c, f, h in zip(cached, fresh, have)]
        ids = perm(sum(have) + sum(need) + 64).to(torch.int32)
        table = torch.full((len(cached), cols), -1, dtype=torch.int32, device=dev)
        rows = torch.repeat_interleave(torch.arange(len(have), device=dev),
                                       torch.tensor(have, device=dev))
        first = torch.tensor(_starts(have)[:-1], device=dev)
        col = torch.arange(sum(have), device=dev) - first[rows]
        table[rows, col] = ids[:sum(have)]
        state.update(cached=_int(cached, dev), fresh=_int(fresh, dev), table=table,
                     free=ids[sum(have):].contiguous(), tokens=sum(fresh), max_fresh=max(fresh))
    elif op == "page_write":
        t, h, d = case["tokens"], case["kv_heads"], case["dim"]
        kv = normal(t, 2 * h, d)  # the projection's rows hold the keys, then the values
        slots = case["pages"] * case["page"]
        slot = perm(slots)[:t].contiguous()
        if case["missing"]:  # tokens that have no page
            slot[torch.rand(t, generator=g, device=dev) < case["missing"]] = -1
        shape = (case["pages"], h, case["page"], d)
        state.update(k=kv[:, :h], v=kv[:, h:], slot=slot, k_pages=normal(*shape),
                     v_pages=normal(*shape))
    else:
        cached, fresh = _lengths(case)
        t, hq, hk, d = sum(fresh), case["heads"], case["kv_heads"], case["dim"]
        state.update(row_start=_int(_starts(fresh), dev), cached_host=cached, fresh_host=fresh)
        if op == "prompt":  # slices of one fused projection
            qkv = normal(t, hq + 2 * hk, d)
            qkv[:, :hq] *= 1.5  # scores with a standard deviation of 1.5
            state.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hk], v=qkv[:, hq + hk:])
        else:
            page = case["page"]
            have = [-(-(c + f) // page) for c, f in zip(cached, fresh)]
            ids = perm(sum(have) + 8).to(torch.int32)
            table = torch.full((len(have), max(have) + 3), -1, dtype=torch.int32, device=dev)
            at = 0
            for r, n in enumerate(have):
                table[r, :n] = ids[at:at + n]
                at += n
            shape = (sum(have) + 8, hk, page, d)
            state.update(q=normal(t, hq, d, spread=1.5), k_pages=normal(*shape),
                         v_pages=normal(*shape), table=table, cached=_int(cached, dev),
                         max_fresh=max(fresh))
    if own:
        from paper_2110_14007_amd import tod
        state["tod"], state["ws"] = tod, tod.Workspace()
    return state


# ---------------------------------------------------------------------------
# the operators: this library's calls, and their plain forms in 32 bits
# ---------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if not own:
        return {"page_map": _map_plain, "page_write": _write_plain, "prompt": _prompt_plain,
                "paged": _paged_plain}[op](state)
    tod, s = state["tod"], state
    if op == "page_map":
        row_start, slot, pos, used = tod.tod_page_map(s["cached"], s["fresh"], s["free"],
                                                      s["table"], s["case"]["page"], s["tokens"])
        return row_start, slot, pos, used, s["table"]
    if op == "page_write":
        tod.tod_page_write(s["k"], s["v"], s["slot"], s["k_pages"], s["v_pages"])
        return s["k_pages"], s["v_pages"]
    if op == "prompt":
        return tod.tod_attn_prompt(s["q"], s["k"], s["v"], s["row_start"],
                                   causal=s["case"]["causal"], workspace=s["ws"],
                                   return_lse=True)
    return tod.tod_attn_paged(s["q"], s["k_pages"], s["v_pages"], s["table"], s["row_start"],
                              s["cached"], max_fresh=s["max_fresh"], workspace=s["ws"],
                              return_lse=True)


def _map_plain(s):
    page, cols, dev = s["case"]["page"], s["case"]["cols"], s["table"].device
    cached, fresh, free, table = s["cached"].long(), s["fresh"].long(), s["free"], s["table"]
    have = ((cached + page - 1) // page).clamp(max=cols)
    need = ((cached + fresh + page - 1) // page).clamp(max=cols) - have
    row_start = torch.nn.functional.pad(torch.cumsum(fresh, 0), (1, 0))
    base = torch.cumsum(need, 0) - need
    col = torch.arange(cols, device=dev)[None, :]
    new = (col >= have[:, None]) & (col < (have + need)[:, None])
    g = base[:, None] + col - have[:, None]
    ids = torch.where(g < free.numel(), free[g.clamp(0, free.numel() - 1)], -1)
    table.copy_(torch.where(new, ids, table))
    t = torch.arange(s["tokens"], device=dev)
    r = torch.searchsorted(row_start[1:], t, right=True).clamp(max=cached.numel() - 1)
    live = t < row_start[-1]
    pos = cached[r] + t - row_start[r]
    at = torch.where(pos // page < cols, table[r, (pos // page).clamp(max=cols - 1)], -1)
    slot = torch.where(live & (at >= 0), at.long() * page + pos % page, -1)
    pos = torch.where(live, pos, -1)
    used = torch.stack([need.sum(), fresh.sum() - (slot >= 0).sum()])
    return row_start.clamp(max=s["tokens"]).int(), slot, pos.int(), used, table


def _write_plain(s):
    page = s["case"]["page"]
    ok = s["slot"] >= 0
    slot = s["slot"][ok]
    s["k_pages"][slot // page, :, slot % page] = s["k"][ok]
    s["v_pages"][slot // page, :, slot % page] = s["v"][ok]
    return s["k_pages"], s["v_pages"]


def _attend(q, k, v, causal, out, lse):
    """softmax(q k^T / sqrt(d)) v of one sequence into out [n, hq, d] and lse [n, hq], the
    softmax's log sum: q [n, hq, d] are the newest of k's and v's [len, hk, d] tokens.  In
    blocks of query rows, so that the scores take 1 GiB at most."""
    n, hq, d = q.shape
    length, hk, _ = k.shape
    kt = k.float().permute(1, 2, 0).contiguous()
    vh = v.float().permute(1, 0, 2).contiguous()
    step = max(1, (1 << 28) // (hq * length))
    for b in range(0, n, step):
        e = min(n, b + step)
        seen = length - n + e if causal else length  # keys that some row of the block sees
        qh = q[b:e].float().reshape(e - b, hk, hq // hk, d).permute(1, 2, 0, 3)
        s = torch.matmul(qh.reshape(hk, -1, d).contiguous(), kt[:, :, :seen].contiguous())
        s = s.mul_(1.0 / math.sqrt(d)).view(hk, hq // hk, e - b, seen)
        if causal:
            row = torch.arange(length - n + b, length - n + e, device=q.device)
            col = torch.arange(seen, device=q.device)
            s = s.masked_fill_(col[None, :] > row[:, None], -math.inf)
        top = s.amax(3, keepdim=True)
        p = s.sub_(top).exp_()
        total = p.sum(3, keepdim=True)
        o = torch.matmul(p.view(hk, -1, seen), vh[:, :seen].contiguous())
        o = o.view(hk, hq // hk, e - b, d) / total
        out[b:e] = o.permute(2, 0, 1, 3).reshape(e - b, hq, d).to(out.dtype)
        lse[b:e] = (top + total.log()).squeeze(3).permute(2, 0, 1).reshape(e - b, hq)


def _prompt_plain(s):
    q = s["q"]
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    at = 0
    for n in s["fresh_host"]:
        r = slice(at, at + n)
        _attend(q[r], s["k"][r], s["v"][r], s["case"]["causal"], out[r], lse[r])
        at += n
    return out, lse


def _paged_plain(s):
    q, (hk, page, d) = s["q"], s["k_pages"].shape[1:]
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    at = 0
    for r, (c, n) in enumerate(zip(s["cached_host"], s["fresh_host"])):
        ids = s["table"][r, :-(-(c + n) // page)].long()
        k, v = (p[ids].transpose(1, 2).reshape(-1, hk, d)[:c + n]
                for p in (s["k_pages"], s["v_pages"]))
        _attend(q[at:at + n], k, v, True, out[at:at + n], lse[at:at + n])
        at += n
    return out, lse


def work(case):
    """Each input read once and each output written once; four operations per query head,
    visible (query, key) pair and element."""
    op = case["op"]
    if op == "page_write":
        return {"bytes": float(case["tokens"] * (8 + 8 * case["kv_heads"] * case["dim"])),
                "flops": 0.0}
    cached, fresh = _lengths(case)
    t = sum(fresh)
    if op == "page_map":
        page = case["page"]
        need = sum(-(-(c + f) // page) + -c // page for c, f in zip(cached, fresh))
        return {"bytes": float(12 * len(cached) + 12 * t + 8 * need), "flops": 0.0}
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    keys = sum(c + f for c, f in zip(cached, fresh))
    if op == "prompt" and not case["causal"]:
        pairs = sum(f * f for f in fresh)
    else:
        pairs = sum(f * c + f * (f + 1) // 2 for c, f in zip(cached, fresh))
    side = 4 * len(cached) + (4 * sum(-(-(c + f) // case["page"]) for c, f in zip(cached, fresh))
                              if op == "paged" else 0)
    return {"bytes": float(t * hq * (4 * d + 4) + 4 * keys * hk * d + side),
            "flops": 4.0 * pairs * hq * d}


# ---------------------------------------------------------------------------
# the same results in 64 bits, head by head
# ---------------------------------------------------------------------------

def _exact_head(q, k, v, first, causal):
    """(out [n, d], lse [n]) in fp64 of one head: query row i stands at position first + i."""
    n, d = q.shape
    outs, lses = [], []
    pos = torch.arange(k.shape[0], device=q.device)
    for b in range(0, n, max(1, (1 << 26) // k.shape[0])):
        rows = q[b:b + max(1, (1 << 26) // k.shape[0])].double()
        end = min(k.shape[0], first + b + rows.shape[0]) if causal else k.shape[0]
        s = rows @ k[:end].double().T / math.sqrt(d)
        if causal:
            at = first + b + torch.arange(rows.shape[0], device=q.device)
            s[pos[None, :end] > at[:, None]] = -math.inf
        z = torch.logsumexp(s, dim=1)
        outs.append(torch.exp(s - z[:, None]) @ v[:end].double())
        lses.append(z)
    return torch.cat(outs), torch.cat(lses)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "page_map":
        return None  # whole numbers
    if op == "page_write":  # copies: each token's row, head by head, at its slot
        pages = []
        for new, old in ((s["k"], s["k_pages"]), (s["v"], s["v_pages"])):
            flat = old.double()
            for h in range(case["kv_heads"]):
                rows = flat[:, h].reshape(-1, case["dim"])
                keep = torch.nonzero(s["slot"] >= 0).squeeze(1)
                rows.index_copy_(0, s["slot"][keep], new[keep, h].double())
                flat[:, h] = rows.view(-1, case["page"], case["dim"])
            pages.append(flat)
        return tuple(pages)
    group = case["heads"] // case["kv_heads"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=s["q"].device)
    at = 0
    for r, (c, n) in enumerate(zip(s["cached_host"], s["fresh_host"])):
        t = slice(at, at + n)
        if op == "paged":
            j = torch.arange(c + n, device=out.device)
            page_of, row_of = s["table"][r][j // case["page"]].long(), j % case["page"]
        for h in range(case["heads"]):
            if op == "prompt":
                k, v = s["k"][t, h // group], s["v"][t, h // group]
            else:
                k = s["k_pages"][page_of, h // group, row_of]
                v = s["v_pages"][page_of, h // group, row_of]
            out[t, h], lse[t, h] = _exact_head(s["q"][t, h], k, v, c,
                                               op == "paged" or case["causal"])
        at += n
    return out, lse
