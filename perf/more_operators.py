"""Timed cases of the operators around a cache of few bits and around what a decoder answers.

A case is one pass:
  op "append"      append_quantized: T new tokens of each of `seqs` sequences go into `pools` pools as they are quantised, behind up to
                   `held` tokens that the sequences have; what the pools then hold of them is read back, and the tokens are dropped again
  op "read"        read_quantized: `tokens` tokens of each sequence, from a place of its own on, out of `pools` pools
  op "attention"   quantized_attention: T new tokens of each of `batch` sequences over up to `keys` keys of its own in such pools
  op "logprobs"    token_logprobs: log probabilities of given tokens, entropies and the `top` likeliest tokens of rows of logits
  op "grad"        token_logprobs_grad: the gradient of the first two with respect to the logits

A cache row of a token holds, head after head, `bits` bits an element (e2m1 or e4m3), then an exponent byte for each block of 32
elements of a head: 2^(byte - 127) is the block's unit, the power of two under its largest magnitude over that under the format's largest.
Sizes: heads, head dimension and key counts as in this repository's other attention cases (32 heads of 128, 8192 keys), its
vocabularies of 32000 and 128256, and generic ones.  `own` chooses between the plain form and the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_BLOCK = 32       # elements with one exponent
_LOWEST = -117    # the least exponent


def _cache(name, op, seqs, held, tokens, page, pools, kv_heads, dim, bits, dtype):
    return dict(name=name, op=op, seqs=seqs, held=held, tokens=tokens, page=page, pools=pools, kv_heads=kv_heads, dim=dim, bits=bits, dtype=dtype)


def _attention(name, batch, tokens, heads, kv_heads, dim, keys, page, bits, dtype):
    return dict(name=name, op="attention", batch=batch, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, keys=keys, page=page, bits=bits, dtype=dtype)


def _logits(name, op, batch, tokens, vocab, top, dtype, pad=0, banned=0.0):
    return dict(name=name, op=op, batch=batch, tokens=tokens, vocab=vocab, top=top, dtype=dtype, pad=pad, banned=banned)


def listed():
    return [
        # Two sequences of a few hundred keys, one new token each: the latency of a call.
        _attention("attention_small", 2, 1, 8, 2, 64, 230, 16, 4, "bf16"),
        # The ordinary decoding step: 64 sequences of up to 8192 keys, 32 heads on 8 of keys and values.
        _attention("attention_step", 64, 1, 32, 8, 128, 8192, 16, 4, "bf16"),
        # Verification step of drafted tokens: five positions of each sequence, 8 bits an element, pages of an odd size.
        _attention("attention_drafts", 24, 5, 32, 4, 64, 5801, 24, 8, "f16"),
        # A further turn of two long conversations: 512 new tokens each over what is there, the most work of one call.
        _attention("attention_turn", 2, 512, 32, 8, 128, 16384, 32, 4, "bf16"),
        # Four sequences take a token each, one layer's two pools: launches and latency.
        _cache("append_small", "append", 4, 1000, 1, 16, 2, 2, 64, 4, "bf16"),
        # Two prompts of 4000 tokens go into all layers' pools.
        _cache("append_prompt", "append", 2, 40, 4000, 16, 24, 8, 128, 4, "bf16"),
        # A short piece of one sequence, in half precision.
        _cache("read_small", "read", 1, 300, 200, 16, 2, 2, 64, 4, "f16"),
        # Eight sequences whole, 8 bits an element, for a pass that wants them dense.
        _cache("read_large", "read", 8, 8192, 8192, 32, 2, 8, 128, 8, "bf16"),
        # One token's scores with the five likeliest, the smallest vocabulary in use.
        _logits("logprobs_one", "logprobs", 1, 1, 32000, 5, "f32"),
        # Scores of the drafts of a batch with the twenty likeliest, rows that lie apart by a padded stride.
        _logits("logprobs_batch", "logprobs", 64, 5, 128256, 20, "bf16", 64),
        # A few positions, a vocabulary of which a fifth is banned.
        _logits("grad_small", "grad", 2, 3, 32000, 0, "f32", 0, 0.2),
        # Samples of 512 tokens, scored for training.
        _logits("grad_batch", "grad", 8, 512, 32000, 0, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more pass: the same ranges, sizes spread over their logarithms, odd ones among them."""
    while True:
        op = rng.choice(("attention", "attention", "attention", "append", "read", "logprobs", "logprobs", "grad"))
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        shape = dict(page=rng.choice((8, 16, 16, 24, 32, 64)), kv_heads=rng.choice((1, 2, 4, 5, 8, 16)), dim=rng.choice((32, 64, 96, 128, 128, 192, 256)), bits=rng.choice((4, 4, 8)),
                     dtype=dtype)
        if op == "attention":
            case = dict(op=op, batch=_log_int(rng, 1, 64), tokens=rng.choice((1, 1, 1, 2, 3, 5, 16, _log_int(rng, 16, 512))), heads=shape["kv_heads"] * rng.choice((1, 2, 4, 5, 8)),
                        keys=_log_int(rng, 8, 131072), **shape)
            scores = case["batch"] * case["tokens"] * case["heads"] * case["keys"]
            # in single precision a product takes three
            if (work(case)["flops"] * (3 if dtype == "f32" else 1) > work(listed()[3])["flops"] or work(case)["bytes"] > work(listed()[1])["bytes"] or scores > 1 << 29
                    or case["batch"] * case["keys"] * case["kv_heads"] * case["dim"] > 1 << 29):
                continue
        elif op in ("append", "read"):
            tokens = _log_int(rng, 1, 8192)
            case = dict(op=op, seqs=_log_int(rng, 1, 64), held=_log_int(rng, 1, 2000) if op == "append" else tokens + _log_int(rng, 1, 2000), tokens=tokens, pools=2 * _log_int(rng, 1, 12), **shape)
            if work(case)["bytes"] > work(listed()[5])["bytes"] or case["pools"] * case["seqs"] * (case["held"] + tokens) * case["kv_heads"] * case["dim"] > 1 << 28:
                continue
        else:
            case = dict(op=op, batch=_log_int(rng, 1, 64), tokens=_log_int(rng, 1, 512), vocab=_log_int(rng, 1000, 160000), top=rng.choice((0, 1, 5, 20, 32)) if op == "logprobs" else 0,
                        dtype=dtype, pad=rng.choice((0, 0, 7, 64)), banned=rng.choice((0.0, 0.0, 0.2, 0.9)))
            if work(case)["bytes"] > work(listed()[9 if op == "logprobs" else 11])["bytes"]:
                continue
        return case


def _row_bytes(c):
    """Bytes of a token in a pool: codes and exponents, in whole 16 bytes."""
    return -(-c["kv_heads"] * (c["dim"] * c["bits"] // 8 + c["dim"] // _BLOCK) // 16) * 16


def work(c):
    es = _BYTES[c["dtype"]]
    if c["op"] == "attention":
        mean = max(0.75 * c["keys"], c["tokens"])
        cache = 2 * c["batch"] * mean * c["kv_heads"] * (c["dim"] * c["bits"] // 8 + c["dim"] // _BLOCK)
        io = c["batch"] * c["tokens"] * c["heads"] * (2 * c["dim"] * es + 4)
        return {"bytes": cache + io, "flops": 4.0 * c["dim"] * c["heads"] * c["tokens"] * c["batch"] * mean}
    if c["op"] in ("append", "read"):
        n = c["pools"] * c["seqs"] * c["tokens"]
        dense = c["kv_heads"] * c["dim"] * es
        # append: values in, a pool's bytes out, and those values out again; read: a pool's bytes in, values out
        return {"bytes": float(n * (_row_bytes(c) + dense * (2 if c["op"] == "append" else 1))), "flops": 2.0 * n * c["kv_heads"] * c["dim"]}
    rows = c["batch"] * c["tokens"]
    if c["op"] == "logprobs":
        return {"bytes": float(rows * (c["vocab"] * es + 16 + 8 * c["top"])), "flops": 5.0 * rows * c["vocab"]}
    return {"bytes": float(rows * (2 * c["vocab"] * es + 24)), "flops": 8.0 * rows * c["vocab"]}


# ------------------------------------------------------------------------------------------------------------ the format

def _power(e):
    """2^e of int32 exponents of normal numbers, exactly."""
    return ((e + 127) << 23).view(torch.float32)


def _grid(bits, device):
    """Magnitudes of the codes without sign."""
    mantissa, bias = (1, 1) if bits == 4 else (3, 7)
    code = torch.arange(8 if bits == 4 else 127, device=device)
    e, m = code >> mantissa, (code & ((1 << mantissa) - 1)).float() / (1 << mantissa)
    return torch.where(e == 0, m * 2.0 ** (1 - bias), (1 + m) * torch.exp2((e - bias).float()))


def _encode(x, bits):
    """Rows of a pool (..., _row_bytes) uint8 of values (..., heads, dim), in 32 bits."""
    heads, dim = x.shape[-2:]
    mantissa, least, top, largest = (1, 0, 2, 6.0) if bits == 4 else (3, -6, 8, 448.0)
    y = x.float().unflatten(-1, (dim // _BLOCK, _BLOCK))
    amax = y.abs().amax(-1)
    e = torch.where(amax > 0, torch.frexp(amax).exponent - 1 - top, _LOWEST).clamp(min=_LOWEST)
    y = y * _power(-e)[..., None]
    step = (torch.frexp(y.abs()).exponent - 1).clamp(min=least) - mantissa
    rounded = (torch.round(y * _power(-step)) * _power(step)).abs().clamp(max=largest)
    code = torch.searchsorted(_grid(bits, x.device), rounded, out_int32=True) | (torch.signbit(y).int() << (bits - 1))
    code = code.to(torch.uint8).flatten(-2)
    if bits == 4:
        code = code[..., 0::2] | (code[..., 1::2] << 4)
    row = torch.cat([code.flatten(-2), (e + 127).to(torch.uint8).flatten(-2)], -1)
    return torch.nn.functional.pad(row, (0, -row.shape[-1] % 16))


def _decode(rows, heads, dim, bits):
    """Values (..., heads, dim) in 32 bits of rows of a pool."""
    codes = heads * dim * bits // 8
    code = rows[..., :codes]
    if bits == 4:
        code = torch.stack([code & 15, code >> 4], -1).flatten(-2)
    grid = _grid(bits, rows.device)
    if bits == 8:
        grid = torch.cat([grid, torch.full((1,), math.nan, device=rows.device)])
    values = torch.cat([grid, -grid])[code.int()].unflatten(-1, (heads, dim // _BLOCK, _BLOCK))
    e = rows[..., codes:codes + heads * dim // _BLOCK].int() - 127
    return (values * _power(e).unflatten(-1, (heads, dim // _BLOCK))[..., None]).flatten(-2)


# ---------------------------------------------------------------------------------------------------------------- inputs

def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"attention": _prepare_attention, "append": _prepare_cache, "read": _prepare_cache, "logprobs": _prepare_logits, "grad": _prepare_logits}[c["op"]](c, g)


def _randint(g, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int64)


def _pools(c, g, pools, pages):
    """Pools as they are after values of the case's type went into them, a few million at a time."""
    out = torch.empty((pools, pages, c["page"], _row_bytes(c)), dtype=torch.uint8, device="cuda")
    flat = out.view(-1, _row_bytes(c))
    some = max(1, (1 << 25) // (c["kv_heads"] * c["dim"]))
    for i in range(0, flat.shape[0], some):
        n = min(some, flat.shape[0] - i)
        flat[i:i + n] = _encode(torch.randn((n, c["kv_heads"], c["dim"]), generator=g, device="cuda").to(_DTYPES[c["dtype"]]), c["bits"])
    return out


def _prepare_attention(c, g):
    B, T, ps, dt = c["batch"], c["tokens"], c["page"], _DTYPES[c["dtype"]]
    most = max(c["keys"], T)
    lens = torch.clamp(most - _randint(g, 0, most // 2 + 1, (B,)), min=T)
    M = -(-most // ps)
    table = torch.randperm(B * M, generator=g, device="cuda").reshape(B, M)
    k, v = _pools(c, g, 2, B * M)
    q = torch.randn((B, T, c["heads"], c["dim"]), generator=g, device="cuda").to(dt)
    return dict(op="attention", q=q, k=k, v=v, table=table.int(), lens=lens.int(), kv_heads=c["kv_heads"], bits=c["bits"], scale=c["dim"] ** -0.5)


def _prepare_cache(c, g):
    n, T, ps, P = c["seqs"], c["tokens"], c["page"], c["pools"]
    lens = torch.clamp(c["held"] - _randint(g, 0, ps, (n,)), min=T if c["op"] == "read" else 1)
    used = (lens + ps - 1) // ps
    M = -(-(c["held"] + T) // ps) + 1
    pages = n * M + 1
    ids = torch.randperm(pages, generator=g, device="cuda")
    table = torch.where(torch.arange(M, device="cuda")[None, :] < used[:, None], ids[:n * M].reshape(n, M), -1)
    refs = torch.zeros((pages,), dtype=torch.int64, device="cuda")
    refs[table[table >= 0]] = 1
    rest = torch.nonzero(refs == 0)[:, 0].flip(0)
    free = torch.full((pages,), -1, dtype=torch.int64, device="cuda")
    free[:rest.numel()] = rest
    ints = dict(page_table=table.int(), lens=lens.int(), refs=refs.int(), free_pages=free.int(), n_free=torch.tensor([rest.numel()], device="cuda").int())
    state = dict(op=c["op"], pools=_pools(c, g, P, pages) if c["op"] == "read" else torch.zeros((P, pages, ps, _row_bytes(c)), dtype=torch.uint8, device="cuda"),
                 seqs=torch.randperm(n, generator=g, device="cuda").int(), tokens=T, kv_heads=c["kv_heads"], dim=c["dim"], bits=c["bits"], dtype=_DTYPES[c["dtype"]])
    if c["op"] == "read":
        starts = _randint(g, 0, 1 << 30, (n,)) % (lens[state["seqs"].long()] - T + 1)
    else:
        starts = lens[state["seqs"].long()]
        state["values"] = torch.randn((P, n, T, c["kv_heads"], c["dim"]), generator=g, device="cuda").to(_DTYPES[c["dtype"]])
        state["drop"] = torch.full((n,), T, dtype=torch.int32, device="cuda")
    state["starts"] = starts.int()
    state["pool_list"], state["value_list"] = list(state["pools"]), list(state.get("values", ()))
    if own:
        import paper_2412_04358_amd as atk

        state["tables"] = atk.PageTables(page_size=ps, **ints)
    else:
        state["tables"] = dict(page=ps, **ints)
    return state


def _prepare_logits(c, g):
    B, T, V, dt = c["batch"], c["tokens"], c["vocab"], _DTYPES[c["dtype"]]
    logits = torch.zeros((B, T, V + c["pad"]), dtype=dt, device="cuda")[..., :V]
    logits.copy_(3 * torch.randn((B, T, V), generator=g, device="cuda"))
    tokens = _randint(g, 0, V, (B, T))
    if c["banned"]:
        logits.masked_fill_(torch.rand((B, T, V), generator=g, device="cuda") < c["banned"], -math.inf)
        logits.scatter_(2, tokens[..., None], torch.randn((B, T, 1), generator=g, device="cuda").to(dt))
    if T > 1:
        tokens[:, T - 1:] = torch.where(torch.rand((B, 1), generator=g, device="cuda") < 0.25, -1, tokens[:, T - 1:])   # some requests are a token shorter
    state = dict(op=c["op"], logits=logits, tokens=tokens.int(), top=c["top"])
    if c["op"] == "grad":
        lse = torch.logsumexp(logits.float(), -1)
        logp = logits.float() - lse[..., None]
        state |= dict(lse=lse, entropy=-torch.where(logp > -math.inf, torch.exp(logp) * logp, 0.0).sum(-1), grad_logprobs=torch.randn((B, T), generator=g, device="cuda"),
                      grad_entropy=0.01 * torch.randn((B, T), generator=g, device="cuda"))
    return state


# ------------------------------------------------------------------------------------------------------------------ passes

def run(s):
    return (_run_own if own else _run_plain)[s["op"]](s)


def _own_attention(s):
    import paper_2412_04358_amd as atk

    out, lse = atk.quantized_attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["kv_heads"], bits=s["bits"], scale=s["scale"], return_lse=True)
    return {"out": out, "lse": lse}


def _own_append(s):
    import paper_2412_04358_amd as atk

    t, pools = s["tables"], s["pool_list"]
    atk.append_quantized(t, pools, s["seqs"], s["value_list"], bits=s["bits"])
    values = atk.read_quantized(t, pools, s["seqs"], s["starts"], s["tokens"], s["kv_heads"], s["dim"], bits=s["bits"], dtype=s["dtype"])
    atk.free_sequences(t, s["seqs"], drop=s["drop"])
    return {"values": values, "page_table": t.page_table, "lens": t.lens, "refs": t.refs, "n_free": t.n_free}


def _own_read(s):
    import paper_2412_04358_amd as atk

    return {"values": atk.read_quantized(s["tables"], s["pool_list"], s["seqs"], s["starts"], s["tokens"], s["kv_heads"], s["dim"], bits=s["bits"], dtype=s["dtype"])}


def _own_logprobs(s):
    import paper_2412_04358_amd as atk

    logprobs, entropy, lse, top_logprobs, top_tokens = atk.token_logprobs(s["logits"], s["tokens"], top=s["top"])
    return {"logprobs": logprobs, "entropy": entropy, "lse": lse, "top_logprobs": top_logprobs, "top_tokens": top_tokens}


def _own_grad(s):
    import paper_2412_04358_amd as atk

    return {"grad": atk.token_logprobs_grad(s["logits"], s["tokens"], s["lse"], s["entropy"], s["grad_logprobs"], s["grad_entropy"])}


def _plain_attention(s):
    q, table, lens, Hk = s["q"], s["table"].long(), s["lens"].long(), s["kv_heads"]
    B, T, H, D = q.shape
    G, n = H // Hk, table.shape[1] * s["k"].shape[1]
    k = _decode(s["k"][table], Hk, D, s["bits"]).reshape(B, n, Hk, D).permute(0, 2, 3, 1).contiguous()
    rows = q.float().reshape(B, T, Hk, G, D).transpose(1, 2).reshape(B, Hk, T * G, D)
    scores = torch.matmul(rows, k).reshape(B, Hk, T, G, n) * s["scale"]
    del k
    limit = lens[:, None] - (T - 1) + torch.arange(T, device=q.device)[None, :]
    hidden = torch.arange(n, device=q.device) >= limit[:, None, :, None, None]
    scores = scores.masked_fill_(hidden, -math.inf).reshape(B, Hk, T * G, n)
    m = scores.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), 0.0, m)
    w = torch.exp(scores - m)
    total = w.sum(-1, keepdim=True)
    v = _decode(s["v"][table], Hk, D, s["bits"]).reshape(B, n, Hk, D).transpose(1, 2).contiguous()
    out = torch.matmul(w, v) / torch.where(total > 0, total, 1.0)
    lse = (m + torch.log(total))[..., 0]
    return {"out": out.reshape(B, Hk, T, G, D).transpose(1, 2).reshape(B, T, H, D).to(q.dtype), "lse": lse.reshape(B, Hk, T, G).transpose(1, 2).reshape(B, T, H)}


def _places(s, rows):
    """Page and place of the tokens from `starts` on, in rows of the table."""
    at = s["starts"].long()[:, None] + torch.arange(s["tokens"], device=rows.device)[None, :]
    ps = s["tables"]["page"]
    return rows.gather(1, at // ps).long(), at % ps


def _plain_append(s):
    t, seqs, T = s["tables"], s["seqs"].long(), s["tokens"]
    ps, rows, lens = t["page"], t["page_table"][seqs], t["lens"][seqs].long()
    used, after = (lens + ps - 1) // ps, (lens + T + ps - 1) // ps
    takes = after - used
    first = t["n_free"].long() - 1 - (torch.cumsum(takes, 0) - takes)
    place = torch.arange(rows.shape[1], device=rows.device)[None, :]
    fresh = t["free_pages"][(first[:, None] - (place - used[:, None])).clamp(0, t["free_pages"].numel() - 1)]
    rows = torch.where((place >= used[:, None]) & (place < after[:, None]), fresh, rows)
    page, slot = _places(s, rows)
    s["pools"][:, page, slot] = _encode(s["values"], s["bits"])
    values = _decode(s["pools"][:, page, slot], s["kv_heads"], s["dim"], s["bits"]).to(s["dtype"])
    # the new tokens are dropped again: the tables are what they were
    return {"values": list(values), "page_table": t["page_table"], "lens": t["lens"], "refs": t["refs"], "n_free": t["n_free"]}


def _plain_read(s):
    page, slot = _places(s, s["tables"]["page_table"][s["seqs"].long()])
    return {"values": list(_decode(s["pools"][:, page, slot], s["kv_heads"], s["dim"], s["bits"]).to(s["dtype"]))}


def _chosen(tokens, vocab):
    """Where a token is one, and a number that can be looked up."""
    return (tokens >= 0) & (tokens < vocab), tokens.long().clamp(0, vocab - 1)


def _plain_logprobs(s):
    x, V = s["logits"].float(), s["logits"].shape[-1]
    m = x.amax(-1, keepdim=True)
    lse = m + torch.log(torch.exp(x - m).sum(-1, keepdim=True))
    logp = x - lse
    entropy = -torch.where(logp > -math.inf, torch.exp(logp) * logp, 0.0).sum(-1)
    there, token = _chosen(s["tokens"], V)
    logprobs = torch.where(there, logp.gather(2, token[..., None])[..., 0], -math.inf)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :s["top"]]
    return {"logprobs": logprobs, "entropy": entropy, "lse": lse[..., 0], "top_logprobs": logp.gather(2, order), "top_tokens": order.int()}


def _plain_grad(s):
    logits = s["logits"]
    logp = logits.float() - s["lse"][..., None]
    p = torch.exp(logp)
    there, token = _chosen(s["tokens"], logits.shape[-1])
    given = s["grad_logprobs"][..., None]
    # d logp[token] / dx = [token] - p; d entropy / dx = -p (log p + entropy)
    grad = -p * torch.where(there[..., None], given, 0.0)
    grad -= s["grad_entropy"][..., None] * torch.where(logp > -math.inf, p * (logp + s["entropy"][..., None]), 0.0)
    grad.scatter_add_(2, token[..., None], torch.where(there[..., None], given, 0.0))
    return {"grad": grad.to(logits.dtype)}


_run_own = {"attention": _own_attention, "append": _own_append, "read": _own_read, "logprobs": _own_logprobs, "grad": _own_grad}
_run_plain = {"attention": _plain_attention, "append": _plain_append, "read": _plain_read, "logprobs": _plain_logprobs, "grad": _plain_grad}


# --------------------------------------------------------------------------------------------------- definitions in 64 bits

def exact(c, seed):
    """What a pass returns, from the definition in 64 bits."""
    s = prepare(c, seed)
    return {"attention": _exact_attention, "append": _exact_append, "read": _exact_read, "logprobs": _exact_logprobs, "grad": _exact_grad}[c["op"]](s)


def _ladder(bits):
    """Every magnitude of a format in order, as Python numbers."""
    if bits == 4:
        return [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    small = [m / 512 for m in range(8)]
    return small + [(8 + m) / 8 * 2.0 ** e for e in range(-6, 9) for m in range(8) if (e, m) != (8, 7)]


def _exact_values(rows, heads, dim, bits):
    """(tokens, heads, dim) of a pool's rows (tokens, bytes)."""
    rows = rows.long()
    each, blocks = dim * bits // 8, dim // 32
    code = rows[:, :heads * each].reshape(-1, heads, each)
    if bits == 4:
        code = torch.stack([code % 16, code // 16], -1).reshape(-1, heads, dim)
    ladder = _ladder(bits)
    steps = torch.tensor(ladder, dtype=torch.float64, device=rows.device)
    half = 1 << (bits - 1)
    x = torch.where(code >= half, -1.0, 1.0).double() * steps[(code % half).clamp(max=len(ladder) - 1)]
    unit = rows[:, heads * each:heads * (each + blocks)].reshape(-1, heads, blocks)
    return x * torch.pow(torch.tensor(2.0, dtype=torch.float64, device=rows.device), (unit - 127).double()).repeat_interleave(32, 2)


def _exact_attention(s):
    q, heads_of = s["q"], s["q"].shape[2] // s["kv_heads"]
    B, T, H, D = q.shape
    out = torch.zeros((B, T, H, D), dtype=torch.float64, device=q.device)
    lse = torch.full((B, T, H), -math.inf, dtype=torch.float64, device=q.device)
    ps = s["k"].shape[1]
    for b in range(B):
        n = int(s["lens"][b])
        at = torch.arange(n, device=q.device)
        page = s["table"][b].long()[at // ps]
        keys, values = (_exact_values(pool[page, at % ps], s["kv_heads"], D, s["bits"]) for pool in (s["k"], s["v"]))
        seen = at[None, :] <= (n - T + torch.arange(T, device=q.device))[:, None]
        for h in range(H):
            z = s["scale"] * torch.mm(q[b, :, h].double(), keys[:, h // heads_of].t())
            z = torch.where(seen, z, -math.inf)
            lse[b, :, h] = torch.logsumexp(z, -1)
            out[b, :, h] = torch.mm(torch.softmax(z, -1), values[:, h // heads_of])
    return {"out": out, "lse": lse}


def _exact_append(s):
    ladder = _ladder(s["bits"])
    top = 2 if s["bits"] == 4 else 8
    steps = torch.tensor(ladder, dtype=torch.float64, device="cuda")
    middle = (steps[1:] + steps[:-1]) / 2
    even = torch.arange(middle.numel(), device="cuda") % 2 == 0          # a middle goes down to an even code
    values = []
    for x in s["values"]:
        y = x.double().reshape(-1, 32)
        e = torch.floor(torch.log2(y.abs().amax(1, keepdim=True)))
        unit = torch.pow(torch.tensor(2.0, dtype=torch.float64, device="cuda"), e - top)
        z = y.abs() / unit
        code = torch.bucketize(z, middle, right=False)                   # middles below z
        tie = (code < middle.numel()) & (z == middle[code.clamp(max=middle.numel() - 1)])
        code = code + (tie & ~even[code.clamp(max=middle.numel() - 1)]).long()
        values.append((torch.where(y < 0, -1.0, 1.0) * steps[code] * unit).reshape(x.shape))
    return {"values": values, "page_table": None, "lens": None, "refs": None, "n_free": None}


def _exact_read(s):
    get = s["tables"].__getitem__ if isinstance(s["tables"], dict) else lambda k: getattr(s["tables"], k)
    table = get("page_table")
    ps = s["pools"].shape[2]
    values = []
    for pool in s["pools"]:
        rows = []
        for i in range(s["starts"].shape[0]):
            at = torch.arange(s["tokens"], device="cuda") + int(s["starts"][i])
            rows.append(_exact_values(pool[table[int(s["seqs"][i])].long()[at // ps], at % ps], s["kv_heads"], s["dim"], s["bits"]))
        values.append(torch.stack(rows))
    return {"values": values}


def _exact_logprobs(s):
    B, T, V = s["logits"].shape
    x = s["logits"].double().reshape(B * T, V)
    logp = torch.log_softmax(x, -1)
    p = torch.exp(logp)
    entropy = -(torch.xlogy(p, p)).sum(-1)
    tokens = s["tokens"].reshape(-1).long()
    logprobs = torch.tensor([float(logp[i, t]) if 0 <= t < V else -math.inf for i, t in enumerate(tokens.tolist())], dtype=torch.float64)
    # by value, then by number: a sort by number first, and a stable one by value behind it
    best = torch.argsort(-x, dim=-1, stable=True)[:, :s["top"]]
    return {"logprobs": logprobs.reshape(B, T), "entropy": entropy.reshape(B, T), "lse": torch.logsumexp(x, -1).reshape(B, T),
            "top_logprobs": logp.gather(1, best).reshape(B, T, -1), "top_tokens": best.int().reshape(B, T, -1)}


def _exact_grad(s):
    B, T, V = s["logits"].shape
    grad = torch.empty((B, T, V), dtype=torch.float64, device="cuda")
    at = torch.arange(V, device="cuda")
    for b in range(B):
        logp = s["logits"][b].double() - s["lse"][b].double()[:, None]
        p = torch.exp(logp)
        hit = (at[None, :] == s["tokens"][b].long()[:, None]).double()
        real = ((s["tokens"][b] >= 0) & (s["tokens"][b] < V)).double()[:, None]
        grad[b] = s["grad_logprobs"][b].double()[:, None] * (hit - p * real) - s["grad_entropy"][b].double()[:, None] * (torch.xlogy(p, p) + p * s["entropy"][b].double()[:, None])
    return {"grad": grad}
