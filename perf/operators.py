"""Timed cases of the decoding operators: attention over a shared prefix, verification of drafted tokens, and a cache's pages.

A case is one pass of what a decoder of many samples of one prompt does:
  op "attention"   shared_prefix_attention: T new tokens of each of B sequences over a paged cache whose first `prefix` tokens
                   are the same pages for all of them, and up to `own` tokens of each sequence's own (the T new ones included)
  op "verify"      verify_drafts: up to `drafts` drafted tokens of each of B requests against rows of `vocab` probabilities
  op "samples"     fork_sequences, append_tokens, free_sequences: `prompts` sequences are forked to `samples` children each, every
                   child takes `tokens` new tokens, gives half of them back as rejected, and ends
  op "compact"     compact_pages of a cache in which `live` of the pages are held, in disorder
  op "copy"        copy_pages from one cache to another
Sizes: heads, head dimension and key counts as in the attention scores of this repository's other benchmarks (32 heads of 128,
8192 keys), its vocabulary of 128256, and generic ones.  `own` chooses between the plain form and the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _attention(name, batch, tokens, heads, kv_heads, dim, prefix, own_len, page, dtype, layout="nhd"):
    return dict(name=name, op="attention", batch=batch, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, prefix=prefix,
                own_len=own_len, page=page, dtype=dtype, layout=layout)


def _verify(name, batch, drafts, vocab, dtype, pad=0):
    return dict(name=name, op="verify", batch=batch, drafts=drafts, vocab=vocab, dtype=dtype, pad=pad)


def _samples(name, prompts, samples, prompt_len, tokens, page, pools, kv_heads, dim, dtype):
    return dict(name=name, op="samples", prompts=prompts, samples=samples, prompt_len=prompt_len, tokens=tokens, page=page, pools=pools,
                kv_heads=kv_heads, dim=dim, dtype=dtype)


def _pages(name, op, pages, live, page, pools, kv_heads, dim, dtype):
    return dict(name=name, op=op, pages=pages, live=live, page=page, pools=pools, kv_heads=kv_heads, dim=dim, dtype=dtype)


def listed():
    return [
        # Two samples of a short prompt, one new token each: the latency of a call.
        _attention("attention_small", 2, 1, 8, 2, 64, 200, 30, 16, "bf16"),
        # The ordinary decoding step: 64 samples of a prompt of 8192 tokens, 32 heads on 8 of keys and values.
        _attention("attention_samples", 64, 1, 32, 8, 128, 8192, 512, 16, "bf16"),
        # Verification step of drafted tokens: five positions of each sequence, a prompt that ends inside a page, head-major pages.
        _attention("attention_drafts", 24, 5, 32, 4, 64, 5001, 777, 64, "f16", "hnd"),
        # In single precision, every head with keys of its own.
        _attention("attention_f32", 12, 1, 16, 16, 128, 2047, 255, 16, "f32"),
        # A book as the prompt and 128 readers: the most work of one call.
        _attention("attention_book", 128, 1, 32, 8, 128, 65536, 1500, 32, "bf16"),
        # One request of the smallest vocabulary in use, four drafts.
        _verify("verify_one", 1, 4, 32000, "f32"),
        # A batch of requests, the vocabulary of the other benchmarks, rows that lie apart by a padded stride.
        _verify("verify_batch", 64, 5, 128256, "bf16", 64),
        # One prompt to four samples, one token each, one layer's two pools: launches and latency.
        _samples("samples_small", 1, 4, 1000, 1, 16, 2, 2, 64, "bf16"),
        # Sixteen prompts to 32 samples each in all layers' pools, five drafted tokens each.
        _samples("samples_batch", 16, 32, 4000, 5, 16, 24, 8, 128, "bf16"),
        # A small cache after its requests ended in disorder.
        _pages("compact_small", "compact", 256, 100, 16, 2, 2, 64, "bf16"),
        # A large one: half of the pages are held, every layer's pools move together.
        _pages("compact_large", "compact", 6000, 3000, 16, 16, 8, 128, "bf16"),
        # Pages of a few sequences handed from a prefilling cache to a decoding one, in single precision.
        _pages("copy_pages", "copy", 1024, 500, 24, 8, 4, 96, "f32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more pass: the same ranges, sizes spread over their logarithms, odd ones among them."""
    while True:
        op = rng.choice(("attention", "attention", "attention", "verify", "verify", "samples", "samples", "compact", "copy"))
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        page = rng.choice((8, 16, 16, 24, 32, 64))
        kv_heads = rng.choice((1, 2, 4, 5, 8, 16))
        dim = rng.choice((64, 80, 96, 128, 128, 192, 256))
        if op == "attention":
            case = dict(op=op, batch=_log_int(rng, 1, 128), tokens=rng.choice((1, 1, 1, 2, 3, 5, 8)), heads=kv_heads * rng.choice((1, 2, 4, 5, 8)), kv_heads=kv_heads,
                        dim=dim, prefix=rng.choice((0, _log_int(rng, 16, 65536), _log_int(rng, 16, 65536), _log_int(rng, 16, 65536))), own_len=_log_int(rng, 8, 4096),
                        page=page, dtype=dtype, layout=rng.choice(("nhd", "nhd", "hnd")))
            w, most = work(case), work(listed()[4])
            # in single precision a product takes some 16 times as long
            if w["flops"] * (16 if dtype == "f32" else 1) > most["flops"] or w["bytes"] > most["bytes"]:
                continue
        elif op == "verify":
            case = dict(op=op, batch=_log_int(rng, 1, 128), drafts=rng.randint(1, 8), vocab=_log_int(rng, 1000, 160000), dtype=dtype, pad=rng.choice((0, 0, 7, 64)))
            if case["batch"] * (2 * case["drafts"] + 1) * case["vocab"] > 1 << 27:
                continue
        elif op == "samples":
            case = dict(op=op, prompts=_log_int(rng, 1, 16), samples=_log_int(rng, 1, 64), prompt_len=_log_int(rng, 10, 8000), tokens=rng.choice((1, 1, 2, 5, 8)), page=page,
                        pools=2 * _log_int(rng, 1, 12), kv_heads=kv_heads, dim=dim, dtype=dtype)
            if work(case)["bytes"] > work(listed()[8])["bytes"] or _pool_bytes(case) > 8e9:
                continue
        else:
            pages = _log_int(rng, 64, 8000)
            case = dict(op=op, pages=pages, live=rng.randint(1, pages - 1), page=page, pools=2 * _log_int(rng, 1, 12), kv_heads=kv_heads, dim=dim, dtype=dtype)
            if work(case)["bytes"] > work(listed()[10])["bytes"] or _pool_bytes(case) > 8e9:
                continue
        return case


def _sample_pages(c):
    """Pages of the cache of a "samples" case: the prompts', what every child may take, and a third left over."""
    held = c["prompts"] * -(-c["prompt_len"] // c["page"])
    taken = c["prompts"] * c["samples"] * (1 + -(-c["tokens"] // c["page"]))
    return (held + taken) * 4 // 3 + 1


def _pool_bytes(c):
    pages = _sample_pages(c) if c["op"] == "samples" else c["pages"] * (2 if c["op"] == "copy" else 1)
    return pages * c["page"] * c["kv_heads"] * c["dim"] * _BYTES[c["dtype"]] * c["pools"]


def work(c):
    if c["op"] == "attention":
        es, mean_own = _BYTES[c["dtype"]], 0.75 * c["own_len"]
        kv = 2 * (c["prefix"] + c["batch"] * mean_own) * c["kv_heads"] * c["dim"] * es
        io = 2 * c["batch"] * c["tokens"] * c["heads"] * c["dim"] * es
        return {"bytes": kv + io, "flops": 4.0 * c["dim"] * c["heads"] * c["tokens"] * c["batch"] * (c["prefix"] + mean_own)}
    if c["op"] == "verify":
        # one row of the target's probabilities and, after a rejection, one of the draft's; most drafts have one
        return {"bytes": 2.0 * c["batch"] * c["vocab"] * _BYTES[c["dtype"]], "flops": 3.0 * c["batch"] * c["vocab"]}
    token = c["kv_heads"] * c["dim"] * _BYTES[c["dtype"]] * c["pools"]
    if c["op"] == "samples":
        n = c["prompts"] * c["samples"]
        row = 4.0 * (c["prompt_len"] // c["page"] + 2)
        # the filled tokens of part-filled pages and the new ones, read and written; the children's rows, written and given back
        return {"bytes": n * (2.0 * (0.5 * c["page"] + c["tokens"]) * token + 4 * row), "flops": 0}
    if c["op"] == "compact":
        moved = c["live"] * (c["pages"] - c["live"]) / c["pages"]
        return {"bytes": 2.0 * moved * c["page"] * token + 24.0 * c["pages"], "flops": 0}
    return {"bytes": 2.0 * c["live"] * c["page"] * token, "flops": 0}


# ---------------------------------------------------------------------------------------------------------------- inputs

def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"attention": _prepare_attention, "verify": _prepare_verify, "samples": _prepare_samples, "compact": _prepare_compact,
            "copy": _prepare_copy}[c["op"]](c, g)


def _randint(g, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int64)


def _randn(g, shape, dtype):
    if math.prod(shape) > 1 << 28:   # one slice after the other: the 32-bit numbers of all would not stay small
        return torch.stack([_randn(g, shape[1:], dtype) for _ in range(shape[0])])
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _prepare_attention(c, g):
    B, T, ps, dt = c["batch"], c["tokens"], c["page"], _DTYPES[c["dtype"]]
    # whole length of every sequence: the prefix, what it has decoded, and the T new tokens
    lens = c["prefix"] + torch.clamp(c["own_len"] - _randint(g, 0, c["own_len"] // 2 + 1, (B,)), min=T)
    shared = c["prefix"] // ps                       # whole pages of the prefix: the same ones in every row
    most = -(-(c["prefix"] + max(c["own_len"], T)) // ps)
    pages = shared + B * (most - shared)
    ids = torch.randperm(pages, generator=g, device="cuda")
    table = torch.empty((B, most), dtype=torch.int64, device="cuda")
    table[:, :shared] = ids[:shared]
    table[:, shared:] = ids[shared:].reshape(B, most - shared)
    shape = (pages, ps, c["kv_heads"], c["dim"])
    if c["layout"] == "hnd":
        kv = [_randn(g, (pages, c["kv_heads"], ps, c["dim"]), dt).transpose(1, 2) for _ in range(2)]
    else:
        kv = [_randn(g, shape, dt) for _ in range(2)]
    left = c["prefix"] - shared * ps                 # a prefix that ends inside a page: every sequence holds a copy of that part
    if left:
        for pool in kv:
            pool[table[:, shared], :left] = pool[table[0, shared], :left].clone()
    q = _randn(g, (B, T, c["heads"], c["dim"]), dt)
    return dict(op="attention", q=q, k=kv[0], v=kv[1], table=table.int(), lens=lens.int(), prefix=c["prefix"], scale=c["dim"] ** -0.5)


def _prepare_verify(c, g):
    B, L, V, dt = c["batch"], c["drafts"], c["vocab"], _DTYPES[c["dtype"]]
    wide = V + c["pad"]
    target = torch.zeros((B, L + 1, wide), dtype=dt, device="cuda")
    draft = torch.zeros((B, L, wide), dtype=dt, device="cuda")
    tokens = torch.empty((B, L), dtype=torch.int32, device="cuda")
    for b in range(B):
        # a model and a cheaper one that mostly agrees with it
        logits = 3 * torch.randn((L + 1, V), generator=g, device="cuda")
        other = logits[:L] + 0.7 * torch.randn((L, V), generator=g, device="cuda")
        target[b, :, :V] = torch.softmax(logits, -1).to(dt)
        probs = torch.softmax(other, -1)
        draft[b, :, :V] = probs.to(dt)
        tokens[b] = torch.multinomial(probs, 1, generator=g).squeeze(-1).int()
    return dict(op="verify", target=target[..., :V], draft=draft[..., :V], tokens=tokens, u=torch.rand((B, L), generator=g, device="cuda"),
                r=torch.rand((B,), generator=g, device="cuda"))


def _tables(page_table, lens, refs, free_pages, n_free, page):
    state = dict(page_table=page_table.int(), lens=lens.int(), refs=refs.int(), free_pages=free_pages.int(), n_free=n_free.int())
    if own:
        import paper_2412_04358_amd as atk

        return atk.PageTables(page_size=page, **state)
    return dict(page=page, **state)


def _prepare_samples(c, g):
    dt, ps, N = _DTYPES[c["dtype"]], c["page"], c["prompts"] * c["samples"]
    P = _sample_pages(c)
    used = -(-c["prompt_len"] // ps)
    M = -(-(c["prompt_len"] + c["tokens"]) // ps) + 1
    ids = torch.randperm(P, generator=g, device="cuda")
    S = c["prompts"] + N
    table = torch.full((S, M), -1, dtype=torch.int64, device="cuda")
    lens = torch.zeros((S,), dtype=torch.int64, device="cuda")
    held = ids[:c["prompts"] * used].reshape(c["prompts"], used)
    table[:c["prompts"], :used] = held
    # prompts end at places of their own, in their last pages
    lens[:c["prompts"]] = c["prompt_len"] - _randint(g, 0, (c["prompt_len"] - 1) % ps + 1, (c["prompts"],))
    refs = torch.zeros((P,), dtype=torch.int64, device="cuda")
    refs[held.flatten()] = 1
    free = torch.full((P,), -1, dtype=torch.int64, device="cuda")
    rest = torch.sort(ids[c["prompts"] * used:], descending=True).values
    free[:rest.numel()] = rest
    pools = [_randn(g, (P, ps, c["kv_heads"], c["dim"]), dt) for _ in range(c["pools"])]
    values = [_randn(g, (N, c["tokens"], c["kv_heads"], c["dim"]), dt) for _ in range(c["pools"])]
    parents = torch.arange(N, device="cuda") % c["prompts"]
    children = c["prompts"] + torch.randperm(N, generator=g, device="cuda")
    rejected = torch.full((N,), c["tokens"] // 2, device="cuda")
    return dict(op="samples", tables=_tables(table, lens, refs, free, torch.tensor([rest.numel()], device="cuda"), ps), pools=pools, values=values,
                parents=parents.int(), children=children.int(), rejected=rejected.int())


def _prepare_compact(c, g):
    dt, ps, P, live = _DTYPES[c["dtype"]], c["page"], c["pages"], c["live"]
    ids = torch.randperm(P, generator=g, device="cuda")
    S = max(1, live // 50)                           # sequences of some 50 pages; those of one prompt share its first page
    M = -(-live // S) + 1
    flat = torch.full((S * (M - 1),), -1, dtype=torch.int64, device="cuda")
    flat[:live] = ids[:live]
    table = torch.full((S, M), -1, dtype=torch.int64, device="cuda")
    table[:, 1:] = flat.reshape(S, M - 1)
    table[:, 0] = ids[0]
    lens = (table >= 0).sum(1) * ps
    refs = torch.zeros((P,), dtype=torch.int64, device="cuda")
    refs[ids[:live]] = 1
    refs[ids[0]] = S + 1
    free = torch.full((P,), -1, dtype=torch.int64, device="cuda")
    free[:P - live] = ids[live:]
    pools = [_randn(g, (P, ps, c["kv_heads"], c["dim"]), dt) for _ in range(c["pools"])]
    t = _tables(table, lens, refs, free, torch.tensor([P - live], device="cuda"), ps)
    left = {k: (t[k] if isinstance(t, dict) else getattr(t, k)).clone() for k in ("page_table", "refs", "free_pages", "n_free")}
    return dict(op="compact", tables=t, left=left, pools=pools)


def _prepare_copy(c, g):
    dt, n = _DTYPES[c["dtype"]], c["live"]
    shape = (c["pages"], c["page"], c["kv_heads"], c["dim"])
    src = [_randn(g, shape, dt) for _ in range(c["pools"])]
    dst = [torch.zeros(shape, dtype=dt, device="cuda") for _ in range(c["pools"])]
    return dict(op="copy", src=src, dst=dst, src_ids=torch.randperm(c["pages"], generator=g, device="cuda")[:n].int(),
                dst_ids=torch.randperm(c["pages"], generator=g, device="cuda")[:n].int())


# ------------------------------------------------------------------------------------------------------------------ passes

def run(s):
    return (_run_own if own else _run_plain)[s["op"]](s)


def _own_attention(s):
    import paper_2412_04358_amd as atk

    out, lse = atk.shared_prefix_attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["prefix"], scale=s["scale"], return_lse=True)
    return {"out": out, "lse": lse}


def _own_verify(s):
    import paper_2412_04358_amd as atk

    accepted, tokens = atk.verify_drafts(s["target"], s["tokens"], s["draft"], s["u"], s["r"])
    return {"accepted": accepted, "tokens": tokens}


def _tables_out(t, pools):
    get = t.__getitem__ if isinstance(t, dict) else lambda k: getattr(t, k)
    return {**{k: get(k) for k in ("page_table", "lens", "refs", "free_pages", "n_free")}, "pools": pools}


def _own_samples(s):
    import paper_2412_04358_amd as atk

    t = s["tables"]
    atk.fork_sequences(t, s["pools"], s["parents"], s["children"])
    atk.append_tokens(t, s["pools"], s["children"], s["values"])
    atk.free_sequences(t, s["children"], drop=s["rejected"])
    rows, lens = t.page_table.clone(), t.lens.clone()
    atk.free_sequences(t, s["children"])
    return {"rows": rows, "row_lens": lens, **_tables_out(t, s["pools"])}


def _own_compact(s):
    import paper_2412_04358_amd as atk

    t = s["tables"]
    for k, v in s["left"].items():   # the disorder that ended requests leave
        getattr(t, k).copy_(v)
    remap = atk.compact_pages(t, s["pools"])
    return {"remap": remap, **_tables_out(t, s["pools"])}


def _own_copy(s):
    import paper_2412_04358_amd as atk

    atk.copy_pages(s["src"], s["src_ids"], s["dst"], s["dst_ids"])
    return s["dst"]


def _plain_attention(s):
    q, k, v, table, lens, prefix = s["q"], s["k"], s["v"], s["table"].long(), s["lens"].long(), s["prefix"]
    B, T, H, D = q.shape
    ps, Hk = k.shape[1], k.shape[2]
    G = H // Hk
    limit = (lens[:, None] - (T - 1) + torch.arange(T, device=q.device)[None, :])      # (B, T): visible keys
    rows = q.float().reshape(B, T, Hk, G, D)
    parts = []
    if prefix:
        # the shared part once: rows of all sequences against the first one's pages, head by head
        n = -(-prefix // ps)
        kp = k[table[0, :n]].float().reshape(n * ps, Hk, D)[:prefix].permute(1, 2, 0).contiguous()
        vp = v[table[0, :n]].float().reshape(n * ps, Hk, D)[:prefix].transpose(0, 1).contiguous()
        sc = torch.matmul(rows.permute(2, 0, 1, 3, 4).reshape(Hk, B * T * G, D), kp).reshape(Hk, B, T, G, prefix) * s["scale"]
        seen = torch.arange(prefix, device=q.device) < limit[:, :, None, None]
        parts.append(_plain_part(sc.masked_fill_(~seen, float("-inf")), lambda w: torch.matmul(w.reshape(Hk, B * T * G, prefix), vp).reshape(Hk, B, T, G, D)))
        del sc, kp, vp
    first = prefix // ps
    most = table.shape[1] * ps - first * ps
    if most > 0:
        ko = k[table[:, first:].clamp(min=0)].float().reshape(B, most, Hk, D).permute(2, 0, 3, 1).contiguous()
        at = torch.arange(first * ps, first * ps + most, device=q.device)
        sc = torch.matmul(rows.permute(2, 0, 1, 3, 4).reshape(Hk, B, T * G, D), ko).reshape(Hk, B, T, G, most) * s["scale"]
        del ko
        seen = (at >= prefix) & (at < limit[:, :, None, None])
        vo = v[table[:, first:].clamp(min=0)].float().reshape(B, most, Hk, D)
        vo = vo.masked_fill_((at >= lens[:, None])[:, :, None, None], 0.0).permute(2, 0, 1, 3).contiguous()
        parts.append(_plain_part(sc.masked_fill_(~seen, float("-inf")), lambda w: torch.matmul(w.reshape(Hk, B, T * G, most), vo).reshape(Hk, B, T, G, D)))
    top = parts[0][0]
    for m, _, _ in parts[1:]:
        top = torch.maximum(top, m)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    total = sum(torch.exp(m - top) * l for m, l, _ in parts)
    out = sum(torch.exp(m - top)[..., None] * o for m, _, o in parts) / torch.where(total > 0, total, torch.ones_like(total))[..., None]
    lse = torch.where(total > 0, top + torch.log(total), torch.full_like(total, float("-inf")))
    return {"out": out.permute(1, 2, 0, 3, 4).reshape(B, T, H, D).to(q.dtype), "lse": lse.permute(1, 2, 0, 3).reshape(B, T, H)}


def _plain_part(sc, product):
    """Maximum, sum and weighted values of one range of keys."""
    m = sc.amax(-1)
    w = torch.exp(sc - torch.where(torch.isinf(m), torch.zeros_like(m), m)[..., None])
    return m, w.sum(-1), product(w)


def _plain_verify(s):
    target, draft, tokens = s["target"], s["draft"], s["tokens"].long()
    B, L = tokens.shape
    p = target[:, :L].gather(2, tokens[..., None])[..., 0].double()
    q = draft.gather(2, tokens[..., None])[..., 0].double()
    taken = s["u"].double() * q < p
    accepted = torch.cumprod(taken.long(), 1).sum(1)
    rows = torch.arange(B, device=tokens.device)
    pr = target[rows, accepted].double()
    qr = torch.where((accepted < L)[:, None], draft[rows, accepted.clamp(max=L - 1)].double(), 0.0)
    w = pr - qr
    w = torch.where(w > 0, w, 0.0)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, torch.where(pr > 0, pr, 0.0))
    c = torch.cumsum(w, 1)
    above = c > (s["r"].double() * c[:, -1])[:, None]
    last = (w > 0).long().cumsum(1).argmax(1)
    token = torch.where(above.any(1), above.long().argmax(1), last)
    token = torch.where((w > 0).any(1), token, -1)
    at = torch.arange(L + 1, device=tokens.device)[None, :]
    padded = torch.cat([tokens, tokens.new_zeros((B, 1))], 1)
    out = torch.where(at < accepted[:, None], padded, torch.where(at == accepted[:, None], token[:, None], -1))
    return {"accepted": accepted.int(), "tokens": out.int()}


def _plain_fork(t, pools, parents, children):
    ps, parents, children = t["page"], parents.long(), children.long()
    lens = t["lens"][parents].long()
    part = lens % ps
    takes = (part > 0).long()
    rank = torch.cumsum(takes, 0) - takes
    fresh = t["free_pages"][(t["n_free"].long() - 1 - rank).clamp(min=0)].long()
    rows = t["page_table"][parents].long()
    last = ((lens + ps - 1) // ps - 1).clamp(min=0)
    old = rows.gather(1, last[:, None])[:, 0]
    new = torch.where(takes > 0, fresh, old)
    for pool in pools:
        copied = torch.arange(ps, device=lens.device)[None, :, None, None] < part[:, None, None, None]
        pool[new] = torch.where(copied, pool[old], pool[new])
    rows.scatter_(1, last[:, None], new[:, None])
    t["page_table"][children] = rows.int()
    t["lens"][children] = lens.int()
    held = rows[rows >= 0]
    t["refs"].index_add_(0, held, torch.ones_like(held).int())
    t["n_free"] -= takes.sum().int()


def _plain_append(t, pools, seqs, values):
    ps, seqs = t["page"], seqs.long()
    n, T = values[0].shape[:2]
    lens = t["lens"][seqs].long()
    used, after = (lens + ps - 1) // ps, (lens + T + ps - 1) // ps
    last = (used - 1).clamp(min=0)
    old = t["page_table"][seqs, last].long()
    copies = ((lens % ps > 0) & (t["refs"][old.clamp(min=0)] > 1)).long()
    takes = after - used + copies
    base = t["n_free"].long() - 1 - (torch.cumsum(takes, 0) - takes)
    fresh = t["free_pages"][base.clamp(min=0)].long()
    new = torch.where(copies > 0, fresh, old.clamp(min=0))
    for pool in pools:
        copied = (torch.arange(ps, device=lens.device)[None, :] < (copies * (lens % ps))[:, None])[:, :, None, None]
        pool[new] = torch.where(copied, pool[old], pool[new])
    t["page_table"][seqs, last] = torch.where(copies > 0, new, old).int()
    t["refs"].index_add_(0, old.clamp(min=0), -copies.int())
    t["refs"].index_add_(0, new, copies.int())
    for j in range(-(-T // ps) + 1):
        at = used + j
        wanted = at < after
        page = t["free_pages"][(base - copies - j).clamp(min=0)]
        place = at.clamp(max=t["page_table"].shape[1] - 1)
        t["page_table"][seqs, place] = torch.where(wanted, page, t["page_table"][seqs, place])
        t["refs"].index_add_(0, page.long().clamp(min=0), wanted.int())
    at = lens[:, None] + torch.arange(T, device=lens.device)[None, :]
    page = t["page_table"][seqs[:, None], at // ps].long()
    for pool, value in zip(pools, values):
        pool[page, at % ps] = value
    t["lens"][seqs] = (lens + T).int()
    t["n_free"] -= takes.sum().int()


def _plain_free(t, seqs, drop=None):
    ps, seqs = t["page"], seqs.long()
    lens = t["lens"][seqs].long()
    keep = torch.zeros_like(lens) if drop is None else (lens - drop.long()).clamp(min=0)
    rows = t["page_table"][seqs].long()
    at = torch.arange(rows.shape[1], device=rows.device)[None, :]
    gone = (at >= ((keep + ps - 1) // ps)[:, None]) & (rows >= 0)
    pages = rows[gone]
    before = t["refs"] > 0
    t["refs"].index_add_(0, pages, -torch.ones_like(pages).int())
    t["page_table"][seqs] = torch.where(gone, -1, rows).int()
    t["lens"][seqs] = keep.int()
    ended = torch.nonzero(before & (t["refs"] == 0))[:, 0].flip(0)
    place = t["n_free"].long() + torch.arange(ended.numel(), device=rows.device)
    t["free_pages"][place] = ended.int()
    t["n_free"] += ended.numel()


def _plain_samples(s):
    t = s["tables"]
    _plain_fork(t, s["pools"], s["parents"], s["children"])
    _plain_append(t, s["pools"], s["children"], s["values"])
    _plain_free(t, s["children"], s["rejected"])
    rows, lens = t["page_table"].clone(), t["lens"].clone()
    _plain_free(t, s["children"])
    return {"rows": rows, "row_lens": lens, **_tables_out(t, s["pools"])}


def _plain_compact(s):
    t = s["tables"]
    for k, v in s["left"].items():
        t[k].copy_(v)
    refs = t["refs"]
    P = refs.numel()
    ids = torch.arange(P, device=refs.device)
    held = refs > 0
    live = held.sum()
    moved = torch.nonzero(held & (ids >= live))[:, 0]
    holes = torch.nonzero(~held & (ids < live))[:, 0]
    remap = torch.where(held, ids, -1)
    remap[moved] = holes
    for pool in s["pools"]:
        pool[holes] = pool[moved]
    refs[holes] = refs[moved]
    refs[moved] = 0
    table = t["page_table"].long()
    t["page_table"].copy_(torch.where(table >= 0, remap[table.clamp(min=0)], -1))
    t["free_pages"].copy_(torch.where(ids < P - live, P - 1 - ids, t["free_pages"]))
    t["n_free"].copy_(P - live)
    return {"remap": remap.int(), **_tables_out(t, s["pools"])}


def _plain_copy(s):
    for a, b in zip(s["src"], s["dst"]):
        b[s["dst_ids"].long()] = a[s["src_ids"].long()]
    return s["dst"]


_run_own = {"attention": _own_attention, "verify": _own_verify, "samples": _own_samples, "compact": _own_compact, "copy": _own_copy}
_run_plain = {"attention": _plain_attention, "verify": _plain_verify, "samples": _plain_samples, "compact": _plain_compact, "copy": _plain_copy}


# --------------------------------------------------------------------------------------------------- definitions in 64 bits

def exact(c, seed):
    """What a pass returns, from the definition in 64 bits; pages are moved bit by bit, so their passes have no such values."""
    if c["op"] == "attention":
        if work(c)["flops"] > 4e11:
            return None
        s = prepare(c, seed)
        return _exact_attention(s)
    if c["op"] == "verify":
        return _exact_verify(prepare(c, seed))
    return None


def _exact_attention(s):
    q, k, v = s["q"], s["k"], s["v"]
    B, T, H, D = q.shape
    ps, Hk = k.shape[1], k.shape[2]
    out = torch.zeros((B, T, H, D), dtype=torch.float64, device=q.device)
    lse = torch.full((B, T, H), float("-inf"), dtype=torch.float64, device=q.device)
    for b in range(B):
        n = int(s["lens"][b])
        # the sequence's keys one after the other, the shared ones through the first sequence's row
        at = torch.arange(n, device=q.device)
        page = torch.where(at < s["prefix"], s["table"][0].long()[at // ps], s["table"][b].long()[at // ps])
        for h in range(Hk):
            keys, vals = k[page, at % ps, h].double(), v[page, at % ps, h].double()
            for t in range(T):
                m = n - (T - 1 - t)
                if m <= 0:
                    continue
                heads = slice(h * (H // Hk), (h + 1) * (H // Hk))
                z = s["scale"] * torch.mm(q[b, t, heads].double(), keys[:m].t())
                lse[b, t, heads] = torch.logsumexp(z, -1)
                out[b, t, heads] = torch.mm(torch.softmax(z, -1), vals[:m])
    return {"out": out, "lse": lse}


def _exact_verify(s):
    import numpy as np

    u, r = s["u"].cpu().numpy().astype(np.float64), s["r"].cpu().numpy().astype(np.float64)
    tokens = s["tokens"].cpu().numpy()
    B, L = tokens.shape
    accepted, out = np.zeros((B,), np.int64), np.full((B, L + 1), -1, np.int64)
    for b in range(B):
        i = 0
        while i < L:
            d = int(tokens[b, i])
            if not u[b, i] * float(s["draft"][b, i, d]) < float(s["target"][b, i, d]):
                break
            out[b, i] = d
            i += 1
        accepted[b] = i
        p = s["target"][b, i].double().cpu().numpy()
        w = np.maximum(p - s["draft"][b, i].double().cpu().numpy(), 0) if i < L else p
        if not w.any():
            w = p
        c = np.cumsum(w)
        out[b, i] = np.searchsorted(c, r[b] * c[-1], side="right") if w.any() else -1
    return {"accepted": torch.from_numpy(accepted).int(), "tokens": torch.from_numpy(out).int()}
