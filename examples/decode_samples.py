"""Several samples of one prompt, decoded together with drafted tokens: the decoding operators as a program uses them.

    python examples/decode_samples.py [--samples 8] [--prompt 500] [--steps 12] [--drafts 3]

A tiny random transformer of one layer stands for the model, and a coarser copy of it for the model that drafts.  Per step: the drafting model proposes
tokens, each among its k most likely (exact_topk); their keys and values go into the samples' pages (append_tokens); one attention over the shared
prompt and each sample's own tokens gives the target's probabilities at all positions (shared_prefix_attention); verify_drafts decides; what was rejected
is given back (free_sequences).  At the end the samples' pages are closed up (compact_pages).  Nothing in a step waits for the GPU.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2412_04358_amd as atk  # noqa: E402

HEADS, KV_HEADS, DIM, VOCAB, PAGE, TOP = 8, 2, 64, 4096, 16, 32


class Model:
    """Embedding, one attention layer, unembedding; `noise` makes a copy that only mostly agrees."""

    def __init__(self, device, noise=0.0):
        g = torch.Generator(device=device).manual_seed(0)

        def weight(rows, cols):
            w = torch.randn((rows, cols), generator=g, device=device) * rows ** -0.5
            e = torch.randn((rows, cols), generator=g, device=device) * rows ** -0.5
            return (w + noise * e).bfloat16()

        width = HEADS * DIM
        self.embed, self.wq, self.wkv, self.wo, self.head = weight(VOCAB, width), weight(width, width), weight(width, 2 * KV_HEADS * DIM), weight(width, width), weight(width, VOCAB)
        self.embed = self.embed * VOCAB ** 0.5

    def keys_values(self, tokens):
        kv = (self.embed[tokens.long()] @ self.wkv).unflatten(-1, (2, KV_HEADS, DIM))
        return [kv[..., 0, :, :].contiguous(), kv[..., 1, :, :].contiguous()]

    def queries(self, tokens):
        return (self.embed[tokens.long()] @ self.wq).unflatten(-1, (HEADS, DIM))

    def logits(self, tokens, attended):
        return (self.embed[tokens.long()] + attended.flatten(-2) @ self.wo) @ self.head


def likely(logits, r):
    """The distribution of the TOP most likely tokens, and a token drawn from it."""
    rows = logits.reshape(-1, VOCAB).contiguous()
    vals, idx = atk.exact_topk(rows, TOP)
    probs = torch.zeros(rows.shape, device=rows.device).scatter_(1, idx.long(), torch.softmax(2 * vals.float(), -1))
    token = (probs.cumsum(1) > r.reshape(-1, 1) * probs.sum(1, keepdim=True)).int().argmax(1)
    return probs.reshape(logits.shape), token.int().reshape(logits.shape[:-1])


def run(samples=8, prompt=500, steps=12, drafts=3, check=False, quiet=False):
    device = torch.device("cuda")
    g = torch.Generator(device=device).manual_seed(1)
    target, drafter = Model(device), Model(device, noise=0.1)
    own = steps * (drafts + 1) + drafts + 2
    row_pages = -(-(prompt + own) // PAGE) + 1
    pages = row_pages * (samples + 1)
    t = atk.PageTables.empty(pages, PAGE, samples + 1, row_pages)
    pools = [torch.zeros((pages, PAGE, KV_HEADS, DIM), dtype=torch.bfloat16, device=device) for _ in range(4)]  # keys and values of the target and of the drafting model
    children = torch.arange(1, samples + 1, dtype=torch.int32, device=device)

    def both(tokens):
        return target.keys_values(tokens) + drafter.keys_values(tokens)

    def attend(model, tokens):
        which = 0 if model is target else 2
        return model.logits(tokens, atk.shared_prefix_attention(model.queries(tokens), pools[which], pools[which + 1], t.page_table, t.lens, prompt - 1, seqs=children, status=t.status))

    first = torch.randint(0, VOCAB, (1, prompt), generator=g, device=device).int()
    row = torch.zeros((1,), dtype=torch.int32, device=device)
    atk.append_tokens(t, pools, row, both(first[:, :-1]))
    atk.fork_sequences(t, pools, row.expand(samples).contiguous(), children)
    last = first[:, -1:].expand(samples, 1).contiguous()    # the newest token of each sample: not in the cache yet
    history, counts, worst = [], [], 0.0
    for _ in range(steps):
        # drafts, one after the other
        tokens, probs = [last], []
        for _ in range(drafts):
            atk.append_tokens(t, pools, children, both(tokens[-1]))
            p, token = likely(attend(drafter, tokens[-1]), torch.rand((samples, 1), generator=g, device=device))
            probs.append(p)
            tokens.append(token)
        atk.append_tokens(t, pools, children, both(tokens[-1]))
        # the target, all positions at once
        given = torch.cat(tokens, 1)
        logits = attend(target, given)
        if check:
            worst = max(worst, _distance(target, logits, first[:, :-1], history, given))
        probs_target, _ = likely(logits, torch.zeros((samples, drafts + 1), device=device))
        accepted, drawn = atk.verify_drafts(probs_target, given[:, 1:].contiguous(), torch.cat(probs, 1), torch.rand((samples, drafts), generator=g, device=device),
                                            torch.rand((samples,), generator=g, device=device))
        atk.free_sequences(t, children, drop=drafts - accepted)
        last = drawn.gather(1, accepted.long()[:, None]).int()
        history.append((given, accepted))
        counts.append(accepted)
    remap = atk.compact_pages(t, pools)
    torch.cuda.synchronize()
    assert t.status.item() == 0
    counts = torch.stack(counts).float()
    report = {"tokens": int(counts.sum().item()) + samples * steps, "accepted": counts.mean().item() / drafts, "pages": int((remap >= 0).sum().item()), "worst": worst}
    if not quiet:
        print("%d samples, %d steps: %d tokens, %.0f %% of the drafts accepted, %d of %d pages held" % (samples, steps, report["tokens"], 100 * report["accepted"], report["pages"], pages))
    return report


def _distance(model, logits, prompt, history, given):
    """How far the logits are from those of the same tokens without a cache, in units of what rounding to bfloat16 may do."""
    worst = 0.0
    for b in range(given.shape[0]):
        seq = [prompt[0]] + [tokens[b, :1 + int(n[b])] for tokens, n in history] + [given[b]]
        seq = torch.cat(seq).unsqueeze(0)
        T = given.shape[1]
        k, v = (x[0].double().repeat_interleave(HEADS // KV_HEADS, 1) for x in model.keys_values(seq))
        q = model.queries(seq[:, -T:])[0].double()
        s = (q.unsqueeze(1) * k.unsqueeze(0)).sum(-1) * DIM ** -0.5
        n = k.shape[0]
        hidden = torch.arange(n, device=s.device)[None, :] > (n - T + torch.arange(T, device=s.device))[:, None]
        w = torch.softmax(s.masked_fill(hidden.unsqueeze(-1), float("-inf")), 1)
        out = (w.unsqueeze(-1) * v.unsqueeze(0)).sum(1)
        want = model.logits(seq[0, -T:], out.bfloat16())
        # the attention's output is off by two roundings of 2^-8 of sum w |v| at most; the products behind it carry that to the logits
        off = (w.unsqueeze(-1) * v.abs().unsqueeze(0)).sum(1).flatten(-2) * 2.0 ** -7
        allowed = off @ model.wo.double().abs() @ model.head.double().abs() + want.double().abs() * 2.0 ** -6 + 2.0 ** -6 * model.embed.float().abs().max().item()
        worst = max(worst, ((logits[b].double() - want.double()).abs() / allowed).max().item())
    return worst


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    for name, value in (("samples", 8), ("prompt", 500), ("steps", 12), ("drafts", 3)):
        a.add_argument("--" + name, type=int, default=value)
    run(**vars(a.parse_args()))
