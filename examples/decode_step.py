"""Decoding with drafts on a fetched prefix: how the copies and the operators over a paged cache work together.

    python examples/decode_step.py [--batch 8] [--prefix 2000] [--drafts 4] [--steps 8] [--kind fp8|int8] [--dtype bfloat16|float16]

A shared prefix lies in pinned host memory, as blocks that hold a page each (codes of keys and values and their scales).  Its blocks are
fetched into whatever pages of the device's pool are free (dl_batch_copy).  Then, step by step and for all sequences at once, drafts are
proposed, the keys and values of the last token and of the drafts are written into the cache (dl_kv_write), the queries attend to the
prefix and to their own sequence (dl_prefix_attention), and what the target makes of the drafts decides how many stay (dl_verify_draft).
Places of refused drafts are written over by the next step.

The target is one layer of attention with random weights between an embedding and an output matrix, the draft the same without attention.
The last step is checked: the attention against a dense one in float32 over what dl_kv_read gives back, the verification against its rule.
"""

from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2511_06605_amd as dl  # noqa: E402

CODES = {"fp8": torch.float8_e4m3fn, "int8": torch.int8}


class Blocks:
    """A pool of pages, each one block: codes of keys, codes of values, scales of keys, scales of values."""

    def __init__(self, pages, page, heads, dim, kind, on_device):
        codes, scales = page * heads * dim, page * heads * 4
        self.page, self.block = page, 2 * (codes + scales)
        if on_device:
            self.pool = torch.zeros((pages, self.block), dtype=torch.uint8, device="cuda")
        else:
            self.pool = torch.zeros((pages, self.block), dtype=torch.uint8, pin_memory=True)

        def code(at):
            return self.pool[:, at:at + codes].view(CODES[kind]).unflatten(1, (page, heads, dim))

        def scale(at):
            return self.pool[:, at:at + scales].view(torch.float32).unflatten(1, (page, heads))

        self.views = code(0), code(codes), scale(2 * codes), scale(2 * codes + scales)

    def address(self, page):
        return self.pool.data_ptr() + int(page) * self.block


def slots_of(table, tokens, page):
    """Slots of the tokens `tokens` [..., n] of sequences with the page tables `table` [..., pages]."""
    return table.long().gather(-1, tokens // page) * page + tokens % page


def dense(q, k, v, visible):
    """q [M, H, D], k and v [n, heads, D] of float32, visible [M, n]: attention as its formula says it."""
    group = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    s = torch.stack([q[:, h] @ k[:, h].T.contiguous() for h in range(q.shape[1])], 1) * q.shape[2] ** -0.5
    p = torch.softmax(s.masked_fill(~visible[:, None], float("-inf")), -1)
    return torch.stack([p[:, h] @ v[:, h].contiguous() for h in range(q.shape[1])], 1)


def run(batch=8, prefix=2000, drafts=4, steps=8, kind="fp8", dtype="bfloat16", q_heads=14, heads=2, dim=64, vocab=4000, page=16, seed=0):
    dtype = getattr(torch, dtype)
    stream = torch.cuda.current_stream()
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = q_heads * dim
    rand = lambda *shape: torch.randn(shape, device="cuda", generator=g)  # noqa: E731
    most = steps * (drafts + 1) + drafts + 2
    embed, place = rand(vocab, width), 0.3 * rand(prefix + most, width)
    wq, wk, wv = rand(width, width) * width ** -0.5, rand(width, heads * dim) * width ** -0.5, rand(width, heads * dim) * width ** -0.5
    wo = rand(width, vocab) * 2.0 * width ** -0.5

    def keys_values(x):
        return tuple((x @ w).unflatten(-1, (heads, dim)).to(dtype).reshape(-1, heads, dim) for w in (wk, wv))

    # pages of the device's pool, handed out in no particular order
    n_prefix, n_own = -(-prefix // page), -(-most // page)
    free = torch.randperm(n_prefix + batch * n_own, device="cuda", generator=g).int()
    prefix_pages, own_pages = free[:n_prefix].contiguous(), free[n_prefix:].view(batch, n_own)
    device, host = (Blocks(n, page, heads, dim, kind, on) for n, on in ((len(free), True), (n_prefix, False)))
    cache = dl.KvCache(*device.views)

    # The prefix, computed once and kept on the host: written into the first pages, whose blocks are moved out (and forgotten here) ...
    tokens = torch.randint(vocab, (prefix,), device="cuda", generator=g)
    k, v = keys_values(embed[tokens] + place[:prefix])
    dl.dl_kv_write(cache, dl.KvRows(k, v, torch.arange(prefix, device="cuda")), stream)
    dl.dl_batch_copy([(device.address(i), host.address(i), device.block) for i in range(n_prefix)], stream)
    device.pool.zero_()
    # ... and fetched into the pages that this batch has for it.
    dl.dl_batch_copy([(host.address(i), device.address(p), device.block) for i, p in enumerate(prefix_pages.tolist())], stream)

    M = drafts + 1
    q = torch.empty((batch, M, q_heads, dim), dtype=dtype, device="cuda")
    out = torch.empty_like(q)
    target = torch.empty((batch, M, vocab), device="cuda")
    proposed = torch.empty((batch, drafts, vocab), device="cuda")
    x = torch.empty((batch, drafts), dtype=torch.int32, device="cuda")
    uniform, race = torch.empty((batch, drafts), device="cuda"), torch.empty((batch, vocab), device="cuda")
    result, accepted = torch.empty((batch, M), dtype=torch.int32, device="cuda"), torch.empty(batch, dtype=torch.int32, device="cuda")
    lens = torch.empty(batch, dtype=torch.int32, device="cuda")

    attention = dl.PrefixAttention(cache, q, out, own_pages, lens, prefix_pages=prefix_pages, prefix_tokens=prefix)
    verification = dl.DraftVerify(target, x, uniform, race, result, accepted, draft_probs=proposed)
    workspace = torch.zeros(max(dl.dl_prefix_attention_workspace(attention), dl.dl_verify_draft_workspace(verification)), dtype=torch.uint8,
                            device="cuda")
    attention.use_workspace(workspace)
    verification.use_workspace(workspace)

    length = torch.zeros(batch, dtype=torch.long, device="cuda")  # own tokens that have stayed and whose keys are in the cache
    last = torch.randint(vocab, (batch,), device="cuda", generator=g)
    texts = [[] for _ in range(batch)]
    taken = 0
    for _ in range(steps):
        line = [last]
        for i in range(drafts):
            proposed[:, i] = torch.softmax((embed[line[-1]] + place[prefix + length + i]) @ wo, -1)
            line.append(torch.multinomial(proposed[:, i], 1, generator=g)[:, 0])
        line = torch.stack(line, 1)
        x.copy_(line[:, 1:])
        at = length[:, None] + torch.arange(M, device="cuda")
        h = embed[line] + place[prefix + at]
        k, v = keys_values(h)
        q.copy_((h @ wq).unflatten(-1, (q_heads, dim)))
        lens.copy_(length + M)
        dl.dl_kv_write(cache, dl.KvRows(k, v, slots_of(own_pages, at, page).reshape(-1)), stream)
        dl.dl_prefix_attention(attention, stream)
        target.copy_(torch.softmax((h + out.float().flatten(2)) @ wo, -1))
        uniform.uniform_(generator=g)
        race.exponential_(generator=g).clamp_(min=2.0 ** -100)
        dl.dl_verify_draft(verification, stream)
        last = result.long().gather(1, accepted.long()[:, None])[:, 0]
        length += accepted + 1
        taken += int(accepted.sum())  # (the host waits here: it is the end of a step)
        for text, row in zip(texts, result.tolist()):
            text += [t for t in row if t >= 0]

    # The last step once more, as the formulas say it.  Two roundings to 16 bits, of the weights and of the output, are at most
    # a unit each of the largest |v|; scores in 32 bits add less than a quarter of that.
    unit = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    worst = 0.0
    for b in range(batch):
        n = int(lens[b])
        where = torch.cat([slots_of(prefix_pages, torch.arange(prefix, device="cuda"), page),
                           slots_of(own_pages[b], torch.arange(n, device="cuda"), page)])
        k, v = (torch.empty((prefix + n, heads, dim), device="cuda") for _ in range(2))
        dl.dl_kv_read(cache, dl.KvRows(k, v, where), stream)
        sees = torch.arange(prefix + n, device="cuda") <= prefix + n - M + torch.arange(M, device="cuda")[:, None]
        off = (dense(q[b].float(), k, v, sees) - out[b].float()).abs().max() / v.abs().max()
        worst = max(worst, float(off) / unit)
        stays = [float(uniform[b, i]) * float(proposed[b, i, x[b, i]]) < float(target[b, i, x[b, i]]) for i in range(drafts)] + [False]
        a = stays.index(False)
        w = (target[b, a] - proposed[b, a]).clamp(min=0) if a < drafts else target[b, a]
        assert accepted[b] == a and result[b].tolist() == x[b, :a].tolist() + [int((w / race[b]).argmax())] + [-1] * (drafts - a)
    assert worst <= 2.25, worst
    return {"texts": texts, "accepted": taken, "proposed": batch * steps * drafts, "worst": worst}


def main():
    p = argparse.ArgumentParser(description="Decoding with drafts on a fetched prefix.")
    for name, value in (("batch", 8), ("prefix", 2000), ("drafts", 4), ("steps", 8), ("seed", 0)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--kind", choices=sorted(CODES), default="fp8")
    p.add_argument("--dtype", choices=("bfloat16", "float16"), default="bfloat16")
    args = p.parse_args()
    torch.cuda.set_device(0)
    dl.dl_init(0)
    try:
        r = run(**vars(args))
    finally:
        dl.dl_shutdown()
    new = sum(len(t) for t in r["texts"])
    print(f"{new} tokens in {args.steps} steps of {args.batch} sequences ({r['accepted']} of {r['proposed']} drafts accepted); "
          f"attention within {r['worst']:.2f} units of a dense one")


if __name__ == "__main__":
    main()
