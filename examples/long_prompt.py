"""A long prompt in a bounded cache: how the operators that take a prompt into a paged cache work together.

    python examples/long_prompt.py [--batch 2] [--prompt 1500] [--chunk 400] [--keep 512] [--kind fp8|int8] [--dtype bfloat16|float16]

The prompts of a batch come in chunks.  Of each chunk, queries and keys are normed and rotated by their positions (dl_norm_rotate, in place),
keys and values go into the pages of the cache (dl_kv_write), and the chunk attends to all that lies there (dl_chunk_attention).  The last
chunk's last queries then say what each token of the prompt has been given (dl_kv_weigh); the tokens that were given least are left
behind (dl_kv_evict), the pages of the whole prompt are free again, and one token is decoded on what was kept (dl_prefix_attention).

Each step is checked against a dense one in float32 over what dl_kv_read gives back.
"""

from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2511_06605_amd as dl  # noqa: E402

CODES = {"fp8": torch.float8_e4m3fn, "int8": torch.int8}
EPS = 1e-6


def slots_of(table, tokens, page):
    """Slots of the tokens `tokens` [n] of a sequence with the page table `table` [pages]."""
    return table.long()[tokens // page] * page + tokens % page


def weights_of(q, k, visible):
    """q [M, H, D], k [n, heads, D] of float32, visible [M, n]: attention weights [M, H, n] and their lse, as the formula says it."""
    k = k.repeat_interleave(q.shape[1] // k.shape[1], 1)
    s = torch.stack([q[:, h] @ k[:, h].T.contiguous() for h in range(q.shape[1])], 1) * q.shape[2] ** -0.5
    s = s.masked_fill(~visible[:, None], float("-inf"))
    return torch.softmax(s, -1), torch.logsumexp(s, -1)


def dense(q, k, v, visible):
    p, _ = weights_of(q, k, visible)
    v = v.repeat_interleave(q.shape[1] // v.shape[1], 1)
    return torch.stack([p[:, h] @ v[:, h].contiguous() for h in range(q.shape[1])], 1)


def turned(x, weight, table, positions):
    """Norm and rotation of rows x [T, H, D] of float32."""
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight
    c, s = table[positions][:, None].chunk(2, -1)
    a, b = y.chunk(2, -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def run(batch=2, prompt=1500, chunk=400, keep=512, window=16, first=4, recent=32, kind="fp8", dtype="bfloat16", q_heads=8, heads=2, dim=64, page=16, seed=0):
    name, dtype = dtype, getattr(torch, dtype)
    unit = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[name]
    stream = torch.cuda.current_stream()
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, device="cuda", generator=g)  # noqa: E731
    lens = [max(1, prompt - 177 * b) for b in range(batch)]  # prompts of different lengths
    # pages of a pool, handed out in no particular order: for the prompts, and for what is kept of them (and one token more)
    wide, kept_wide = -(-prompt // page), -(-(keep + 1) // page)
    shape = (batch * (wide + kept_wide), page, heads, dim)
    codes = [torch.zeros(shape, dtype=torch.uint8, device="cuda").view(CODES[kind]) for _ in range(2)]
    scales = [torch.zeros(shape[:3], device="cuda") for _ in range(2)]
    cache = dl.KvCache(*codes, *scales)
    free = torch.randperm(shape[0], device="cuda", generator=g).int()
    pages, kept_pages = free[:batch * wide].view(batch, wide).contiguous(), free[batch * wide:].view(batch, kept_wide).contiguous()
    angle = torch.arange(prompt + 1, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(dim // 2, device="cuda") / (dim / 2))
    table = torch.cat([torch.cos(angle), torch.sin(angle)], 1).float()
    q_weight, k_weight = 1 + 0.1 * rand(dim), 1 + 0.1 * rand(dim)

    def write(k, v, tables, positions, sequence):
        slots = torch.cat([slots_of(tables[b], positions[sequence == b], page) for b in range(batch)])
        dl.dl_kv_write(cache, dl.KvRows(k, v, slots), stream)

    def read(table, n):
        k, v = (torch.empty((n, heads, dim), device="cuda") for _ in range(2))
        dl.dl_kv_read(cache, dl.KvRows(k, v, slots_of(table, torch.arange(n, device="cuda"), page)), stream)
        return k, v

    def rows(n):
        return (rand(n, q_heads, dim).to(dtype), rand(n, heads, dim).to(dtype), rand(n, heads, dim).to(dtype))

    workspace = torch.zeros(1, dtype=torch.uint8, device="cuda")

    def with_workspace(request, size):
        nonlocal workspace
        if workspace.numel() < size(request):
            workspace = torch.zeros(size(request), dtype=torch.uint8, device="cuda")
        request.use_workspace(workspace)
        return request

    # chunk by chunk
    worst = {"norm": 0.0, "chunk": 0.0, "weights": 0.0, "decode": 0.0}
    done, last = [0] * batch, {}
    while done != lens:
        new = [min(chunk, n - d) for n, d in zip(lens, done)]
        starts = torch.tensor([sum(new[:b]) for b in range(batch + 1)], dtype=torch.int32, device="cuda")
        positions = torch.cat([torch.arange(d, d + m, device="cuda") for d, m in zip(done, new)])
        sequence = torch.cat([torch.full((m,), b, device="cuda") for b, m in enumerate(new)])
        done = [d + m for d, m in zip(done, new)]
        held = torch.tensor(done, dtype=torch.int32, device="cuda")
        q, k, v = rows(sum(new))
        want = turned(q.float(), q_weight, table, positions)
        dl.dl_norm_rotate(dl.NormRotate(q, k, q_weight=q_weight, k_weight=k_weight, eps=EPS, table=table, positions=positions), stream)
        worst["norm"] = max(worst["norm"], float(((q.float() - want).abs() / (unit * want.abs() + 2.0 ** -18 * want.abs().amax())).max()))
        write(k, v, pages, positions, sequence)
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        dl.dl_chunk_attention(with_workspace(dl.ChunkAttention(cache, q, out, starts, pages, held, lse=lse), dl.dl_chunk_attention_workspace), stream)
        for b, (n, m) in enumerate(zip(done, new)):
            if m:
                mine = sequence == b
                kb, vb = read(pages[b], n)
                sees = torch.arange(n, device="cuda") <= n - m + torch.arange(m, device="cuda")[:, None]
                off = (dense(q[mine].float(), kb, vb, sees) - out[mine].float()).abs().max() / vb.abs().max()
                worst["chunk"] = max(worst["chunk"], float(off) / unit)
                last[b] = q[mine][-window:], lse[mine][-window:]

    # what the last queries of each prompt gave to its tokens, and the cut
    q, lse = (torch.cat([last[b][i] for b in range(batch)]).contiguous() for i in range(2))
    new = [last[b][0].shape[0] for b in range(batch)]
    starts = torch.tensor([sum(new[:b]) for b in range(batch + 1)], dtype=torch.int32, device="cuda")
    held = torch.tensor(lens, dtype=torch.int32, device="cuda")
    weights = torch.empty((batch, wide * page), device="cuda")
    dl.dl_kv_weigh(with_workspace(dl.KvWeigh(cache, q, lse, starts, pages, held, weights), dl.dl_kv_weigh_workspace), stream)
    kept, kept_lens = torch.empty((batch, keep), dtype=torch.int32, device="cuda"), torch.empty(batch, dtype=torch.int32, device="cuda")
    # (of the pages for what is kept, those that the tokens of the prompt need)
    dl.dl_kv_evict(with_workspace(dl.KvEvict(cache, weights, pages, held, kept_pages[:, :-(-keep // page)], kept, kept_lens, first=first, recent=recent),
                                  dl.dl_kv_evict_workspace), stream)
    for b, (n, m) in enumerate(zip(lens, new)):
        kb, vb = read(pages[b], n)
        sees = torch.arange(n, device="cuda") <= n - m + torch.arange(m, device="cuda")[:, None]
        p, _ = weights_of(q[starts[b]:starts[b + 1]].float(), kb, sees)
        want = p.sum((0, 1))
        worst["weights"] = max(worst["weights"], float((weights[b, :n] - want).abs().max() / want.max()))
        stays = min(n, keep)
        assert int(kept_lens[b]) == stays and not weights[b, n:].any()
        chosen = kept[b, :stays].long()
        assert bool((chosen[1:] > chosen[:-1]).all()) and (kept[b, stays:] == -1).all()
        kk, vv = read(kept_pages[b], stays)
        assert torch.equal(kk, kb[chosen]) and torch.equal(vv, vb[chosen])
        if n > keep:
            left = torch.ones(n, dtype=torch.bool, device="cuda")
            left[chosen] = False
            fixed = torch.zeros(n, dtype=torch.bool, device="cuda")
            fixed[:first], fixed[n - recent:] = True, True
            assert bool(~left[fixed].any()) and weights[b, :n][left].max() <= weights[b, :n][~left & ~fixed].min()

    # one token more, on what was kept: its place in the pages is the next one, its position that behind the prompt
    q, k, v = rows(batch)
    dl.dl_norm_rotate(dl.NormRotate(q, k, q_weight=q_weight, k_weight=k_weight, eps=EPS, table=table, positions=held.long()), stream)
    write(k, v, kept_pages, kept_lens.long(), torch.arange(batch, device="cuda"))
    kept_lens += 1
    out = torch.empty_like(q)
    dl.dl_prefix_attention(with_workspace(dl.PrefixAttention(cache, q[:, None], out[:, None], kept_pages, kept_lens), dl.dl_prefix_attention_workspace), stream)
    for b in range(batch):
        kb, vb = read(kept_pages[b], int(kept_lens[b]))
        off = (dense(q[b:b + 1].float(), kb, vb, torch.ones((1, kb.shape[0]), dtype=torch.bool, device="cuda")) - out[b].float()).abs().max() / vb.abs().max()
        worst["decode"] = max(worst["decode"], float(off) / unit)
    # A rounding of the weights and one of the output are a unit each of the largest |v|, of the normed rows one (and 2^-18 of the largest for
    # 32-bit steps, the formula's own here among them); weights have the 32-bit errors of scores of some tens on both sides.
    assert worst["norm"] <= 1.0 and worst["chunk"] <= 2.25 and worst["decode"] <= 2.25 and worst["weights"] <= 2.0 ** -13, worst
    return {"lens": lens, "kept": [int(n) - 1 for n in kept_lens], "worst": worst}


def main():
    p = argparse.ArgumentParser(description="A long prompt in a bounded cache.")
    for name, value in (("batch", 2), ("prompt", 1500), ("chunk", 400), ("keep", 512), ("seed", 0)):
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
    print(f"prompts of {r['lens']} tokens cut to {r['kept']}; attention within {max(r['worst']['chunk'], r['worst']['decode']):.2f} units of a dense one")


if __name__ == "__main__":
    main()
