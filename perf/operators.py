"""The operators of a decoding step with drafted tokens over a paged cache in 8 bits, and the cases whose speed counts:
keys and values quantised as they are written into the pages of a cache, the same read back, attention of a batch whose
sequences share a long prefix, and the verification of drafted tokens.

Kinds of case (field "op"):
  write      `tokens` new tokens, `kv_heads` rows of `head_dim` elements of `dtype` each for keys and for values, go to
             scattered slots of a cache of `cache` codes ("fp8" or "int8") with one 32-bit scale per row
  read       as many tokens of such a cache come back as dense rows of `dtype`
  attention  `batch` sequences of `q_tokens` queries each (the last ones of their own tokens) on `q_heads` heads; all share a
             prefix of `prefix` tokens, and each has up to `own` tokens more, fewer from one sequence to the next
  verify     `batch` sequences of `drafts` drafted tokens over a vocabulary of `vocab`; `accept` is the chance by which a draft
             was likely

Plain forms are elementary operations of torch in 32 bits; `exact` computes the same in 64 bits by loops of its own.
"""

import math

import torch

own = False

PAGE = 16                        # tokens of a cache page, as the block copies of this library have them
LIMIT = {"fp8": 448.0, "int8": 127.0}
FLOOR = 2.0 ** -100              # a row's largest magnitude counts as at least this
_TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "f32": 4}
_CODE = {"fp8": torch.float8_e4m3fn, "int8": torch.int8}


def listed():
    return [
        # one decoded token of one sequence: launch-bound
        {"name": "write 1", "op": "write", "tokens": 1, "kv_heads": 8, "head_dim": 128, "page": PAGE, "dtype": "bf16", "cache": "fp8"},
        # a prompt of no particular length as it is prefilled
        {"name": "write 20001", "op": "write", "tokens": 20001, "kv_heads": 8, "head_dim": 128, "page": PAGE, "dtype": "fp16", "cache": "int8"},
        # the last tokens of a few sequences, looked at again
        {"name": "read 240", "op": "read", "tokens": 240, "kv_heads": 4, "head_dim": 64, "page": PAGE, "dtype": "f32", "cache": "int8"},
        # a cached prompt for a pass that wants its keys and values in 16 bits
        {"name": "read 16384", "op": "read", "tokens": 16384, "kv_heads": 8, "head_dim": 128, "page": PAGE, "dtype": "bf16", "cache": "fp8"},
        # one sequence, one token: nothing is shared, the work is split over the length
        {"name": "attn 1x1 own 5000", "op": "attention", "batch": 1, "q_tokens": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": PAGE,
         "prefix": 0, "own": 5000, "dtype": "bf16", "cache": "fp8"},
        # small heads that share nothing, lengths off every grid
        {"name": "attn 5x3 on 777", "op": "attention", "batch": 5, "q_tokens": 3, "q_heads": 12, "kv_heads": 12, "head_dim": 64, "page": PAGE,
         "prefix": 777, "own": 101, "dtype": "fp16", "cache": "int8"},
        # a decode batch behind one system prompt
        {"name": "attn 32x1 on 2048", "op": "attention", "batch": 32, "q_tokens": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": PAGE,
         "prefix": 2048, "own": 300, "dtype": "bf16", "cache": "fp8"},
        # drafted tokens behind a shared document, seven query heads a cache head
        {"name": "attn 48x5 on 16400", "op": "attention", "batch": 48, "q_tokens": 5, "q_heads": 28, "kv_heads": 4, "head_dim": 128, "page": 64,
         "prefix": 16400, "own": 700, "dtype": "fp16", "cache": "int8"},
        # four long conversations: a gigabyte of cache, each byte read once
        {"name": "attn 4x1 own 131072", "op": "attention", "batch": 4, "q_tokens": 1, "q_heads": 64, "kv_heads": 8, "head_dim": 128, "page": PAGE,
         "prefix": 0, "own": 131072, "dtype": "bf16", "cache": "fp8"},
        # many users of one long document: bound by the matrix units
        {"name": "attn 256x1 on 32768", "op": "attention", "batch": 256, "q_tokens": 1, "q_heads": 64, "kv_heads": 8, "head_dim": 128, "page": PAGE,
         "prefix": 32768, "own": 500, "dtype": "bf16", "cache": "fp8"},
        # one sequence's drafts
        {"name": "verify 1x5", "op": "verify", "batch": 1, "drafts": 5, "vocab": 32000, "accept": 0.7, "dtype": "f32"},
        # a decode batch's drafts over a large vocabulary
        {"name": "verify 128x4", "op": "verify", "batch": 128, "drafts": 4, "vocab": 128000, "accept": 0.8, "dtype": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "read", "attention", "attention", "attention", "verify"])
    dim, page = rng.choice([64, 128, 128, 256]), rng.choice([16, 16, 32, 64, 128])
    if op in ("write", "read"):
        return {"op": op, "tokens": _log(rng, 1, 30000), "kv_heads": rng.choice([1, 2, 4, 8, 12]), "head_dim": rng.choice([64, 80, 96, 128, 128]),
                "page": page, "dtype": rng.choice(["bf16", "bf16", "fp16", "f32"]), "cache": rng.choice(["fp8", "int8"])}
    if op == "verify":
        vocab = _log(rng, 1000, 160000)
        return {"op": op, "batch": _log(rng, 1, max(1, min(256, 16000000 // vocab))), "drafts": rng.randint(1, 8), "vocab": vocab,
                "accept": rng.choice([0.5, 0.7, 0.9]), "dtype": rng.choice(["f32", "f32", "bf16", "fp16"])}
    heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8])
    c = {"op": op, "batch": _log(rng, 1, 256), "q_tokens": rng.choice([1, 1, 1, 2, 3, 4, 5, 8]), "q_heads": heads * group, "kv_heads": heads,
         "head_dim": dim, "page": page, "prefix": rng.choice([0, 1, 1]) and _log(rng, 16, 32768)}
    rows = c["batch"] * c["q_tokens"] * c["q_heads"]
    # no more work than the largest listed case, and no more cache than a long one
    most = min(65536, (1 << 19) // c["batch"], (1 << 29) // (c["batch"] * heads * dim))
    c["own"] = max(c["q_tokens"], _log(rng, 1, max(2, most)))
    while rows * dim * (c["prefix"] + c["own"]) > 60e9:
        c["prefix"], c["own"] = c["prefix"] // 2, max(c["q_tokens"], c["own"] // 2)
    c["dtype"], c["cache"] = rng.choice(["bf16", "fp16"]), rng.choice(["fp8", "int8"])
    return c


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(gen, shape, spread=True):
    """N(0, 1); keys also have a few channels that stand out, the same ones in every token."""
    x = torch.randn(shape, dtype=torch.float32, device="cuda", generator=gen)
    if spread:
        x *= 1.0 + 3.0 * (torch.rand(shape[-2:], device="cuda", generator=gen) < 0.05)
    return x


def _lens(case):
    """How many tokens of its own each sequence has: from all of `own` down to its queries alone."""
    n, b = case["own"], case["batch"]
    return [n - (n - case["q_tokens"]) * i // max(1, b - 1) for i in range(b)]


def _quantised(x, kind):
    """Codes and scales of rows, in 32 bits: the formula of the operator."""
    top = x.abs().amax(-1, keepdim=True).clamp_min(FLOOR)
    scaled = x * (LIMIT[kind] / top)
    codes = scaled.to(torch.float8_e4m3fn) if kind == "fp8" else torch.round(scaled).to(torch.int8)
    return codes, (top / LIMIT[kind]).squeeze(-1)


def _cache(gen, case, pages, filled):
    shape = (pages, case["page"], case["kv_heads"], case["head_dim"])
    made = []
    for spread in (True, False):
        if filled:
            codes, scale = _quantised(_rows(gen, shape, spread), case["cache"])
        else:
            codes, scale = torch.zeros(shape, dtype=torch.uint8, device="cuda").view(_CODE[case["cache"]]), torch.zeros(shape[:3], device="cuda")
        made.append((codes, scale))
    return {"k": made[0][0], "k_scale": made[0][1], "v": made[1][0], "v_scale": made[1][1]}


def _inputs(case, seed):
    gen, op, dt = _gen(seed), case["op"], _TORCH[case["dtype"]]
    if op in ("write", "read"):
        T, H, D = case["tokens"], case["kv_heads"], case["head_dim"]
        pages = -(-T // case["page"]) + 2
        s = _cache(gen, case, pages, op == "read")
        # page after page of the pool, in no order; the tokens of one follow each other
        order = torch.randperm(pages, device="cuda", generator=gen)[:-(-T // case["page"])]
        s["slots"] = (order[:, None] * case["page"] + torch.arange(case["page"], device="cuda")).reshape(-1)[:T].contiguous()
        if op == "write":
            s["new_k"], s["new_v"] = _rows(gen, (T, H, D)).to(dt), _rows(gen, (T, H, D), False).to(dt)
        else:
            s["new_k"], s["new_v"] = (torch.zeros((T, H, D), dtype=dt, device="cuda") for _ in range(2))
        return s
    B = case["batch"]
    if op == "verify":
        V, n = case["vocab"], case["drafts"]
        sharp = torch.randn((B, n + 1, V), device="cuda", generator=gen) * 2.0
        # the draft model is near the target by as much as `accept` says
        near = sharp[:, :n] + torch.randn((B, n, V), device="cuda", generator=gen) * (2.0 * (1.0 - case["accept"]))
        s = {"target": torch.softmax(sharp, -1).to(dt), "draft": torch.softmax(near, -1).to(dt)}
        noise = torch.empty((B, n, V), device="cuda").exponential_(generator=gen)
        s["tokens"] = (s["draft"].float() / noise).argmax(-1).to(torch.int32)
        s["uniform"] = torch.rand((B, n), device="cuda", generator=gen)
        s["race"] = torch.empty((B, V), device="cuda").exponential_(generator=gen)
        s["out"] = torch.zeros((B, n + 1), dtype=torch.int32, device="cuda")
        s["accepted"] = torch.zeros((B,), dtype=torch.int32, device="cuda")
        return s
    M, Hq, D, page = case["q_tokens"], case["q_heads"], case["head_dim"], case["page"]
    lens = _lens(case)
    wide, shared = -(-case["own"] // page), -(-case["prefix"] // page)
    pages = B * wide + shared + 3
    s = _cache(gen, case, pages, True)
    order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    s["prefix_pages"], s["pages"] = order[:shared].contiguous(), order[shared:shared + B * wide].view(B, wide).contiguous()
    mixed = torch.randperm(B, device="cuda", generator=gen)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")[mixed].contiguous()
    s["q"] = torch.randn((B, M, Hq, D), device="cuda", generator=gen).to(dt)
    s["out"] = torch.zeros((B, M, Hq, D), dtype=dt, device="cuda")
    s["lse"] = torch.zeros((B, M, Hq), dtype=torch.float32, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2511_06605_amd as dl

        dl.dl_init(0)
        s["dl"], s["stream"] = dl, torch.cuda.current_stream()
        if case["op"] == "verify":
            s["request"] = dl.DraftVerify(s["target"], s["tokens"], s["uniform"], s["race"], s["out"], s["accepted"], draft_probs=s["draft"])
            s["request"].use_workspace(torch.zeros(dl.dl_verify_draft_workspace(s["request"]), dtype=torch.uint8, device="cuda"))
        else:
            s["cache"] = dl.KvCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
            if case["op"] == "attention":
                s["request"] = dl.PrefixAttention(s["cache"], s["q"], s["out"], s["pages"], s["lens"], prefix_pages=s["prefix_pages"],
                                                  prefix_tokens=case["prefix"], lse=s["lse"])
                s["request"].use_workspace(torch.zeros(dl.dl_prefix_attention_workspace(s["request"]), dtype=torch.uint8, device="cuda"))
            else:
                s["request"] = dl.KvRows(s["new_k"], s["new_v"], s["slots"])
    torch.cuda.synchronize()
    return s


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    op = s["case"]["op"]
    if op == "write":
        if own:
            s["dl"].dl_kv_write(s["cache"], s["request"], s["stream"])
        else:
            _plain_write(s)
        return [s["k"], s["k_scale"], s["v"], s["v_scale"]]
    if op == "read":
        if own:
            s["dl"].dl_kv_read(s["cache"], s["request"], s["stream"])
        else:
            _plain_read(s)
        return [s["new_k"], s["new_v"]]
    if op == "attention":
        if own:
            s["dl"].dl_prefix_attention(s["request"], s["stream"])
        else:
            _plain_attention(s)
        return [s["out"], s["lse"]]
    if own:
        s["dl"].dl_verify_draft(s["request"], s["stream"])
    else:
        _plain_verify(s)
    return [s["out"], s["accepted"]]


def _flat(s, what):
    """The codes or scales of a cache by slot."""
    return s[what].flatten(0, 1)


def _put(s, new, to):
    codes, scale = _quantised(s[new].float(), s["case"]["cache"])
    _flat(s, to).view(torch.uint8)[s["slots"]] = codes.view(torch.uint8)
    _flat(s, to + "_scale")[s["slots"]] = scale


def _plain_write(s):
    _put(s, "new_k", "k")
    _put(s, "new_v", "v")


def _values(s, what, slots):
    """What the cache holds at slots, in 32 bits."""
    codes = _flat(s, what).view(torch.uint8)[slots].view(_CODE[s["case"]["cache"]])
    return codes.float() * _flat(s, what + "_scale")[slots].unsqueeze(-1)


def _plain_read(s):
    s["new_k"].copy_(_values(s, "k", s["slots"]))
    s["new_v"].copy_(_values(s, "v", s["slots"]))


def _slots(pages, tokens, page):
    """The slots of the first `tokens` tokens of each row of pages."""
    i = torch.arange(tokens, device="cuda")
    return pages[..., i // page].long() * page + i % page


def _plain_attention(s):
    case = s["case"]
    B, M, Hq, Hk, D = case["batch"], case["q_tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
    G, P, L = Hq // Hk, case["prefix"], case["own"]
    # heads of the cache first: their queries are the rows of one product with the prefix, and of one for each sequence
    q = (s["q"].float() / math.sqrt(D)).view(B, M, Hk, G, D).permute(2, 0, 1, 3, 4).contiguous()
    at = _slots(s["prefix_pages"], P, case["page"])
    k, v = (_values(s, w, at).transpose(0, 1).contiguous() for w in ("k", "v"))
    shared = torch.matmul(q.view(Hk, B * M * G, D), k.transpose(1, 2).contiguous()).view(Hk, B, M * G, P)
    at = _slots(s["pages"], L, case["page"])
    k2, v2 = (_values(s, w, at).permute(2, 0, 1, 3).contiguous() for w in ("k", "v"))
    alone = torch.matmul(q.view(Hk, B, M * G, D), k2.transpose(2, 3).contiguous()).view(Hk, B, M, G, L)
    last = s["lens"][:, None] - M + torch.arange(M, device="cuda")
    seen = (torch.arange(L, device="cuda") <= last[:, :, None])[None, :, :, None]
    alone = alone.masked_fill(~seen, -math.inf).view(Hk, B, M * G, L)
    top = alone.amax(-1, keepdim=True)
    if P:
        top = torch.maximum(top, shared.amax(-1, keepdim=True))
    a, b = torch.exp(shared - top), torch.exp(alone - top)
    total = a.sum(-1, keepdim=True) + b.sum(-1, keepdim=True)
    y = torch.matmul(a.view(Hk, B * M * G, P), v).view(Hk, B, M * G, D) + torch.matmul(b, v2)
    s["out"].copy_((y / total).view(Hk, B, M, G, D).permute(1, 2, 0, 3, 4).reshape(B, M, Hq, D))
    s["lse"].copy_((top + torch.log(total)).view(Hk, B, M, G).permute(1, 2, 0, 3).reshape(B, M, Hq))


def _first_largest(x):
    """The lowest index of each row's largest value."""
    i = torch.arange(x.shape[-1], device=x.device)
    return torch.where(x == x.amax(-1, keepdim=True), i, x.shape[-1]).amin(-1)


def _plain_verify(s):
    p, q, x = s["target"], s["draft"], s["tokens"].long()
    n = x.shape[1]
    px = p[:, :n].gather(2, x[..., None])[..., 0].float()
    qx = q.gather(2, x[..., None])[..., 0].float()
    kept = torch.cumprod((s["uniform"] * qx < px).to(torch.int32), 1)
    a = kept.sum(1)
    row = torch.arange(p.shape[0], device="cuda")
    left = p[row, a].float()
    rest = torch.where((a < n)[:, None], (left - q[row, a.clamp_max(n - 1)].float()).clamp_min(0.0), left)
    rest = torch.where((rest > 0).any(-1, keepdim=True), rest, left)
    chosen = _first_largest(torch.where(rest > 0, rest / s["race"], -1.0))
    chosen = torch.where((rest > 0).any(-1), chosen, -1)
    i = torch.arange(n + 1, device="cuda")
    drafted = torch.cat([x, x.new_zeros((x.shape[0], 1))], 1)
    s["out"].copy_(torch.where(i < a[:, None], drafted, torch.where(i == a[:, None], chosen[:, None], -1)))
    s["accepted"].copy_(a)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    op, size = case["op"], _BYTES[case["dtype"]]
    if op in ("write", "read"):
        rows = 2 * case["tokens"] * case["kv_heads"]
        return {"bytes": rows * (case["head_dim"] * (size + 1) + 4) + 8 * case["tokens"], "flops": 2 * rows * case["head_dim"]}
    if op == "verify":
        # a row of the target and of the race, and one of the draft where one was refused
        n, B, V = case["drafts"], case["batch"], case["vocab"]
        refused = 1.0 - case["accept"] ** n
        return {"bytes": B * V * (size + 4 + size * refused) + B * n * (12 + 2 * size) + B * (n + 2) * 4, "flops": 3 * B * V}
    B, M, Hq, Hk, D = case["batch"], case["q_tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
    alone = sum(_lens(case))
    held = (case["prefix"] + alone) * Hk * 2 * (D + 4) + 4 * (-(-case["prefix"] // case["page"]) + alone // case["page"])
    return {"bytes": held + B * M * Hq * (2 * D * size + 4), "flops": 4 * M * Hq * D * (B * case["prefix"] + alone)}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _exact_rows(x, kind):
    x = x.double()
    top = x.abs().max(-1).values.clamp(min=FLOOR)
    y = x * (LIMIT[kind] / top).unsqueeze(-1)
    if kind == "fp8":
        # three bits behind the first one, down to 2^-9
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).clamp(min=-6.0) - 3.0)
        y = torch.round(y / step) * step
    else:
        y = torch.round(y)
    return y, top / LIMIT[kind]


def exact(case, seed):
    op = case["op"]
    s = _inputs(case, seed)
    if op == "write":
        answer = []
        for new, to in (("new_k", "k"), ("new_v", "v")):
            codes, scale = (t.double() for t in (s[to].float(), s[to + "_scale"]))
            y, z = _exact_rows(s[new], case["cache"])
            page, at = s["slots"] // case["page"], s["slots"] % case["page"]
            codes[page, at], scale[page, at] = y, z
            answer += [codes if case["cache"] == "fp8" else None, scale]
        return answer
    if op == "read":
        page, at = s["slots"] // case["page"], s["slots"] % case["page"]
        return [s[w].float()[page, at].double() * s[w + "_scale"][page, at].double().unsqueeze(-1) for w in ("k", "v")]
    if op == "verify":
        out = torch.full(s["out"].shape, -1, dtype=torch.int64)
        accepted = []
        for b in range(case["batch"]):
            a = 0
            while a < case["drafts"]:
                t = int(s["tokens"][b, a])
                if not float(s["uniform"][b, a]) * float(s["draft"][b, a, t]) < float(s["target"][b, a, t]):
                    break
                out[b, a] = t
                a += 1
            w = s["target"][b, a].double()
            if a < case["drafts"]:
                rest = (w - s["draft"][b, a].double()).clamp(min=0.0)
                w = rest if bool((rest > 0).any()) else w
            out[b, a] = int(torch.argmax(w / s["race"][b].double()))
            accepted.append(a)
        return [out, torch.tensor(accepted)]
    Hk, M, D, page = case["kv_heads"], case["q_tokens"], case["head_dim"], case["page"]
    G = case["q_heads"] // Hk

    def held(what, table, tokens):
        got = s[what][table.long()].float().double() * s[what + "_scale"][table.long()].double().unsqueeze(-1)
        return got.flatten(0, 1)[:tokens].transpose(0, 1)

    kp, vp = (held(w, s["prefix_pages"], case["prefix"]) for w in ("k", "v"))
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        k, v = (torch.cat([p, held(w, s["pages"][b, :-(-n // page)], n)], 1).contiguous() for w, p in (("k", kp), ("v", vp)))
        for j in range(M):
            seen = case["prefix"] + n - M + j + 1
            q = s["q"][b, j].double().view(Hk, G, D) * D ** -0.5
            score = torch.bmm(q, k[:, :seen].transpose(1, 2).contiguous())
            whole = torch.logsumexp(score, -1)
            out[b, j] = torch.bmm(torch.exp(score - whole.unsqueeze(-1)), v[:, :seen].contiguous()).view(Hk * G, D)
            lse[b, j] = whole.view(Hk * G)
    return [out, lse]
