"""The operators that take a prompt into a bounded paged cache in 8 bits, and the cases whose speed counts: queries and keys normed
and rotated by their positions, attention of chunks of new tokens, the weight that cached tokens have been given, and the eviction
of those that were given least.

Kinds of case (field "op"):
  rotate     `tokens` tokens with `q_heads` + `kv_heads` rows of `head_dim` elements of `dtype`: each row is divided by its root mean
             square, multiplied by a weight, and its first `rotary` elements are turned by the angles of the token's position, element i
             with i + rotary / 2, or with its neighbour ("neighbours"); positions lie below `positions`
  chunk      `batch` sequences with up to `chunk` new tokens each behind up to `context` cached ones, fewer from one sequence to the
             next; queries lie packed, sequence behind sequence; causal
  weigh      such queries and their lse: what every cached token has been given by them, over all heads, is added to what it had
  evict      `batch` sequences of up to `context` tokens are cut to `keep`: the `first`, the `recent` and the heaviest of the others move
             to other pages, in order

Plain forms are elementary operations of torch in 32 bits; `exact` computes the same in 64 bits by loops of its own.
"""

import math

import torch

own = False

LIMIT = {"fp8": 448.0, "int8": 127.0}
_TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "f32": 4}
_CODE = {"fp8": torch.float8_e4m3fn, "int8": torch.int8}
EPS = 1e-6
BASE = 500000.0                  # of the rotation's angles
MOST_PAIRS = 2048 * 32 * 32768   # of a query row and a key, in a case


def listed():
    return [
        # a decoding step of one sequence far into its text: launch-bound
        {"name": "rotate 1", "op": "rotate", "tokens": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "rotary": 128, "neighbours": False,
         "positions": 131072, "dtype": "bf16"},
        # a short prompt in 32 bits, part of each row turned, neighbours as pairs
        {"name": "rotate 333", "op": "rotate", "tokens": 333, "q_heads": 12, "kv_heads": 12, "head_dim": 80, "rotary": 32, "neighbours": True,
         "positions": 4096, "dtype": "f32"},
        # a prompt of no particular length
        {"name": "rotate 20001", "op": "rotate", "tokens": 20001, "q_heads": 28, "kv_heads": 4, "head_dim": 128, "rotary": 128,
         "neighbours": False, "positions": 32768, "dtype": "fp16"},
        # a few new tokens of one conversation: latency counts
        {"name": "chunk 1x16 on 500", "op": "chunk", "batch": 1, "chunk": 16, "context": 500, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 16, "dtype": "bf16", "cache": "fp8"},
        # small heads that share nothing, lengths off every grid
        {"name": "chunk 5x101 on 777", "op": "chunk", "batch": 5, "chunk": 101, "context": 777, "q_heads": 12, "kv_heads": 12, "head_dim": 64,
         "page": 16, "dtype": "fp16", "cache": "int8"},
        # questions about long documents, seven query heads a cache head
        {"name": "chunk 3x512 on 16400", "op": "chunk", "batch": 3, "chunk": 512, "context": 16400, "q_heads": 28, "kv_heads": 4,
         "head_dim": 128, "page": 64, "dtype": "fp16", "cache": "int8"},
        # a prompt with nothing in front of it: half of the square
        {"name": "chunk 1x8192 on 0", "op": "chunk", "batch": 1, "chunk": 8192, "context": 0, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 16, "dtype": "bf16", "cache": "fp8"},
        # the last chunk of a long prompt: bound by the matrix units
        {"name": "chunk 1x2048 on 30720", "op": "chunk", "batch": 1, "chunk": 2048, "context": 30720, "q_heads": 32, "kv_heads": 8,
         "head_dim": 128, "page": 16, "dtype": "bf16", "cache": "fp8"},
        # a decoding step of one sequence
        {"name": "weigh 1x1 on 5000", "op": "weigh", "batch": 1, "chunk": 1, "context": 5000, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 16, "dtype": "bf16", "cache": "fp8"},
        # the last queries of several prompts look back before these are cut
        {"name": "weigh 8x32 on 16400", "op": "weigh", "batch": 8, "chunk": 32, "context": 16400, "q_heads": 28, "kv_heads": 4,
         "head_dim": 128, "page": 64, "dtype": "fp16", "cache": "int8"},
        # a few short sequences, small heads
        {"name": "evict 3 of 2001", "op": "evict", "batch": 3, "context": 2001, "keep": 500, "first": 4, "recent": 33, "kv_heads": 4,
         "head_dim": 64, "page": 16, "cache": "int8"},
        # long prompts cut to a quarter
        {"name": "evict 4 of 32768", "op": "evict", "batch": 4, "context": 32768, "keep": 8192, "first": 4, "recent": 256, "kv_heads": 8,
         "head_dim": 128, "page": 16, "cache": "fp8"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "chunk", "chunk", "weigh", "evict"])
    dim, page = rng.choice([64, 80, 96, 128, 128, 128, 256]), rng.choice([16, 16, 32, 64, 128])
    kv = rng.choice([1, 2, 4, 8, 12])
    if op == "rotate":
        return {"op": op, "tokens": _log(rng, 1, 20000), "q_heads": kv * rng.choice([1, 2, 4]), "kv_heads": kv, "head_dim": min(dim, 128),
                "rotary": rng.choice([32, 64, min(dim, 128)]), "neighbours": rng.random() < 0.5, "positions": rng.choice([4096, 32768, 131072]),
                "dtype": rng.choice(["bf16", "fp16", "f32"])}
    kind, dtype = rng.choice(["fp8", "int8"]), rng.choice(["bf16", "fp16"])
    if op == "evict":
        batch, context = _log(rng, 1, 8), _log(rng, 64, 32768)
        while batch * context * kv * dim > 4 * 32768 * 8 * 128:
            batch = max(1, batch - 1)
            context = context * 3 // 4
        keep = max(16, int(context * rng.uniform(0.1, 0.9)))
        return {"op": op, "batch": batch, "context": context, "keep": keep, "first": rng.choice([0, 4]), "recent": rng.randrange(keep // 2 + 1),
                "kv_heads": kv, "head_dim": dim, "page": page, "cache": kind}
    batch, group = _log(rng, 1, 16), rng.choice([1, 4, 5, 7, 8])
    chunk, context = (_log(rng, 1, 4096) if op == "chunk" else _log(rng, 1, 64)), _log(rng, 1, 32768)
    while batch * chunk * group * kv * (chunk + context) > MOST_PAIRS * min(1.0, 128 / dim) or batch * (chunk + context) * kv * dim > 1 << 28:
        batch, chunk, context = max(1, batch - 1), max(1, chunk * 7 // 8), context * 7 // 8
    return {"op": op, "batch": batch, "chunk": chunk, "context": context, "q_heads": kv * group, "kv_heads": kv, "head_dim": dim, "page": page,
            "dtype": dtype, "cache": kind}


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(gen, shape, spread=True):
    """N(0, 1); keys also have a few channels that stand out, the same ones in every token."""
    x = torch.randn(shape, dtype=torch.float32, device="cuda", generator=gen)
    if spread:
        x *= 1.0 + 3.0 * (torch.rand(shape[-2:], device="cuda", generator=gen) < 0.05)
    return x


def _sizes(case):
    """(new tokens, all tokens) of each sequence: from all of `chunk` and `context` down to a third of either."""
    b = case["batch"]
    part = [1.0 - 2.0 * i / (3.0 * max(1, b - 1)) for i in range(b)]
    new = [max(1, int(case.get("chunk", 0) * p)) for p in part] if case["op"] != "evict" else [0] * b
    # (contexts shrink the other way round)
    return [(n, n + int(case["context"] * p)) for n, p in zip(new, reversed(part))]


def _cache(gen, case, pages):
    shape = (pages, case["page"], case["kv_heads"], case["head_dim"])
    made = []
    for spread in (True, False):
        x = _rows(gen, shape, spread)
        top = x.abs().amax(-1, keepdim=True)
        scaled = x * (LIMIT[case["cache"]] / top)
        codes = scaled.to(torch.float8_e4m3fn) if case["cache"] == "fp8" else torch.round(scaled).to(torch.int8)
        made.append((codes, (top / LIMIT[case["cache"]]).squeeze(-1)))
    return {"k": made[0][0], "k_scale": made[0][1], "v": made[1][0], "v_scale": made[1][1]}


def _rotate_inputs(case, gen):
    T, D, R, dt = case["tokens"], case["head_dim"], case["rotary"], _TORCH[case["dtype"]]
    s = {"q": _rows(gen, (T, case["q_heads"], D)).to(dt), "k": _rows(gen, (T, case["kv_heads"], D)).to(dt)}
    s["q_weight"], s["k_weight"] = (1.0 + 0.2 * torch.randn(D, device="cuda", generator=gen) for _ in range(2))
    # the cosines and sines of every position, as a program keeps them
    angle = torch.arange(case["positions"], device="cuda", dtype=torch.float64)[:, None] * BASE ** (
        -torch.arange(R // 2, device="cuda", dtype=torch.float64) / (R // 2))
    s["table"] = torch.cat([torch.cos(angle), torch.sin(angle)], 1).float()
    # the tokens of a chunk of a text, or of several
    first = torch.randint(case["positions"], (1,), device="cuda", generator=gen)
    s["positions"] = (first + torch.arange(T, device="cuda")) % case["positions"]
    s["q_out"], s["k_out"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"])
    return s


def _inputs(case, seed):
    gen = _gen(seed)
    if case["op"] == "rotate":
        return _rotate_inputs(case, gen)
    B, page, Hk, D = case["batch"], case["page"], case["kv_heads"], case["head_dim"]
    sizes = _sizes(case)
    wide = max(-(-n // page) for _, n in sizes)
    evict = case["op"] == "evict"
    more = -(-case["keep"] // page) if evict else 0
    s = _cache(gen, case, B * (wide + more) + 3)
    order = torch.randperm(B * (wide + more) + 3, device="cuda", generator=gen).to(torch.int32)
    s["pages"] = order[:B * wide].view(B, wide).contiguous()
    s["lens"] = torch.tensor([n for _, n in sizes], dtype=torch.int32, device="cuda")
    if evict:
        s["to_pages"] = order[B * wide:B * (wide + more)].view(B, more).contiguous()
        # a few tokens get most of the weight
        s["weights"] = torch.exp(2.0 * torch.randn((B, wide * page), device="cuda", generator=gen))
        s["kept"] = torch.zeros((B, case["keep"]), dtype=torch.int32, device="cuda")
        s["kept_lens"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["kept_weights"] = torch.zeros((B, case["keep"]), device="cuda")
        return s
    starts = [0]
    for new, _ in sizes:
        starts.append(starts[-1] + new)
    s["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    shape = (starts[-1], case["q_heads"], D)
    s["q"] = torch.randn(shape, device="cuda", generator=gen).to(_TORCH[case["dtype"]])
    s["lse"] = torch.zeros(shape[:2], device="cuda")
    if case["op"] == "chunk":
        s["out"] = torch.zeros_like(s["q"])
    else:
        s["before"] = torch.rand((B, wide * page), device="cuda", generator=gen)
        s["weights"] = torch.zeros_like(s["before"])
        s["lse"].copy_(torch.logsumexp(_scores(s, case), -1).permute(0, 2, 1, 3).flatten(2)[_sequence_and_row(s)])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2511_06605_amd as dl

        dl.dl_init(0)
        s["dl"], s["stream"] = dl, torch.cuda.current_stream()
        workspace = None
        if case["op"] == "rotate":
            s["request"] = dl.NormRotate(s["q"], s["k"], s["q_out"], s["k_out"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                                         table=s["table"], positions=s["positions"], neighbours=case["neighbours"])
        else:
            cache = dl.KvCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
            if case["op"] == "chunk":
                s["request"] = dl.ChunkAttention(cache, s["q"], s["out"], s["starts"], s["pages"], s["lens"], lse=s["lse"])
                workspace = dl.dl_chunk_attention_workspace
            elif case["op"] == "weigh":
                s["request"] = dl.KvWeigh(cache, s["q"], s["lse"], s["starts"], s["pages"], s["lens"], s["weights"], before=s["before"])
                workspace = dl.dl_kv_weigh_workspace
            else:
                s["request"] = dl.KvEvict(cache, s["weights"], s["pages"], s["lens"], s["to_pages"], s["kept"], s["kept_lens"],
                                          kept_weights=s["kept_weights"], first=case["first"], recent=case["recent"])
                workspace = dl.dl_kv_evict_workspace
        if workspace:
            s["request"].use_workspace(torch.zeros(workspace(s["request"]), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    return s


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    op = s["case"]["op"]
    if op == "rotate":
        if own:
            s["dl"].dl_norm_rotate(s["request"], s["stream"])
        else:
            _plain_rotate(s)
        return [s["q_out"], s["k_out"]]
    if op == "chunk":
        if own:
            s["dl"].dl_chunk_attention(s["request"], s["stream"])
        else:
            _plain_chunk(s)
        return [s["out"], s["lse"]]
    if op == "weigh":
        if own:
            s["dl"].dl_kv_weigh(s["request"], s["stream"])
        else:
            _plain_weigh(s)
        return [s["weights"]]
    if own:
        s["dl"].dl_kv_evict(s["request"], s["stream"])
    else:
        _plain_evict(s)
    return [s["kept"], s["kept_lens"], s["kept_weights"], s["k"], s["k_scale"], s["v"], s["v_scale"]]


def _plain_rotate(s):
    case = s["case"]
    R = case["rotary"]
    c, z = s["table"][s["positions"]][:, None].chunk(2, -1)
    for name in ("q", "k"):
        x = s[name].float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s[name + "_weight"]
        if case["neighbours"]:
            a, b = y[..., 0:R:2], y[..., 1:R:2]
            turned = torch.stack([a * c - b * z, b * c + a * z], -1).flatten(-2)
        else:
            a, b = y[..., :R // 2], y[..., R // 2:R]
            turned = torch.cat([a * c - b * z, b * c + a * z], -1)
        s[name + "_out"].copy_(torch.cat([turned, y[..., R:]], -1))


def _values(s, what, slots):
    """What the cache holds at slots, in 32 bits."""
    codes = s[what].flatten(0, 1).view(torch.uint8)[slots].view(s[what].dtype)
    return codes.float() * s[what + "_scale"].flatten(0, 1)[slots].unsqueeze(-1)


def _slots(pages, page):
    """The slots of all places of each row of pages."""
    return (pages.long()[:, :, None] * page + torch.arange(page, device=pages.device)).flatten(1)


def _sequence_and_row(s):
    """Of every packed query: its sequence, and which of its queries it is."""
    t = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(s["starts"][1:], t, right=True)
    return b, t - s["starts"].long()[b]


def _scores(s, case):
    """[batch, heads of the cache, new tokens, query heads of one, tokens], with -inf where nothing is seen."""
    Hk, D, M = case["kv_heads"], case["head_dim"], case["chunk"]
    G = case["q_heads"] // Hk
    starts, lens = s["starts"].long(), s["lens"].long()
    B, new = lens.shape[0], starts.diff()
    j = torch.arange(M, device="cuda")
    rows = (starts[:-1, None] + j).clamp_max(s["q"].shape[0] - 1)
    q = (s["q"][rows].float() / math.sqrt(D)).view(B, M, Hk, G, D).transpose(1, 2).reshape(B, Hk, M * G, D)
    k = _values(s, "k", _slots(s["pages"], case["page"])).permute(0, 2, 3, 1).contiguous()
    scores = torch.matmul(q, k).view(B, Hk, M, G, -1)
    # (rows behind a sequence's last query see what the last one sees)
    last = (lens - new)[:, None] + torch.minimum(j, new[:, None] - 1)
    unseen = torch.arange(scores.shape[-1], device="cuda") > last[:, :, None]
    return scores.masked_fill_(unseen[:, None, :, None], -math.inf)


def _plain_chunk(s):
    case = s["case"]
    at = _sequence_and_row(s)
    p = _scores(s, case)
    B, Hk, M, G, L = p.shape
    top = p.amax(-1, keepdim=True)
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = _values(s, "v", _slots(s["pages"], case["page"])).transpose(1, 2).contiguous()
    y = torch.matmul(p.view(B, Hk, M * G, L), v).view(B, Hk, M, G, -1) / total
    s["out"].copy_(y.transpose(1, 2).flatten(2, 3)[at])
    s["lse"].copy_((top + torch.log(total)).transpose(1, 2).reshape(B, M, Hk * G)[at])


def _plain_weigh(s):
    case = s["case"]
    p = _scores(s, case)
    B, Hk, M, G, L = p.shape
    new = s["starts"].long().diff()
    j = torch.arange(M, device="cuda")
    rows = (s["starts"].long()[:-1, None] + j).clamp_max(s["q"].shape[0] - 1)
    lse = s["lse"][rows].view(B, M, Hk, G).transpose(1, 2)
    p = p.sub_(lse.unsqueeze(-1)).exp_()
    p = p.mul_((j < new[:, None])[:, None, :, None, None])
    s["weights"].copy_(s["before"] + p.sum((1, 2, 3)))


def _plain_evict(s):
    case = s["case"]
    n, keep, page = s["lens"].long()[:, None], case["keep"], case["page"]
    i = torch.arange(s["weights"].shape[1], device="cuda")
    # the first and the recent ones are heavier than all others, what lies behind the end is lighter; equal ones by their index
    w = s["weights"].masked_fill((i < case["first"]) | (i >= n - case["recent"]), math.inf).masked_fill(i >= n, -math.inf)
    order = torch.sort(w, dim=1, descending=True, stable=True).indices[:, :keep]
    chosen = torch.zeros(w.shape, dtype=torch.bool, device="cuda").scatter_(1, order, True) & (i < n)
    # in order: the index where it is chosen, and a number behind them all where it is not
    kept = torch.sort(torch.where(chosen, i, i.numel()), dim=1).values[:, :keep]
    there = kept < i.numel()
    at = kept.clamp_max(i.numel() - 1)
    s["kept"].copy_(torch.where(there, kept, -1))
    s["kept_lens"].copy_(n[:, 0].clamp_max(keep))
    s["kept_weights"].copy_(torch.where(there, s["weights"].gather(1, at), 0.0))
    source = _slots(s["pages"], page).gather(1, at)
    to = _slots(s["to_pages"], page)[:, :keep]
    for name in ("k", "v", "k_scale", "v_scale"):
        held = s[name].flatten(0, 1)
        held = held if held.dtype == torch.float32 else held.view(torch.uint8)
        mask = there.view(*there.shape, *[1] * (held.dim() - 1))
        held[to] = torch.where(mask, held[source], held[to])


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    op, D = case["op"], case["head_dim"]
    if op == "rotate":
        T, R, rows = case["tokens"], case["rotary"], case["tokens"] * (case["q_heads"] + case["kv_heads"])
        return {"bytes": 2 * rows * D * _BYTES[case["dtype"]] + min(T, case["positions"]) * R * 4 + 8 * T + 8 * D, "flops": rows * (4 * D + 3 * R)}
    sizes, Hk = _sizes(case), case["kv_heads"]
    token = Hk * (D + 4)  # one side of the cache
    if op == "evict":
        kept = [min(n, case["keep"]) for _, n in sizes]
        return {"bytes": 4 * sum(n for _, n in sizes) + sum(kept) * (4 * token + 8 + 4) + 4 * case["batch"] * case["keep"],
                "flops": sum(n for _, n in sizes)}
    pairs = sum(new * (n - new) + new * (new + 1) // 2 for new, n in sizes) * case["q_heads"]
    new, held = sum(m for m, _ in sizes), sum(n for _, n in sizes)
    if op == "weigh":
        return {"bytes": held * (token + 8) + new * case["q_heads"] * (D * _BYTES[case["dtype"]] + 4), "flops": 2 * pairs * D}
    return {"bytes": held * 2 * token + new * case["q_heads"] * (2 * D * _BYTES[case["dtype"]] + 4), "flops": 4 * pairs * D}


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "rotate":
        return [_exact_rotate(s, case, name) for name in ("q", "k")]
    if op == "evict":
        return _exact_evict(s, case)
    Hk, D = case["kv_heads"], case["head_dim"]
    G = case["q_heads"] // Hk
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    if op == "chunk":
        out, lse = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    else:
        weights = s["before"].double()
    for b, n in enumerate(lens):
        table = s["pages"][b, :-(-n // case["page"])].long()
        k, v = (((s[w][table].float().double() * s[w + "_scale"][table].double()[..., None]).flatten(0, 1)[:n]) for w in ("k", "v"))
        new = starts[b + 1] - starts[b]
        for h in range(Hk):
            # (a few queries at a time, for the memory that their scores take)
            for j in range(0, new, 512):
                many = min(512, new - j)
                at, heads = slice(starts[b] + j, starts[b] + j + many), slice(h * G, h * G + G)
                q = s["q"][at, heads].double().reshape(many * G, D)
                score = torch.mm(q, k[:, h].t().contiguous()).view(many, G, n) / math.sqrt(D)
                hidden = torch.ones((many, n), dtype=torch.bool, device="cuda").triu(n - new + j + 1)
                score.masked_fill_(hidden[:, None], -math.inf)
                if op == "chunk":
                    whole = torch.logsumexp(score, -1)
                    out[at, heads] = torch.mm(torch.exp(score - whole[..., None]).view(many * G, n), v[:, h].contiguous()).view(many, G, D)
                    lse[at, heads] = whole
                else:
                    weights[b, :n] += torch.exp(score - s["lse"][at, heads].double()[..., None]).sum((0, 1))
    return [out, lse] if op == "chunk" else [weights]


def _exact_rotate(s, case, name):
    x, R = s[name].double(), case["rotary"]
    size = torch.sqrt(x.pow(2).sum(-1) / case["head_dim"] + EPS)
    y = x / size[..., None] * s[name + "_weight"].double()
    angles = s["table"].double()[s["positions"]]
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if case["neighbours"] else (i, i + R // 2)
        turn = torch.complex(angles[:, i], angles[:, R // 2 + i])[:, None] * torch.complex(y[..., a], y[..., b])
        y[..., a], y[..., b] = turn.real, turn.imag
    return y


def _exact_evict(s, case):
    page, keep = case["page"], case["keep"]
    kept = torch.full(s["kept"].shape, -1, dtype=torch.int64)
    weights = torch.zeros(s["kept_weights"].shape, dtype=torch.float64)
    lens = []
    cache = [s["k"].float(), s["k_scale"].clone(), s["v"].float(), s["v_scale"].clone()]
    for b, n in enumerate(s["lens"].tolist()):
        w = s["weights"][b].tolist()
        fixed = set(range(min(case["first"], n))) | set(range(max(0, n - case["recent"]), n))
        others = sorted((i for i in range(n) if i not in fixed), key=lambda i: (-w[i], i))
        stay = sorted(list(fixed) + others[:max(0, keep - len(fixed))])
        lens.append(len(stay))
        kept[b, :len(stay)] = torch.tensor(stay)
        weights[b, :len(stay)] = torch.tensor([w[i] for i in stay], dtype=torch.float64)
        i, j = torch.tensor(stay, device="cuda"), torch.arange(len(stay), device="cuda")
        for x in cache:
            x[s["to_pages"][b].long()[j // page], j % page] = x[s["pages"][b].long()[i // page], i % page]
    return [kept, torch.tensor(lens), weights] + [x.double() if x.dim() == 3 or case["cache"] == "fp8" else x.to(torch.int8) for x in cache]
