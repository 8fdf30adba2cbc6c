"""Performance cases of a decoding or prefill step's operators around a paged KV cache: one call each, as a serving
replica makes it per layer.

* ``rotate``: queries and keys are normed for each head and rotated by their position in one pass; the keys, with the
  values, go into the cache's pages;
* ``append``: new rows go into e4m3 pages that have a scale, a power of two, for each page, K or V, and head;
* ``attend``: attention over such pages, from one new token per sequence to the tail of a prompt;
* ``bounds``: of each page the lowest and highest K in every column, for the pages that a call's tokens lie in;
* ``score``: from these, what a page's best token can score at most with each new token's queries;
* ``pages``: attention of each new token over the pages that it chose, and no others.

A case names the operator, the layout of the cache (``H`` KV heads, ``G`` query heads for each, ``D``, ``BS`` tokens a
page, ``nhd`` for token-major pages), the types (``fp8``: e4m3 pages) and the sizes.  Of ``seqs`` sequences the longest has
``longest`` tokens and, of these, ``queries`` new ones; in a ``ragged`` batch the others spread below that.  ``budget``:
pages that a new token chooses.

``run`` gives the plain form, in 32 bits, or with ``own`` the framework's call.
"""
import math

import torch

own = False

DEVICE = "cuda:0"

# Layouts, as in the cases of stores and loads: the 27B-class GQA layout (and one rank of a 4-way shard of it), the FP8
# attention layers of the shared-cache deployment with their 32-token pages, and the smallest that the tests use.
B27 = dict(H=8, D=128, BS=16, nhd=False, fp8=False)
SHARD4 = dict(B27, H=2)
PAPER = dict(H=4, D=256, BS=32, nhd=True, fp8=True)
TINY = dict(H=2, D=64, BS=16, nhd=False, fp8=False)

_EPS = 1e-6
_K_SCALE, _V_SCALE = 0.037, 0.021  # of rotated rows in e4m3 pages


def _case(name, op, layout, seqs, longest, **changes):
    return dict(dict(layout, G=1, dtype="bfloat16", queries=1, ragged=True), **changes, name=name, op=op, seqs=seqs,
                longest=longest)


def _rotate(name, layout, seqs, longest, **changes):
    return _case(name, "rotate", layout, seqs, longest,
                 **dict(dict(rotary=layout["D"], interleaved=False, norm=True, moved=0), **changes))


def _attend(name, layout, seqs, longest, **changes):
    return _case(name, "attend", layout, seqs, longest, **dict(dict(softcap=0.0, window=0, slopes=False), **changes))


def listed():
    return [
        # The smallest calls, where latency counts: a decoding step of three short sequences, rotated in pairs of
        # neighbours, behind tokens that a compaction has moved.
        _rotate("rotate_tiny_step", TINY, 3, 100, G=2, dtype="float16", interleaved=True, moved=1000),
        # A session turn: the 2,048 + 37 new tokens behind a 32k prefix.
        _rotate("rotate_27b_turn", B27, 1, 32768 + 2048 + 37, G=5, queries=2048 + 37),
        # A ragged batch decodes into scaled pages: a row each, and now and then a page whose scale grows.
        _case("append_paper_step", "append", PAPER, 48, 8192, G=6),
        # The tails of four prompts behind restored prefixes (1,055 new tokens, one session turn, in the longest).
        _case("append_paper_tails", "append", PAPER, 4, 8192 + 1055, G=6, queries=1055),
        # A ragged batch decodes from scaled pages.
        _attend("attend_paper_batch", PAPER, 16, 32768, G=6),
        # The tails of several prompts together, the largest amount of arithmetic.
        _attend("attend_paper_tails", PAPER, 6, 8192 + 1055, G=6, queries=1055),
        # The bounds of a restored prefix of 128k tokens, and those that a decoding batch's new tokens move.
        _case("bounds_27b_prefix", "bounds", B27, 1, 131072 + 5, G=5, queries=131072 + 5),
        _case("bounds_paper_step", "bounds", PAPER, 48, 8192, G=6),
        # One sequence decodes behind a 128k-token prefix; the tails of three prompts choose pages for every token.
        _case("score_27b_128k", "score", B27, 1, 131072 + 5, G=5),
        _case("score_shard4_tails", "score", SHARD4, 3, 16384 + 517, G=8, queries=517),
        # These attend over what they chose: 4,096 of the 128k tokens; 2,048 tokens each of a ragged batch.
        _case("pages_27b_128k", "pages", B27, 1, 131072 + 5, G=5, budget=256),
        _case("pages_shard4_batch", "pages", SHARD4, 48, 16384, G=8, budget=128),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# What a drawn case has at most: bytes of K (or V) rows in 32 bits, scores in 32 bits, operations, and chosen (row,
# page) pairs.
_MOST_ROWS, _MOST_SCORES, _MOST_FLOPS, _MOST_CHOSEN = 1 << 30, 4 << 30, 3 * 10**11, 1 << 18


def draw(rng):
    op = rng.choice(["rotate", "rotate", "append", "attend", "attend", "bounds", "score", "pages", "pages"])
    while True:
        c = dict(op=op, H=rng.choice([1, 2, 3, 4, 8]), G=rng.choice([1, 2, 4, 5, 6, 8, 12, 16]),
                 D=rng.choice([64, 80, 96, 128, 128, 192, 256]), BS=rng.choice([8, 16, 16, 24, 32, 64]),
                 nhd=rng.random() < 0.4, fp8=op in ("append", "attend") or rng.random() < 0.35,
                 dtype=rng.choice(["bfloat16", "bfloat16", "float16"]), seqs=_log_uniform(rng, 1, 64),
                 longest=_log_uniform(rng, 1, 131072), ragged=rng.random() < 0.7, queries=1)
        if rng.random() < 0.5:
            c["queries"] = min(c["longest"], _log_uniform(rng, 2, 200 if op == "pages" else 4096))
        if op == "bounds" and rng.random() < 0.5:
            c["queries"] = c["longest"]  # of a restored prefix
        if op == "rotate":
            c.update(rotary=rng.choice([c["D"], c["D"], c["D"] // 2, 20]), interleaved=rng.random() < 0.3,
                     norm=rng.random() < 0.7, moved=rng.choice([0, 0, 1000, 500000]))
        if op == "attend":
            c.update(softcap=rng.choice([0.0, 0.0, 30.0, 50.0]), window=rng.choice([0, 0, 0, 512, 4096]),
                     slopes=rng.random() < 0.25)
        if op == "pages":
            c["budget"] = _log_uniform(rng, 1, 512)
        rows = c["seqs"] * c["longest"] * c["H"]
        if rows * c["D"] * 4 > _MOST_ROWS or work(c)["flops"] > _MOST_FLOPS:
            continue
        if op == "attend" and rows * c["queries"] * c["G"] * 4 > _MOST_SCORES:
            continue
        if op == "score" and rows // c["BS"] * c["queries"] * c["G"] * 4 > _MOST_SCORES:
            continue
        if op == "pages":
            chosen = sum(_sizes(c)[1]) * c["H"] * c["budget"]
            if chosen > _MOST_CHOSEN or chosen * c["BS"] * c["D"] * 4 > _MOST_ROWS or sum(_sizes(c)[1]) * c["H"] > 8192:
                continue
        return c


def _spread(case, most, step):
    """Sizes of the sequences: the first has `most`, the others of a ragged batch are spread over (0, most]."""
    if not case["ragged"]:
        return [most] * case["seqs"]
    return [max(1, math.ceil(most * ((1 - i * step) % 1.0 or 1.0))) for i in range(case["seqs"])]


def _sizes(case):
    """(tokens in the cache, new tokens among them) of each sequence."""
    lens = _spread(case, case["longest"], 0.6180339887)
    new = [min(n, q) for n, q in zip(lens, _spread(case, case["queries"], 0.7548776662))]
    return lens, new


def _visible(n, new, window):
    """Tokens that any of the last `new` of n tokens sees, and (query, token) pairs."""
    if window == 0 or window > n:
        window = n
    pairs = sum(min(p + 1, window) for p in range(n - new, n))
    return min(n, new - 1 + window), pairs


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    H, D, BS, B, op = case["H"], case["D"], case["BS"], case["seqs"], case["op"]
    dtype = getattr(torch, case["dtype"])
    lens, new = _sizes(case)
    s = dict(case=case, B=B, max_len=max(lens), max_q=max(new), tokens=sum(new),
             lens=torch.tensor(lens, dtype=torch.int32, device=DEVICE))
    # One new token each needs no list of where a sequence's queries start.
    starts = torch.tensor([0] + new, dtype=torch.int32, device=DEVICE).cumsum(0, dtype=torch.int32)
    s["starts"] = None if s["max_q"] == 1 else starts
    pages = [-(-n // BS) for n in lens]
    num_blocks = sum(pages) + 3
    order = torch.randperm(num_blocks, device=DEVICE, generator=gen, dtype=torch.int32)
    s["tables"] = _table(order, pages)
    scaled = case["fp8"] and op != "rotate"
    # Scores go by bounds alone; the others have a cache.
    shape = (num_blocks, 2, H, 1, D) if op == "score" else \
        (num_blocks, 2, BS, H, D) if case["nhd"] else (num_blocks, 2, H, BS, D)
    layer = torch.randn(shape, device=DEVICE, generator=gen)
    if op == "score":
        layer = layer.mul_(0.4).sub_(1.5 - 3.0 * torch.arange(2, device=DEVICE).view(1, 2, 1, 1, 1))  # low, high
    if case["fp8"]:
        layer = layer.mul_(40).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn)
    else:
        layer = layer.to(dtype)
    s["layer"] = layer
    s["scales"] = None
    if scaled:
        # Exponents of the pages' scales: 2^-8 to 2^-5.
        s["scales"] = torch.randint(119, 123, (num_blocks, 2, H), device=DEVICE, generator=gen, dtype=torch.uint8)
    if op == "bounds":
        s["bounds"] = torch.zeros(num_blocks, 2, H, 1, D, dtype=layer.dtype, device=DEVICE)
        # Which pages the new tokens lie in.
        s["touched"] = sum((n - 1) // BS - (n - q) // BS + 1 for n, q in zip(lens, new))
    else:
        # Queries, keys and values of the new tokens as one projection's output gives them: views of its rows.
        heads = H * case["G"]
        qkv = torch.randn(s["tokens"], heads + 2 * H, D, device=DEVICE, generator=gen).mul_(2).to(dtype)
        s["q"], s["k"], s["v"] = qkv.split([heads, H, H], dim=1)
    if op == "rotate":
        half = case["rotary"] // 2
        s["freqs"] = torch.pow(10000.0, -torch.arange(half, dtype=torch.float64, device=DEVICE) / half)
        s["weights"] = (None, None)
        if case["norm"]:
            s["weights"] = (1 + 0.1 * torch.randn(2, D, device=DEVICE, generator=gen)).unbind(0)
        # Positions that are not the tokens' places, where a compaction has moved these.
        s["positions"] = None
        if case["moved"]:
            seq, place, new_of = _new_tokens(s)
            s["positions"] = (s["lens"][seq] - new_of[seq] + place + case["moved"]).int()
    if op == "attend":
        s["slopes"] = None
        if case["slopes"]:
            s["slopes"] = torch.exp2(-8 * torch.arange(1, heads + 1, device=DEVICE, dtype=torch.float32) / heads)
    if op == "score":
        s["most_pages"] = max(pages)
        s["scores"] = torch.zeros(s["tokens"], H, max(pages), device=DEVICE)
    if op == "pages":
        # Each new token's choice for each head: ascending, its first page and its own among them.
        budget, most = case["budget"], max(pages)
        seq, place, new_of = _new_tokens(s)
        count = (s["lens"][seq] - new_of[seq] + place) // BS + 1
        page = torch.arange(most, device=DEVICE)
        rank = torch.rand(s["tokens"], H, most, device=DEVICE, generator=gen)
        rank.masked_fill_((page == 0) | (page == (count - 1).view(-1, 1, 1)), -1.0)
        rank.masked_fill_(page >= count.view(-1, 1, 1), 2.0)
        chosen = rank.argsort(-1)[..., :budget]
        s["counts"] = count.clamp(max=budget).int()
        gone = torch.arange(chosen.shape[-1], device=DEVICE) >= s["counts"].view(-1, 1, 1)
        chosen = chosen.masked_fill(gone, most).sort(-1).values.masked_fill(gone, -1)
        s["pages"] = torch.full((s["tokens"], H, budget), -1, dtype=torch.int32, device=DEVICE)
        s["pages"][..., :chosen.shape[-1]] = chosen
    if own:
        # The handles of the cache and of the bounds, which a replica makes once.
        from paper_2609_15021_amd import kvx
        size = layer.element_size()
        order_of = kvx.KV_BLOCK_NHD if case["nhd"] else kvx.KV_BLOCK_HND
        ones = kvx.make_layout(1, H, D, size, 1, 1)
        if op == "score":
            s["bounds_cache"] = kvx.Cache([layer], ones, num_blocks)
        else:
            s["cache"] = kvx.Cache([layer], kvx.make_layout(1, H, D, size, BS, BS), num_blocks, block_order=order_of)
        if op == "bounds":
            s["bounds_cache"] = kvx.Cache([s["bounds"]], ones, num_blocks)
    return s


def _table(order, pages):
    """Block tables [sequences][most pages], each sequence's pages taken from `order` in turn; unused entries are 0."""
    table = torch.zeros(len(pages), max(1, max(pages)), dtype=torch.int32, device=DEVICE)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    return table


def run(state):
    op = state["case"]["op"]
    if own:
        return _OWN[op](state)
    return _PLAIN[op](state)


# ---- The framework's calls ----------------------------------------------------------------


def _own_rotate(s):
    from paper_2609_15021_amd import attend
    c = s["case"]
    q = attend.kv_rotate(s["cache"], 0, s["q"], s["k"], s["v"], s["tables"], s["lens"], s["starts"], freqs=s["freqs"],
                         positions=s["positions"], q_weight=s["weights"][0], k_weight=s["weights"][1], eps=_EPS,
                         interleaved=c["interleaved"], max_q=s["max_q"], max_len=s["max_len"],
                         k_scale=_K_SCALE if c["fp8"] else 1.0, v_scale=_V_SCALE if c["fp8"] else 1.0)
    return q, s["layer"]


def _own_append(s):
    from paper_2609_15021_amd import attend
    attend.kv_append(s["cache"], 0, s["k"], s["v"], s["tables"], s["lens"], s["starts"], max_q=s["max_q"],
                     max_len=s["max_len"], scales=s["scales"])
    return s["layer"], s["scales"]


def _own_attend(s):
    from paper_2609_15021_amd import attend
    c = s["case"]
    return attend.kv_attend(s["cache"], 0, s["q"], s["tables"], s["lens"], s["starts"], max_q=s["max_q"],
                            max_len=s["max_len"], softcap=c["softcap"], window=c["window"], slopes=s["slopes"],
                            scales=s["scales"])


def _own_bounds(s):
    from paper_2609_15021_amd import attend
    attend.kv_bounds(s["cache"], 0, s["bounds_cache"], s["tables"], s["lens"], s["starts"], max_q=s["max_q"],
                     max_len=s["max_len"], dtype=s["layer"].dtype)
    return s["bounds"]


def _own_score(s):
    from paper_2609_15021_amd import attend
    return attend.kv_score(s["bounds_cache"], 0, s["q"], s["tables"], s["lens"], s["starts"],
                           block_size=s["case"]["BS"], max_q=s["max_q"], max_len=s["max_len"], scales=s["scales"],
                           out=s["scores"])


def _own_pages(s):
    from paper_2609_15021_amd import attend
    return attend.kv_attend(s["cache"], 0, s["q"], s["tables"], s["lens"], s["starts"], max_q=s["max_q"],
                            max_len=s["max_len"], scales=s["scales"], pages=s["pages"], counts=s["counts"])


_OWN = dict(rotate=_own_rotate, append=_own_append, attend=_own_attend, bounds=_own_bounds, score=_own_score,
            pages=_own_pages)

# ---- The plain form -----------------------------------------------------------------------


def _bytes(x):
    """Indexing of e4m3 goes by its bytes."""
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _power(exponents):
    """2^(e - 127)."""
    return torch.ldexp(torch.ones((), device=DEVICE), exponents.int() - 127)


def _rows(s, kv, at):
    """K (kv 0) or V rows of the tokens `at` [B][n] of each sequence, in 32 bits: [B][n][H][D]."""
    c, layer = s["case"], s["layer"]
    block = s["tables"].gather(1, at // c["BS"]).long()
    slot = at % c["BS"]
    rows = _bytes(layer)[block, kv, slot] if c["nhd"] else _bytes(layer)[block, kv, :, slot]
    rows = rows.view(layer.dtype).float()
    return rows * _power(s["scales"][block, kv])[..., None] if s["scales"] is not None else rows


def _new_tokens(s):
    """Of each new token its sequence and its place among the sequence's new ones; new tokens of each sequence."""
    every = torch.arange(s["B"], device=DEVICE)
    if s["starts"] is None:
        return every, torch.zeros_like(every), torch.ones_like(every)
    new = s["starts"].diff().long()
    seq = torch.repeat_interleave(every, new, output_size=s["tokens"])
    return seq, torch.arange(s["tokens"], device=DEVICE) - s["starts"][seq], new


def _put(s, kv, block, slot, rows):
    """Rows [tokens][H][D] of the cache's type into their slots."""
    if s["case"]["nhd"]:
        _bytes(s["layer"])[block, kv, slot] = _bytes(rows)
    else:
        _bytes(s["layer"])[block, kv, :, slot] = _bytes(rows)


def _plain_rotate(s):
    c = s["case"]
    seq, place, new = _new_tokens(s)
    at = s["lens"][seq] - new[seq] + place
    angle = (at if s["positions"] is None else s["positions"]).double()[:, None] * s["freqs"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(x, weight):
        x = x.float()
        if c["norm"]:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS) * weight
        x, rest = x[..., :c["rotary"]], x[..., c["rotary"]:]
        if c["interleaved"]:
            a, b = x[..., ::2], x[..., 1::2]
            x = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = x.chunk(2, -1)
            x = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([x, rest], -1)

    q, k = turned(s["q"], s["weights"][0]).to(s["q"].dtype), turned(s["k"], s["weights"][1])
    v = s["v"].float()
    if c["fp8"]:
        k, v = (k / _K_SCALE).clamp(-448.0, 448.0), (v / _V_SCALE).clamp(-448.0, 448.0)
    block, slot = s["tables"][seq, at // c["BS"]].long(), at % c["BS"]
    _put(s, 0, block, slot, k.to(s["layer"].dtype))
    _put(s, 1, block, slot, v.to(s["layer"].dtype))
    return q, s["layer"]


def _plain_append(s):
    c, layer, scales = s["case"], s["layer"], s["scales"]
    seq, place, new = _new_tokens(s)
    at = s["lens"][seq] - new[seq] + place
    block, slot = s["tables"][seq, at // c["BS"]].long(), at % c["BS"]
    rows = torch.stack([s["k"], s["v"]], 1).float()  # [tokens][2][H][D]
    # The largest of each page's new rows, and the smallest power of two that brings it to 448 or less.
    most = torch.zeros(scales.shape, device=DEVICE)
    most.scatter_reduce_(0, block.view(-1, 1, 1).expand(-1, 2, c["H"]), rows.abs().amax(-1), "amax")
    mantissa, exponent = torch.frexp(most)
    need = (exponent + 118 + (mantissa > 0.875)).masked_fill(most == 0, 1).clamp(1, 254)
    # A page that begins with a new row has no scale yet; another keeps its own unless it has to grow, and its older
    # rows, which lie in the first page of a sequence's new ones, are rounded to the new one.
    first_at = s["lens"] - new
    first = s["tables"].gather(1, (first_at // c["BS"])[:, None]).view(-1).long()
    older = first_at % c["BS"]
    before = scales[first].int()
    after = torch.where((older > 0).view(-1, 1, 1), torch.maximum(before, need[first]), need[first])
    scales[block] = need[block].to(torch.uint8)
    scales[first] = after.to(torch.uint8)
    held = _bytes(layer)[first].view(layer.dtype)
    factor = torch.ldexp(torch.ones((), device=DEVICE), before - after)
    factor = factor[:, :, None, :, None] if c["nhd"] else factor[:, :, :, None, None]
    old = torch.arange(c["BS"], device=DEVICE) < older.view(-1, 1)
    old = old.view(-1, 1, c["BS"], 1, 1) if c["nhd"] else old.view(-1, 1, 1, c["BS"], 1)
    _bytes(layer)[first] = torch.where(old, _bytes((held.float() * factor).to(layer.dtype)), _bytes(held))
    rows = (rows / _power(scales[block])[..., None]).clamp(-448.0, 448.0).to(layer.dtype)
    _put(s, 0, block, slot, rows[:, 0])
    _put(s, 1, block, slot, rows[:, 1])
    return layer, scales


def _plain_attend(s):
    c = s["case"]
    B, H, G, D, Q, L = s["B"], c["H"], c["G"], c["D"], s["max_q"], s["max_len"]
    seq, place, new = _new_tokens(s)
    # Sequences padded to the most queries and tokens.
    q = torch.zeros(B, Q, H, G, D, device=DEVICE)
    q[seq, place] = s["q"].float().view(-1, H, G, D)
    q = q.permute(0, 2, 1, 3, 4).reshape(B, H, Q * G, D)
    token = torch.arange(L, device=DEVICE)
    every = token.expand(B, L)
    x = torch.matmul(q, _rows(s, 0, every).permute(0, 2, 3, 1)) / math.sqrt(D)
    x = x.view(B, H, Q, G, L)
    if c["softcap"]:
        x = torch.tanh(x / c["softcap"]) * c["softcap"]
    position = s["lens"].view(B, 1) - new.view(B, 1) + torch.arange(Q, device=DEVICE)
    distance = position.view(B, 1, Q, 1, 1) - token
    if c["slopes"]:
        x = x - s["slopes"].view(1, H, 1, G, 1) * distance
    hidden = distance < 0
    if c["window"]:
        hidden = hidden | (distance >= c["window"])
    x = x.masked_fill(hidden, -math.inf)
    most = x.amax(-1, keepdim=True)
    e = torch.exp(x - most)
    total = e.sum(-1, keepdim=True)
    lse = (most + total.log()).squeeze(-1)
    e = e / total
    out = torch.matmul(e.view(B, H, Q * G, L), _rows(s, 1, every).permute(0, 2, 1, 3))
    out = out.view(B, H, Q, G, D).permute(0, 2, 1, 3, 4)[seq, place].reshape(-1, H * G, D).to(s["q"].dtype)
    return out, lse.permute(0, 2, 1, 3)[seq, place].reshape(-1, H * G)


def _plain_bounds(s):
    c, layer = s["case"], s["layer"]
    _, _, new = _new_tokens(s)
    # The pages that new tokens lie in, one after the other.
    first = (s["lens"] - new) // c["BS"]
    many = (s["lens"] - 1) // c["BS"] - first + 1
    seq = torch.repeat_interleave(torch.arange(s["B"], device=DEVICE), many, output_size=s["touched"])
    page = first[seq] + torch.arange(s["touched"], device=DEVICE) - (many.cumsum(0) - many)[seq]
    block = s["tables"][seq, page].long()
    k = _bytes(layer)[block, 0].view(layer.dtype).float()
    k = k.transpose(1, 2) if c["nhd"] else k  # [pages][H][BS][D]
    token = page.view(-1, 1) * c["BS"] + torch.arange(c["BS"], device=DEVICE)
    none = (token >= s["lens"][seq].view(-1, 1)).view(-1, 1, c["BS"], 1)
    low, high = k.masked_fill(none, math.inf).amin(2), k.masked_fill(none, -math.inf).amax(2)
    _bytes(s["bounds"])[block, :, :, 0] = _bytes(torch.stack([low, high], 1).to(layer.dtype))
    return s["bounds"]


def _plain_score(s):
    c, bounds = s["case"], s["layer"]
    B, H, G, D, Q, P = s["B"], c["H"], c["G"], c["D"], s["max_q"], s["most_pages"]
    seq, place, new = _new_tokens(s)
    q = torch.zeros(B, Q, H, G, D, device=DEVICE)
    q[seq, place] = s["q"].float().view(-1, H, G, D)
    q = q.permute(0, 2, 1, 3, 4).reshape(B, H, Q * G, D)
    rows = _bytes(bounds)[s["tables"].long(), :, :, 0].view(bounds.dtype).float()  # [B][P][2][H][D]
    rows = rows.permute(2, 0, 3, 4, 1)  # [2][B][H][D][P]
    # The larger of q low and q high is q high where q is positive, and q low elsewhere.
    x = torch.matmul(q.clamp(min=0.0), rows[1]) + torch.matmul(q.clamp(max=0.0), rows[0])
    x = x.view(B, H, Q, G, P).amax(3)
    if s["scales"] is not None:
        x = x * _power(s["scales"][s["tables"].long(), 0]).transpose(1, 2).unsqueeze(2)
    count = (s["lens"][seq] - new[seq] + place) // c["BS"] + 1
    seen = torch.arange(P, device=DEVICE) < count.view(-1, 1, 1)
    return torch.where(seen, x.permute(0, 2, 1, 3)[seq, place], s["scores"]), count.int()


def _plain_pages(s):
    c, layer = s["case"], s["layer"]
    H, G, D, BS, T, N = c["H"], c["G"], c["D"], c["BS"], s["tokens"], c["budget"] * c["BS"]
    seq, place, new = _new_tokens(s)
    position = s["lens"][seq] - new[seq] + place
    page = s["pages"].long().clamp(min=0)
    block = s["tables"][seq[:, None, None], page].long()  # [tokens][H][budget]
    head = torch.arange(H, device=DEVICE).view(1, H, 1)

    def rows(kv):
        x = _bytes(layer)[block, kv, :, head] if c["nhd"] else _bytes(layer)[block, kv, head]
        x = x.view(layer.dtype).float()
        if s["scales"] is not None:
            x = x * _power(s["scales"][block, kv, head])[..., None, None]
        return x.reshape(T, H, N, D)

    x = torch.matmul(s["q"].float().view(T, H, G, D), rows(0).transpose(2, 3)) / math.sqrt(D)
    token = (page[..., None] * BS + torch.arange(BS, device=DEVICE)).view(T, H, 1, N)
    hidden = (s["pages"] < 0)[..., None].expand(T, H, c["budget"], BS).reshape(T, H, 1, N)
    x = x.masked_fill(hidden | (token > position.view(T, 1, 1, 1)), -math.inf)
    most = x.amax(-1, keepdim=True)
    e = torch.exp(x - most)
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e / total, rows(1)).reshape(T, H * G, D).to(s["q"].dtype)
    return out, (most + total.log()).reshape(T, H * G)


_PLAIN = dict(rotate=_plain_rotate, append=_plain_append, attend=_plain_attend, bounds=_plain_bounds,
              score=_plain_score, pages=_plain_pages)

# ---- The definition, in 64 bits, one sequence and head at a time ----------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return _EXACT[case["op"]](s)


def _each(s):
    """(sequence, tokens, new tokens, first row) of each sequence."""
    at = 0
    for b, (n, q) in enumerate(zip(*_sizes(s["case"]))):
        yield b, n, q, at
        at += q


def _factors(s):
    """The scales of every (block, K or V, head) in 64 bits."""
    if s["scales"] is None:
        return None
    return torch.pow(2.0, s["scales"].double() - 127.0)


def _head(s, factors, b, n, kv, h):
    """The first n rows of head h of one sequence's K or V, page after page, in 64 bits."""
    c = s["case"]
    pages = s["tables"][b, :-(-n // c["BS"])].long()
    block = s["layer"][:, kv, :, h] if c["nhd"] else s["layer"][:, kv, h]
    rows = block.double()[pages]
    if factors is not None:
        rows = rows * factors[pages, kv, h].view(-1, 1, 1)
    return rows.flatten(0, 1)[:n]


def _exact_rotate(s):
    c = s["case"]
    out, layer = s["q"].double(), s["layer"].double()
    rot, half = c["rotary"], c["rotary"] // 2
    i = torch.arange(half, device=DEVICE)
    left, right = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)

    def turned(x, weight, position):
        x = x.double()
        if c["norm"]:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["D"] + _EPS) * weight.double()
        angle = position.double()[:, None] * s["freqs"]
        z = torch.complex(x[:, left], x[:, right]) * torch.polar(torch.ones_like(angle), angle)
        y = x.clone()
        y[:, left], y[:, right] = z.real, z.imag
        return y

    for b, n, q, at in _each(s):
        t = torch.arange(n - q, n, device=DEVICE)
        position = t + c["moved"]
        page, slot = s["tables"][b, t // c["BS"]].long(), t % c["BS"]
        for g in range(c["H"] * c["G"]):
            out[at:at + q, g] = turned(s["q"][at:at + q, g], s["weights"][0], position)
        for h in range(c["H"]):
            k, v = turned(s["k"][at:at + q, h], s["weights"][1], position), s["v"][at:at + q, h].double()
            if c["fp8"]:
                k, v = (k / _K_SCALE).clamp(-448, 448), (v / _V_SCALE).clamp(-448, 448)
            for kv, x in ((0, k), (1, v)):
                if c["nhd"]:
                    layer[page, kv, slot, h] = x
                else:
                    layer[page, kv, h, slot] = x
    return out, layer


def _exact_append(s):
    c = s["case"]
    layer, scales = s["layer"].double(), s["scales"].clone()
    BS = c["BS"]
    for kv, rows in ((0, s["k"]), (1, s["v"])):
        for b, n, q, at in _each(s):
            # New rows by page, those before the first and behind the last new one being zeros.
            first, last = (n - q) // BS, (n - 1) // BS
            x = torch.zeros((last - first + 1) * BS, c["H"], c["D"], dtype=torch.float64, device=DEVICE)
            old = n - q - first * BS
            x[old:old + q] = rows[at:at + q].double()
            x = x.view(-1, BS, c["H"], c["D"])
            most = x.abs().amax((1, 3))
            e = torch.ceil(torch.log2(most / 448)).clamp(min=-126) + 127
            # (A logarithm next to a whole number may lie on the wrong side.)
            e = torch.where(most <= 448 * torch.pow(2.0, e - 128), e - 1, e)
            e = torch.where(most > 448 * torch.pow(2.0, e - 127), e + 1, e).clamp(1, 254)
            page = s["tables"][b, first:last + 1].long()
            if old:
                before = scales[page[0], kv].double()
                e[0] = torch.maximum(e[0], before)
                change = torch.pow(2.0, before - e[0])
                if c["nhd"]:
                    layer[page[0], kv, :old] *= change.view(1, -1, 1)
                else:
                    layer[page[0], kv, :, :old] *= change.view(-1, 1, 1)
            scales[page, kv] = e.to(torch.uint8)
            stored = (x * torch.pow(2.0, 127.0 - e).view(-1, 1, c["H"], 1)).flatten(0, 1)[old:old + q]
            t = torch.arange(n - q, n, device=DEVICE)
            block, slot = s["tables"][b, t // BS].long(), t % BS
            if c["nhd"]:
                layer[block, kv, slot] = stored
            else:
                layer[block, kv, :, slot] = stored
    return layer, scales


def _exact_attend(s):
    c, factors = s["case"], _factors(s)
    H, G, D = c["H"], c["G"], c["D"]
    out = torch.zeros(s["tokens"], H * G, D, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(s["tokens"], H * G, dtype=torch.float64, device=DEVICE)
    for b, n, q, at in _each(s):
        far = torch.arange(n - q, n, device=DEVICE)[:, None] - torch.arange(n, device=DEVICE)
        seen = (far >= 0) & (far < (c["window"] or n))
        for h in range(H):
            k, v = _head(s, factors, b, n, 0, h), _head(s, factors, b, n, 1, h)
            for g in range(h * G, h * G + G):
                z = (s["q"][at:at + q, g].double() @ k.T) / math.sqrt(D)
                if c["softcap"]:
                    z = c["softcap"] * torch.tanh(z / c["softcap"])
                if c["slopes"]:
                    z = z - s["slopes"][g].double() * far
                z = torch.where(seen, z, -math.inf)
                lse[at:at + q, g] = torch.logsumexp(z, 1)
                out[at:at + q, g] = torch.exp(z - lse[at:at + q, g, None]) @ v
    return out, lse


def _exact_bounds(s):
    c = s["case"]
    bounds = s["bounds"].double()
    for b, n, q, _ in _each(s):
        first = (n - q) // c["BS"]
        page = s["tables"][b, first:(n - 1) // c["BS"] + 1].long()
        more = page.numel() * c["BS"] - (n - first * c["BS"])
        for h in range(c["H"]):
            k = _head(s, None, b, n, 0, h)[first * c["BS"]:]
            # The last page's missing rows repeat its last one.
            k = torch.cat([k, k[-1:].expand(more, -1)]).view(-1, c["BS"], c["D"])
            bounds[page, 0, h, 0] = k.min(1).values
            bounds[page, 1, h, 0] = k.max(1).values
    return bounds


def _exact_score(s):
    c, factors = s["case"], _factors(s)
    H, G = c["H"], c["G"]
    scores = s["scores"].double()
    count = torch.zeros(s["tokens"], dtype=torch.int32, device=DEVICE)
    for b, n, q, at in _each(s):
        pages = s["tables"][b, :-(-n // c["BS"])].long()
        own_page = torch.arange(n - q, n, device=DEVICE) // c["BS"]
        count[at:at + q] = own_page.int() + 1
        seen = torch.arange(pages.numel(), device=DEVICE) <= own_page[:, None]
        for h in range(H):
            low, high = (s["layer"][pages, j, h, 0].double() for j in (0, 1))
            if factors is not None:
                low, high = (x * factors[pages, 0, h, None] for x in (low, high))
            best = torch.full((q, pages.numel()), -math.inf, dtype=torch.float64, device=DEVICE)
            for g in range(h * G, h * G + G):
                # max(q low, q high) = q (low + high) / 2 + |q| (high - low) / 2
                x = s["q"][at:at + q, g].double()
                best = torch.maximum(best, 0.5 * (x @ (low + high).T + x.abs() @ (high - low).T))
            scores[at:at + q, h, :pages.numel()] = torch.where(seen, best, scores[at:at + q, h, :pages.numel()])
    return scores, count


def _exact_pages(s):
    c, factors = s["case"], _factors(s)
    H, G, D, BS = c["H"], c["G"], c["D"], c["BS"]
    out = torch.zeros(s["tokens"], H * G, D, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(s["tokens"], H * G, dtype=torch.float64, device=DEVICE)
    for b, n, q, at in _each(s):
        for h in range(H):
            k, v = _head(s, factors, b, n, 0, h), _head(s, factors, b, n, 1, h)
            for i in range(q):
                seen = torch.zeros(-(-n // BS) + 1, dtype=torch.bool, device=DEVICE)
                seen[s["pages"][at + i, h].long()] = True  # (-1: the one behind the last)
                seen = seen[:-1].repeat_interleave(BS)[:n] & (torch.arange(n, device=DEVICE) <= n - q + i)
                z = (s["q"][at + i, h * G:h * G + G].double() @ k.T) / math.sqrt(D)
                z = torch.where(seen, z, -math.inf)
                lse[at + i, h * G:h * G + G] = torch.logsumexp(z, 1)
                out[at + i, h * G:h * G + G] = torch.softmax(z, 1) @ v
    return out, lse


_EXACT = dict(rotate=_exact_rotate, append=_exact_append, attend=_exact_attend, bounds=_exact_bounds,
              score=_exact_score, pages=_exact_pages)

# ---- What a pass cannot do without ----------------------------------------------------------


def work(case):
    lens, new = _sizes(case)
    H, D, BS, op = case["H"], case["D"], case["BS"], case["op"]
    size = 1 if case["fp8"] else 2
    tokens, heads = sum(new), H * case["G"]
    if op == "rotate":
        moved = tokens * D * (4 * heads + 2 * H * (2 + size))
        return {"bytes": moved, "flops": tokens * (heads + H) * D * (9 if case["norm"] else 3)}
    if op == "append":
        pages = sum((n - 1) // BS - (n - q) // BS + 1 for n, q in zip(lens, new))
        return {"bytes": 2 * tokens * H * D * 3 + 2 * H * (pages + case["seqs"]), "flops": 4 * tokens * H * D}
    if op == "bounds":
        first = [(n - q) // BS for n, q in zip(lens, new)]
        pages = sum((n - 1) // BS - f + 1 for n, f in zip(lens, first))
        rows = sum(n - f * BS for n, f in zip(lens, first))
        return {"bytes": (rows + 2 * pages) * H * D * size, "flops": 2 * rows * H * D}
    if op == "score":
        pages = sum(-(-n // BS) for n in lens)
        pairs = sum(p // BS + 1 for n, q in zip(lens, new) for p in range(n - q, n))
        return {"bytes": 2 * pages * H * D * size + tokens * heads * D * 2 + 4 * pairs * H,
                "flops": 4 * D * heads * pairs}
    scales = 2 * H * sum(-(-n // BS) for n in lens) if case["fp8"] else 0
    if op == "pages":
        # What the rows of a sequence choose apart from each other's is at most its pages.
        pairs = [min(p // BS + 1, case["budget"]) for n, q in zip(lens, new) for p in range(n - q, n)]
        at, rows = 0, 0
        for n, q in zip(lens, new):
            rows += min(n, BS * sum(pairs[at:at + q]))
            at += q
        return {"bytes": 2 * rows * H * D * size + tokens * heads * (4 * D + 4) + 4 * H * sum(pairs) + scales,
                "flops": 4 * D * heads * BS * sum(pairs)}
    seen = [_visible(n, q, case["window"]) for n, q in zip(lens, new)]
    pages = sum(-(-n // BS) for n in lens)
    return {"bytes": 2 * sum(n for n, _ in seen) * H * D * size + tokens * heads * (4 * D + 4) + 4 * pages + scales,
            "flops": 4 * D * heads * sum(pairs for _, pairs in seen)}
