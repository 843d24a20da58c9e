"""Operators of batched serving, as measurable cases: attention over packed prompts, and the keys and values of many
sequences in pages, written (bf16 as they are, or e4m3 with a power of two per token and head), read back, and attended to by one
new token of every sequence.

prompt  causal attention inside each of `n_seqs` prompts that lie one behind the other, `pad` rows behind the last of them
decode  one new token per sequence over its pages
store   rows of K and V into the pages of their sequences, `first` tokens behind each sequence's beginning
load    rows of K and V out of the pages, as bf16

The lengths of a case's sequences are spread over (1, `longest`] by their logarithm and depend on the case alone (`mix`).
"""
import math
import random

import torch

own = False

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
HEADS = [(4, 4), (32, 32), (28, 4), (32, 8), (16, 4), (8, 2), (6, 2), (5, 5), (16, 1)]


def _prompt(name, hq, hkv, d, n_seqs, longest, mix=0, pad=0):
    case = dict(kind="prompt", hq=hq, hkv=hkv, d=d, n_seqs=n_seqs, longest=longest, mix=mix, pad=pad)
    return dict(case, name=name) if name else case


def _decode(name, hq, hkv, d, n_seqs, longest, page, e4m3, mix=0):
    case = dict(kind="decode", hq=hq, hkv=hkv, d=d, n_seqs=n_seqs, longest=longest, page=page, e4m3=e4m3, mix=mix)
    return dict(case, name=name) if name else case


def _rows(name, kind, hkv, d, n_seqs, longest, page, e4m3, first=0, by_head=False, mix=0):
    case = dict(kind=kind, hkv=hkv, d=d, n_seqs=n_seqs, longest=longest, page=page, e4m3=e4m3, first=first, by_head=by_head, mix=mix)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the smallest prompt: an image of 24 x 24 patches and 32 tokens of text through one small layer
        _prompt("prompt tiny", 4, 4, 64, 1, 608),
        # a batch of short requests, none of them worth compressing, of very different lengths
        _prompt("prompt batch", 28, 4, 128, 24, 2100, mix=1, pad=37),
        # small heads, odd lengths, an empty prompt among them
        _prompt("prompt ragged d64", 16, 4, 64, 9, 3333, mix=6),
        # a long video's prefix without compression, 64 frames of 256 tokens and the text
        _prompt("prompt long", 32, 8, 128, 1, 16640),
        # one request, a few hundred keys: all launch and latency
        _decode("decode one short", 28, 4, 128, 1, 313, 64, False),
        # compressed caches of a batch, 8 bits a number
        _decode("decode batch e4m3", 32, 8, 128, 32, 2176, 64, True, mix=2),
        # one very long sequence, small pages
        _decode("decode one long e4m3", 28, 4, 128, 1, 131071, 16, True),
        # a full server: many sequences up to 16640 tokens
        _decode("decode full server", 32, 8, 128, 96, 16640, 64, False, mix=3),
        # the current tokens of a batch, one row each at odd places
        _rows("store step e4m3", "store", 8, 128, 48, 1, 64, True, first=1021),
        # a prefix as it leaves the projections, to 8 bits
        _rows("store prefix e4m3", "store", 8, 128, 3, 16640, 64, True, mix=4),
        # a compressed cache taken back into [heads, slots, channels] to go on with
        _rows("load cache e4m3", "load", 4, 128, 1, 1024, 64, True, by_head=True),
        # prefixes of a batch, from small bf16 pages, small heads
        _rows("load batch d64", "load", 32, 64, 12, 9001, 16, False, mix=5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = [work(c) for c in listed()]
    while True:
        kind = rng.choice(["prompt", "prompt", "decode", "decode", "store", "load"])
        hq, hkv = rng.choice(HEADS)
        d = rng.choice([64, 128, 128])
        n_seqs, longest, mix = _log_int(rng, 1, 96), _log_int(rng, 1, 16640), rng.randrange(1 << 20)
        if kind == "prompt":
            case = _prompt(None, hq, hkv, d, n_seqs, longest, mix, rng.choice([0, 0, rng.randint(1, 200)]))
            if n_seqs * hq * longest ** 2 > 32 * 16640 ** 2:
                continue
        else:
            page, e4m3 = rng.choice([16, 32, 64, 64, 128, 256]), rng.random() < 0.5
            if kind == "decode":
                if n_seqs < 4:
                    longest = _log_int(rng, 1, 131071)
                case = _decode(None, hq, hkv, d, n_seqs, longest, page, e4m3, mix)
            else:
                case = _rows(None, kind, hkv, d, n_seqs, longest, page, e4m3, rng.choice([0, rng.randint(0, 3000)]), rng.random() < 0.3, mix)
        w = work(case)
        alike = [m for m, c in zip(most, listed()) if c["kind"] == kind]
        if 0 < w["flops"] + w["bytes"] and w["flops"] <= max(m["flops"] for m in alike) and w["bytes"] <= max(m["bytes"] for m in alike):
            return case


def _lengths(case):
    """One length per sequence, the longest among them; of every eighth sequence beyond the fourth none is left."""
    rng = random.Random(case["mix"])
    n, longest = case["n_seqs"], case["longest"]
    found = [longest] + [0 if i % 8 == 5 and longest > 1 else _log_int(rng, max(1, longest / 50), longest) for i in range(1, n)]
    rng.shuffle(found)
    return found


def _begins(lengths):
    found = [0]
    for n in lengths:
        found.append(found[-1] + n)
    return found


def _numbers(gen, *shape):
    """Keys, values or queries: normal, with channels of larger spread and an offset of their own, as projections leave them."""
    dev, d = gen.device, shape[-1]
    x = torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)
    x *= torch.exp(0.5 * torch.randn((d,), generator=gen, device=dev))
    x += 0.5 * torch.randn(shape[-2:], generator=gen, device=dev)
    return x.to(BF16)


def _pages_for(case, gen, lengths, state):
    """A table of pages in random order, with a few more pages than it names."""
    dev, page = gen.device, case["page"]
    counts = [-(-n // page) for n in lengths]
    width, n_pages = max(1, max(counts)), sum(counts) + 3
    order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
    begin = torch.tensor(_begins(counts), device=dev)
    column = torch.arange(width, device=dev)
    place = (begin[:-1, None] + column).clamp(max=n_pages - 1)
    table = torch.where(column < torch.tensor(counts, device=dev)[:, None], order[place], torch.full_like(order[place], -1))
    shape = (n_pages, case["hkv"], page, case["d"])
    state.update(table=table.contiguous(), k=torch.zeros(shape, device=dev, dtype=BF16), v=torch.zeros(shape, device=dev, dtype=BF16), k_exp=None, v_exp=None)
    if case["e4m3"]:
        state.update(k=state["k"].to(E4M3), v=state["v"].to(E4M3), k_exp=torch.full(shape[:3], 127, device=dev, dtype=torch.uint8),
                     v_exp=torch.full(shape[:3], 127, device=dev, dtype=torch.uint8))


def _fill(case, gen, state):
    """Numbers in all pages, behind the sequences' ends as well."""
    for name in ("k", "v"):
        x = _numbers(gen, state[name].shape[0], case["page"], case["hkv"], case["d"]).transpose(1, 2)
        if case["e4m3"]:
            x, state[name + "_exp"] = _to_e4m3(x)
        state[name] = x.contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dev, lengths, d = gen.device, _lengths(case), case["d"]
    n = sum(lengths)
    state = dict(case=case, seq_begin=torch.tensor(_begins(lengths), device=dev, dtype=torch.int32), longest=max(lengths))
    if case["kind"] == "prompt":
        n += case["pad"]
        kv = _numbers(gen, n, 2, case["hkv"], d)            # K and V of a row as one projection leaves them
        state.update(q=_numbers(gen, n, case["hq"], d), k=kv[:, 0], v=kv[:, 1], out=torch.zeros((n, case["hq"], d), device=dev, dtype=BF16))
        return state
    _pages_for(case, gen, [n + case.get("first", 0) for n in lengths], state)
    if case["kind"] == "decode":
        _fill(case, gen, state)
        state.update(lengths=torch.tensor(lengths, device=dev, dtype=torch.int32), q=_numbers(gen, len(lengths), case["hq"], d),
                     out=torch.empty((len(lengths), case["hq"], d), device=dev, dtype=BF16))
    else:
        state["first"] = torch.full((len(lengths),), case["first"], device=dev, dtype=torch.int32)
        if case["kind"] == "load":
            _fill(case, gen, state)
        if case["by_head"]:
            rows = [_numbers(gen, case["hkv"], n, d).transpose(0, 1) for _ in range(2)]
        else:
            rows = list(_numbers(gen, n, 2, case["hkv"], d).unbind(1))
        state["k_rows"], state["v_rows"] = rows
    if own:
        import paper_2604_16734_amd as kvp
        state["pages"] = kvp.Pages(state["k"], state["v"], state["k_exp"], state["v_exp"])
    return state


def run(state):
    case = state["case"]
    kind = case["kind"]
    if own:
        if kind == "prompt":
            import paper_2604_16734_amd as kvp
            return kvp.prompt_attention(state["q"], state["k"], state["v"], state["seq_begin"], out=state["out"])
        if kind == "decode":
            return state["pages"].decode(state["q"], state["table"], state["lengths"], out=state["out"])
        if kind == "store":
            state["pages"].write(state["k_rows"], state["v_rows"], state["seq_begin"], state["table"], first=state["first"])
            return _held(state)
        state["pages"].read(state["k_rows"], state["v_rows"], state["seq_begin"], state["table"], first=state["first"])
        return dict(k=state["k_rows"], v=state["v_rows"])
    return {"prompt": _plain_prompt, "decode": _plain_decode, "store": _plain_store, "load": _plain_load}[kind](state)


def _held(state):
    held = dict(k=state["k"], v=state["v"])
    return dict(held, k_exp=state["k_exp"], v_exp=state["v_exp"]) if state["case"]["e4m3"] else held


# ---- the plain forms, in 32 bits
def _power(exp):
    """2^exp, exactly"""
    return ((exp.to(torch.int32) + 127) << 23).view(torch.float32)


def _to_e4m3(x):
    """(numbers, exponents + 127): each row of d numbers over the least power of two, from 2^-126 on, that brings its largest to 448 at most."""
    x = x.float()
    size = x.abs()
    most = torch.where(torch.isfinite(size), size, 0.0).amax(-1)
    part, exp = torch.frexp(most)                       # most = part 2^exp, part in [1/2, 1); 448 = 7/8 2^9
    exp = torch.where(part > 0.875, exp - 8, exp - 9).clamp(min=-126)
    exp = torch.where(most > 0, exp, -126)
    scaled = torch.where(torch.isfinite(x), x * _power(-exp)[..., None], math.nan)
    return scaled.to(E4M3), (exp + 127).to(torch.uint8)


def _from_e4m3(x, exp):
    return x.float() * _power(exp.to(torch.int32) - 127)[..., None]


def _softmax(logits):
    most = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - torch.where(torch.isfinite(most), most, 0.0))
    return p / p.sum(-1, keepdim=True).clamp(min=1e-30)


def _plain_prompt(state):
    q, k, v, begin = state["q"], state["k"], state["v"], state["seq_begin"].long()
    n, hq, d = q.shape
    hkv, most, n_seqs = k.shape[1], state["longest"], begin.numel() - 1
    at = torch.arange(most, device=q.device)
    rows = (begin[:-1, None] + at).clamp(max=n - 1)                                           # [seqs, most]
    qs = q[rows].float().view(n_seqs, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n_seqs * hkv, -1, d)
    ks = k[rows].float().permute(0, 2, 3, 1).reshape(n_seqs * hkv, d, most)
    vs = v[rows].float().permute(0, 2, 1, 3).reshape(n_seqs * hkv, most, d)
    logits = torch.bmm(qs, ks).mul_(d ** -0.5).view(-1, most, most)
    o = torch.bmm(_softmax(logits.masked_fill_(at[:, None] < at, -math.inf)).view(n_seqs * hkv, -1, most), vs)
    o = o.view(n_seqs, hkv, hq // hkv, most, d).permute(0, 3, 1, 2, 4).reshape(n_seqs * most, hq, d)
    token = torch.arange(n, device=q.device)
    seq = (torch.searchsorted(begin, token, right=True) - 1).clamp(max=n_seqs - 1)
    place = seq * most + (token - begin[seq]).clamp(max=most - 1)
    return torch.where((token < begin[-1])[:, None, None], o[place].to(BF16), state["out"])


def _gathered(state, name, pages):
    """[..., heads, page, d] of the pages with these numbers, in 32 bits"""
    pages = pages.long()
    return _from_e4m3(state[name][pages], state[name + "_exp"][pages]) if state["case"]["e4m3"] else state[name][pages].float()


def _plain_decode(state):
    q, table, lengths = state["q"], state["table"].clamp(min=0), state["lengths"]
    (n_seqs, hq, d), width = q.shape, table.shape[1]
    hkv, page = state["case"]["hkv"], state["case"]["page"]
    k = _gathered(state, "k", table).permute(0, 2, 4, 1, 3).reshape(n_seqs * hkv, d, width * page)
    logits = torch.bmm(q.float().view(n_seqs * hkv, -1, d), k).mul_(d ** -0.5).view(n_seqs, hq, -1)
    del k
    seen = torch.arange(width * page, device=q.device) < lengths[:, None]
    p = _softmax(logits.masked_fill(~seen[:, None], -math.inf)).view(n_seqs * hkv, -1, width * page)
    v = _gathered(state, "v", table).permute(0, 2, 1, 3, 4).reshape(n_seqs * hkv, width * page, d)
    return torch.bmm(p, v).view(n_seqs, hq, d).to(BF16)


def _places(state):
    """(page, place in it) of every row"""
    begin, page = state["seq_begin"].long(), state["case"]["page"]
    token = torch.arange(state["k_rows"].shape[0], device=begin.device)
    seq = torch.searchsorted(begin, token, right=True) - 1
    at = token - begin[seq] + state["first"][seq]
    return state["table"][seq, at // page].long(), at % page


def _plain_store(state):
    pages, at = _places(state)
    for name in ("k", "v"):
        x = state[name + "_rows"]
        if state["case"]["e4m3"]:
            x, exp = _to_e4m3(x)
            state[name + "_exp"][pages, :, at] = exp
        state[name].view(torch.uint8)[pages, :, at] = x.contiguous().view(torch.uint8)
    return _held(state)


def _plain_load(state):
    pages, at = _places(state)
    for name in ("k", "v"):
        x = state[name][pages, :, at]
        if state["case"]["e4m3"]:
            x = _from_e4m3(x, state[name + "_exp"][pages, :, at])
        state[name + "_rows"].copy_(x)
    return dict(k=state["k_rows"], v=state["v_rows"])


# ---- what the operators are, in 64 bits
def _power_of_two(exp):
    return ((exp.long() + 1023) << 52).view(torch.float64)


def _row_of_pages(state, name, seq, head, length):
    """K or V of one sequence and head, [length, d] in 64 bits"""
    page = state["case"]["page"]
    pages = state["table"][seq, : -(-length // page)].long()
    x = state[name][pages, head].double()
    if state["case"]["e4m3"]:
        x = x * _power_of_two(state[name + "_exp"][pages, head].long() - 127)[..., None]
    return x.reshape(-1, x.shape[-1])[:length]


def _attend(q, k, v, causal):
    """[rows, d] in 64 bits"""
    logits = q @ k.T / math.sqrt(q.shape[-1])
    if causal:
        logits += torch.full_like(logits, -math.inf).triu_(1)
    return torch.softmax(logits, -1) @ v


def _e4m3_of(x):
    """The e4m3 numbers next to x, ties to the even one; four significant bits down to 2^-6, steps of 2^-9 below."""
    step = _power_of_two(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    state = prepare(case, seed)
    kind, lengths = case["kind"], _lengths(case)
    if kind == "prompt":
        out, begin, group = state["out"].double(), _begins(lengths), case["hq"] // case["hkv"]
        for seq, n in enumerate(lengths):
            at = slice(begin[seq], begin[seq] + n)
            for h in range(case["hq"] if n else 0):
                out[at, h] = _attend(state["q"][at, h].double(), state["k"][at, h // group].double(), state["v"][at, h // group].double(), True)
        return out
    if kind == "decode":
        out, group = torch.zeros(state["out"].shape, dtype=torch.float64, device=state["out"].device), case["hq"] // case["hkv"]
        for seq, n in enumerate(lengths):
            for h in range(case["hkv"] if n else 0):
                of = slice(h * group, (h + 1) * group)
                out[seq, of] = _attend(state["q"][seq, of].double(), _row_of_pages(state, "k", seq, h, n), _row_of_pages(state, "v", seq, h, n), False)
        return out
    begin, first, page = _begins(lengths), case["first"], case["page"]
    found = {}
    for name in ("k", "v"):
        rows = state[name + "_rows"].double()
        if kind == "load":
            for seq, n in enumerate(lengths):
                for h in range(case["hkv"]):
                    rows[begin[seq] : begin[seq] + n, h] = _row_of_pages(state, name, seq, h, first + n)[first:]
            found[name] = rows
            continue
        held = state[name].double()
        if case["e4m3"]:
            most = rows.abs().amax(-1).clamp(min=2.0 ** -149)
            exp = torch.ceil(torch.log2(most / 448)).clamp(min=-126)
            rows = _e4m3_of(rows / _power_of_two(exp)[..., None])
            exps = state[name + "_exp"].clone()
        for seq, n in enumerate(lengths):
            for at in range(first // page * page, first + n, page):         # a page at a time
                lo, hi = max(at, first), min(at + page, first + n)
                number, of = int(state["table"][seq, at // page]), slice(begin[seq] + lo - first, begin[seq] + hi - first)
                held[number, :, lo - at : hi - at] = rows[of].transpose(0, 1)
                if case["e4m3"]:
                    exps[number, :, lo - at : hi - at] = (exp[of].T + 127).to(torch.uint8)
        found[name] = held
        if case["e4m3"]:
            found[name + "_exp"] = exps
    return found


def work(case):
    """Rows of the pages read or written once (a byte for the exponent of an e4m3 row), the tables, and the other operands once."""
    lengths, d = _lengths(case), case["d"]
    n = sum(lengths)
    if case["kind"] == "prompt":
        return {"bytes": 2 * (2 * case["hq"] + 2 * case["hkv"]) * n * d + 4 * len(lengths), "flops": 4 * d * case["hq"] * sum(m * (m + 1) // 2 for m in lengths)}
    held = 2 * case["hkv"] * n * (d + 1 if case["e4m3"] else 2 * d) + 4 * sum(-(-m // case["page"]) for m in lengths)
    if case["kind"] == "decode":
        return {"bytes": held + 4 * len(lengths) * case["hq"] * d, "flops": 4 * d * case["hq"] * n}
    return {"bytes": held + 4 * case["hkv"] * n * d, "flops": 2 * case["hkv"] * n * d * 3 if case["e4m3"] else 0}
