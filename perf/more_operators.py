"""An 8-bit cache of keys and values in pages: writing it (with the keys' block rotation), reading it back, and the attention over
it, with or without a sliding window behind a few first tokens, each in plain torch and through the package.

`listed()` gives the fixed cases, `draw(rng)` further ones of the same ranges; `prepare` makes what a program holds on
the GPU before a call, `run` is one call (plain torch operations, or the package's entry points where `own` is true),
`work` what the call cannot do without, `exact` the same outputs in 64 bits.  Hidden sizes are the workload generator's 2048 and
4096, as heads of 64 and 128 channels.

The cache is int8 [pages, heads, page, D] with a step for each page and head, float [pages, heads], once for keys and once for values.
Sequence i has the rows offsets[i] .. offsets[i + 1] of a call; they are its last tokens, at positions lengths[i] - n .. lengths[i] - 1,
and position p lies in page pages[i, p // page].
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
PAGES = (16, 32, 64, 128)
MAX_ROWS = 16384                 # of a call
MAX_CACHE = 1 << 30              # bytes of codes that a call of few rows reads
MAX_PAIRS = 32 * 2 * 8192 * 4096  # (head, query, key) of a call


def _write(name, S, new, before, H, D, page, b, dtype, ragged):
    """S sequences that get up to `new` tokens behind up to `before`."""
    return {"name": name, "op": "write", "S": S, "new": new, "before": before, "H": H, "D": D, "page": page, "b": b, "type": dtype, "ragged": ragged}


def _read(name, S, new, before, H, D, page, b, dtype, ragged):
    return dict(_write(name, S, new, before, H, D, page, b, dtype, ragged), op="read")


def _attend(name, S, new, before, Hq, H, D, page, b, dtype, ragged, window=0, sinks=0):
    return dict(_write(name, S, new, before, H, D, page, b, dtype, ragged), op="attend", Hq=Hq, window=window, sinks=sinks)


def listed():
    return [
        # one token of one conversation: latency
        _write("write_1x1_d128_b128", 1, 1, 1000, 8, 128, 64, 128, "bf16", False),
        # a decode step of a large batch, each sequence somewhere inside a page
        _write("write_256x1_d128_b128", 256, 1, 4000, 8, 128, 64, 128, "bf16", True),
        # prompts of a prefill batch, ragged
        _write("write_4x4096_d128_b32", 4, 4096, 0, 8, 128, 128, 32, "bf16", True),
        # a short prefix for another precision's attention
        _read("read_3x200_d64_b64_f16", 3, 200, 0, 8, 64, 16, 64, "f16", True),
        # the whole cache of a batch that moves elsewhere
        _read("read_8x4096_d128_b128", 8, 4096, 0, 8, 128, 64, 128, "bf16", True),
        # one token of one conversation: latency
        _attend("attend_1x1_of_1000", 1, 1, 1000, 32, 8, 128, 64, 128, "bf16", False),
        # a decode step of a batch, ragged: bound by the cache
        _attend("attend_64x1_of_12000", 64, 1, 12000, 32, 8, 128, 64, 128, "bf16", True),
        # a decode step of few long documents
        _attend("attend_2x1_of_130000_f16", 2, 1, 130000, 32, 8, 128, 128, 64, "f16", True),
        # a few drafted tokens each, behind long contexts of which a window and the first tokens are kept in sight
        _attend("attend_32x5_window", 32, 5, 30000, 32, 4, 64, 32, 64, "bf16", True, 4096, 4),
        # a short ragged prompt batch of a small model, one head of keys to a head of queries
        _attend("attend_5x700_d64_f16", 5, 700, 0, 32, 32, 64, 16, 1, "f16", True),
        # the next chunk of long prompts
        _attend("attend_4x512_of_16000", 4, 512, 16000, 32, 8, 128, 64, 128, "bf16", True),
        # full prompts: the largest call
        _attend("attend_2x8192", 2, 8192, 0, 32, 8, 128, 128, 32, "bf16", True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choices(("write", "read", "attend"), (3, 2, 7))[0]
    D = rng.choice((64, 128, 128))
    c = {"op": op, "H": rng.choice((1, 2, 4, 8, 8)), "D": D, "page": rng.choice(PAGES), "b": rng.choice([v for v in (1, 16, 32, 64, 128) if v <= D]),
         "type": rng.choice(("bf16", "bf16", "f16")), "ragged": rng.random() < 0.8}
    if op != "attend":
        c["S"] = _log_int(rng, 1, 256)
        c["new"] = _log_int(rng, 1, MAX_ROWS // c["S"])
        c["before"] = rng.choice((0, _log_int(rng, 1, 4000)))
        return c
    c["Hq"] = c["H"] * rng.choice((1, 2, 3, 4, 6, 8) if c["H"] < 8 else (1, 2, 4, 5))
    per_token = 2 * c["H"] * D
    if rng.random() < 0.5:       # decode and drafted tokens
        c["S"] = _log_int(rng, 1, 256)
        c["new"] = rng.choice((1, 1, 2, 5, 8))
        c["before"] = _log_int(rng, 1, max(16, min(130000, MAX_CACHE // 2 // (c["S"] * per_token))))
    else:                        # prompts, and chunks of them
        c["S"] = _log_int(rng, 1, 8)
        c["new"] = _log_int(rng, 9, MAX_ROWS // c["S"] // 2)
        most = max(1, MAX_PAIRS // 2 // (c["Hq"] * c["S"] * c["new"]) - c["new"])
        c["before"] = rng.choice((0, _log_int(rng, 1, min(most, 32000))))
    c["window"], c["sinks"] = rng.choice(((0, 0), (0, 0), (_log_int(rng, 1, 8192), rng.choice((0, 4, 64)))))
    return c


# ------------------------------------------------------------------------------------------------------- inputs

def _sizes(case):
    """(rows, tokens) of every sequence, the same for every seed: between a third and all of the case's, or all."""
    gen = torch.Generator()
    gen.manual_seed(100003 * case["S"] + 1009 * case["new"] + case["before"])

    def part(most):
        low = -(-most // 3) if case["ragged"] else most
        return torch.randint(low, most + 1, (case["S"],), generator=gen)

    new = part(case["new"])
    return new, new + part(case["before"])


def _sum(v):
    return int(v.sum())


def _channels(shape, gen, spread):
    """Gaussian heads, of whose channels one in thirty-two is ten times larger in all tokens."""
    x = torch.randn(shape, generator=gen, device="cuda")
    large = torch.rand(shape[-2:], generator=gen, device="cuda") < 1 / 32
    return x * spread * torch.where(large, 10.0, 1.0)


def _codes(pages, H, page, D, gen, spread):
    """What a cache of gaussian (rotated) rows holds: codes whose largest is near 127, a step for each page and head."""
    codes = torch.empty((pages, H, page, D), dtype=torch.int8, device="cuda")
    at, step = 0, max(1, (1 << 26) // (H * page * D))
    while at < pages:
        part = codes[at:at + step]
        part.copy_(torch.clamp(torch.round(34.0 * torch.randn(part.shape, generator=gen, device="cuda")), -127, 127))
        at += step
    steps = torch.exp(0.3 * torch.randn((pages, H), generator=gen, device="cuda"))
    return codes, steps * (spread / 34.0)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    S, H, D, page = case["S"], case["H"], case["D"], case["page"]
    new, length = _sizes(case)
    T, width = _sum(new), -(-int(length.max()) // page)
    used = -(-length // page)
    dtype = DTYPES[case["type"]]
    s = {"op": case["op"], "page": page, "b": case["b"], "dtype": dtype, "T": T, "most": int(new.max()), "longest": int(length.max())}
    s["offsets"] = torch.cat((torch.zeros(1, dtype=torch.int64), new.cumsum(0))).to(torch.int32).cuda()
    s["lengths"] = length.to(torch.int32).cuda()
    # pages of the pool in any order; those behind a sequence's last are any too
    total = _sum(used) + 3
    place = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    first = torch.cat((torch.zeros(1, dtype=torch.int64), used.cumsum(0)[:-1])).cuda()
    s["pages"] = place[(first[:, None] + torch.arange(width, device="cuda")).clamp_max(total - 1)].contiguous()
    # (keys of length 1, so that logits have a spread of about two and a half)
    s["k_codes"], s["k_steps"] = _codes(total, H, page, D, gen, 0.7)
    s["v_codes"], s["v_steps"] = _codes(total, H, page, D, gen, 1.0)
    if case["op"] == "write":
        # keys and values as a projection of queries, keys and values leaves them, side by side
        row = _channels((T, 4 * H + 2 * H, D), gen, 0.7).to(dtype)
        s["k"], s["v"] = row[:, 4 * H:5 * H], row[:, 5 * H:]
    if case["op"] == "attend":
        s["q"] = _channels((T, case["Hq"], D), gen, 2.0).to(dtype)
        s["window"], s["sinks"], s["scale"] = case["window"], case["sinks"], D ** -0.5
    return s


# --------------------------------------------------------------------------------------------------- plain forms

def _rotated(x, b):
    """Blocks of b channels times the normalised Hadamard matrix, in x's type."""
    i = torch.arange(b, device=x.device)
    v = i[:, None] & i[None, :]
    v = v ^ (v >> 4)
    v = v ^ (v >> 2)
    sign = 1.0 - 2.0 * ((v ^ (v >> 1)) & 1).to(x.dtype)
    return (x.reshape(-1, b) @ sign).reshape(x.shape) / math.sqrt(b)


def _row_places(s):
    """Of every sequence, the rows that its first `most` tokens of the call have, and which of them there are."""
    begin, end = s["offsets"][:-1, None].long(), s["offsets"][1:, None].long()
    row = begin + torch.arange(s["most"], device="cuda")
    return row.clamp_max(max(0, s["T"] - 1)), row < end


def _plain_written(y, codes, steps, s):
    """Codes and steps after the call; in 64 bits, because codes are decided at borders."""
    page = s["page"]
    n = s["offsets"][1:].long() - s["offsets"][:-1].long()
    start, length = s["lengths"].long() - n, s["lengths"].long()
    first = start // page
    blocks = (s["most"] + page - 2) // page + 1
    number = first[:, None] + torch.arange(blocks, device="cuda")                              # [S, blocks]
    there = (n[:, None] > 0) & (number * page < length[:, None])
    place = s["pages"].long().gather(1, number.clamp_max(s["pages"].shape[1] - 1))
    position = number[:, :, None] * page + torch.arange(page, device="cuda")                   # [S, blocks, page]
    new = (position >= start[:, None, None]) & (position < length[:, None, None])
    row = (s["offsets"][:-1].long()[:, None, None] + position - start[:, None, None]).clamp(0, s["T"] - 1)
    fresh = torch.where(new[..., None, None], y[row], 0.0).transpose(2, 3)                    # [S, blocks, H, page, D]
    step = (fresh.abs().amax((3, 4)) / 127).float()
    before = torch.where((number * page < start[:, None])[..., None], steps[place], 0.0)       # of tokens that stay
    step = torch.maximum(step, before)
    wide = step.double()[..., None, None]
    safe = torch.where(wide > 0, wide, 1.0)
    q = torch.clamp(torch.round(fresh / safe), -127, 127)
    old = codes[place].double()
    old = torch.where(((step > before) & (before > 0))[..., None, None], torch.round(old * before.double()[..., None, None] / safe), old)
    stays = (position < start[:, None, None])[:, :, None, :, None]
    block = torch.where(new[:, :, None, :, None], q.to(torch.int8), torch.where(stays, old.to(torch.int8), codes[place]))
    codes[place[there]] = block[there]
    steps[place[there]] = step[there]


def _plain_write(s):
    _plain_written(_rotated(s["k"].double(), s["b"]), s["k_codes"], s["k_steps"], s)
    _plain_written(s["v"].double(), s["v_codes"], s["v_steps"], s)
    return s["k_codes"], s["k_steps"], s["v_codes"], s["v_steps"]


def _plain_read(s):
    row = torch.arange(s["T"], device="cuda")
    i = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
    position = s["lengths"].long()[i] - s["offsets"][1:].long()[i] + row
    place, slot = s["pages"].long()[i, position // s["page"]], position % s["page"]
    k = s["k_codes"][place, :, slot].float() * s["k_steps"][place][..., None]
    v = s["v_codes"][place, :, slot].float() * s["v_steps"][place][..., None]
    return _rotated(k, s["b"]).to(s["dtype"]), v.to(s["dtype"])


def _held(codes, steps, s):
    """[S, H, longest, D] of every sequence's tokens, in 32 bits."""
    place = s["pages"].long()
    x = codes[place].float() * steps[place][..., None, None]                                   # [S, width, H, page, D]
    return x.transpose(1, 2).flatten(2, 3)[:, :, :s["longest"]]


def _plain_attend(s):
    q = _rotated(s["q"].float(), s["b"])
    T, Hq, D = q.shape
    H = s["k_codes"].shape[1]
    row, there = _row_places(s)
    S, most = row.shape
    q = q[row].reshape(S, most, H, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(S, H, -1, D)
    x = (q * s["scale"]) @ _held(s["k_codes"], s["k_steps"], s).transpose(2, 3)                # [S, H, most * g, longest]
    n = s["offsets"][1:].long() - s["offsets"][:-1].long()
    i = ((s["lengths"].long() - n)[:, None] + torch.arange(most, device="cuda"))[:, None, :, None, None]
    j = torch.arange(s["longest"], device="cuda")
    seen = j <= i
    if s["window"]:
        seen = seen & ((j > i - s["window"]) | (j < s["sinks"]))
    x = x.reshape(S, H, most, Hq // H, -1).masked_fill_(~seen, -math.inf).reshape(S, H, most * (Hq // H), -1)
    top = x.amax(3, keepdim=True)
    x.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = x.sum(3, keepdim=True)
    y = (x @ _held(s["v_codes"], s["v_steps"], s)) / torch.where(total > 0, total, 1.0)
    y = y.reshape(S, H, most, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(S, most, Hq, D)
    return y[there].to(s["dtype"])


def run(s):
    if not own:
        return _plain_write(s) if s["op"] == "write" else _plain_read(s) if s["op"] == "read" else _plain_attend(s)
    from paper_2601_22347_b200 import binding as B
    cache = (s["k_codes"], s["k_steps"], s["v_codes"], s["v_steps"])
    if s["op"] == "write":
        B.perq_cache_write_i8(s["k"], s["v"], *cache, s["offsets"], s["lengths"], s["pages"], b=s["b"])
        return cache
    if s["op"] == "read":
        return B.perq_cache_read_i8(*cache, s["offsets"], s["lengths"], s["pages"], s["T"], b=s["b"], out_dtype=s["dtype"])
    return B.perq_attention_i8(s["q"], *cache, s["offsets"], s["lengths"], s["pages"], s["most"], b=s["b"], scale=s["scale"], window=s["window"],
                               sinks=s["sinks"])


# ---------------------------------------------------------------------------------------------------------- work

def _seen(new, length, window, sinks):
    """(pairs of a query and a key, keys that a query sees) of one head, over all sequences."""
    pairs = keys = 0
    for n, l in zip(new.tolist(), length.tolist()):
        i = torch.arange(l - n, l, dtype=torch.int64)
        low = (i - window + 1).clamp_min(0) if window else torch.zeros_like(i)
        first = torch.minimum(low, torch.full_like(i, sinks))
        pairs += _sum(i + 1 - low + first)
        keys += l - int(low[0]) + min(int(low[0]), sinks)
    return pairs, keys


def work(case):
    new, length = _sizes(case)
    T, H, D = _sum(new), case["H"], case["D"]
    if case["op"] != "attend":
        steps = 8 * H * _sum((length - 1) // case["page"] - (length - new) // case["page"] + 1)
        rotation = T * H * D * math.log2(case["b"])
        return {"bytes": T * H * D * 2 * 3 + steps, "flops": rotation + 4 * T * H * D}
    pairs, keys = _seen(new, length, case["window"], case["sinks"])
    return {"bytes": 2 * keys * H * D + 8 * H * keys // case["page"] + 2 * 2 * T * case["Hq"] * D, "flops": 4 * D * case["Hq"] * pairs}


# --------------------------------------------------------------------------------------------------------- exact

def _butterflies(x, b):
    """x times the Hadamard matrix of blocks of b, without its factor 1 / sqrt(b)."""
    half = b // 2
    while half >= 1:
        z = x.reshape(-1, 2, half)
        x = torch.stack((z[:, 0] + z[:, 1], z[:, 0] - z[:, 1]), 1).reshape(x.shape)
        half //= 2
    return x


def _token_places(s, i, begin, end):
    position = torch.arange(begin, end, device="cuda")
    return s["pages"][i].to(torch.int64)[torch.div(position, s["page"], rounding_mode="floor")], position % s["page"]


def _values(s, what, place, slot):
    return s[what + "_codes"][place, :, slot].to(torch.float64) * s[what + "_steps"][place].to(torch.float64)[:, :, None]


def exact(case, seed):
    s = prepare(case, seed)
    offsets, lengths = s["offsets"].tolist(), s["lengths"].tolist()
    root = math.sqrt(case["b"])
    if case["op"] == "write":
        steps = []
        for x, before in ((_butterflies(s["k"].to(torch.float64).contiguous(), case["b"]) / root, s["k_steps"]), (s["v"].to(torch.float64), s["v_steps"])):
            after = before.to(torch.float64)
            for i in range(case["S"]):
                n = offsets[i + 1] - offsets[i]
                place, slot = _token_places(s, i, lengths[i] - n, lengths[i])
                opened = place[slot == 0]
                after[opened] = 0.0
                top = x[offsets[i]:offsets[i + 1]].abs().amax(2) / 127
                after.scatter_reduce_(0, place[:, None].expand_as(top), top, "amax")
            steps.append(after)
        # codes are whole numbers, which have to be equal as they are
        return None, steps[0], None, steps[1]
    if case["op"] == "read":
        k, v = [], []
        for i in range(case["S"]):
            place, slot = _token_places(s, i, lengths[i] - (offsets[i + 1] - offsets[i]), lengths[i])
            k.append(_butterflies(_values(s, "k", place, slot), case["b"]) / root)
            v.append(_values(s, "v", place, slot))
        return torch.cat(k), torch.cat(v)
    q = _butterflies(s["q"].to(torch.float64), case["b"]) / root
    g = case["Hq"] // case["H"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for i in range(case["S"]):
        place, slot = _token_places(s, i, 0, lengths[i])
        k = _values(s, "k", place, slot).permute(1, 2, 0)
        v = _values(s, "v", place, slot).transpose(0, 1)
        n = offsets[i + 1] - offsets[i]
        for at in range(0, n, 256):
            rows = slice(offsets[i] + at, offsets[i] + min(n, at + 256))
            position = lengths[i] - n + at + torch.arange(rows.stop - rows.start, device="cuda")
            key = torch.arange(lengths[i], device="cuda")
            hidden = key[None, :] > position[:, None]
            if case["window"]:
                hidden |= (key[None, :] <= position[:, None] - case["window"]) & (key[None, :] >= case["sinks"])
            for h in range(g):
                part = q[rows, h::g].transpose(0, 1)
                x = (part @ k) * s["scale"]
                x[:, hidden] = -math.inf
                out[rows, h::g] = (torch.softmax(x, 2) @ v).transpose(0, 1)
    return out
