"""The 8-bit integer linear layers that read the path's codes: a rotation with 8-bit codes, the product of codes with a
scale for each token and channel, and that product grouped by expert, each in plain torch and through the package.

`listed()` gives the fixed cases, `draw(rng)` further ones of the same ranges; `prepare` makes what a program holds on
the GPU before a call, `run` is one call (plain torch operations, or the package's entry points where `own` is true),
`work` what the call cannot do without, `exact` the same outputs in 64 bits.  Widths are the workload generator's
(hidden sizes 2048 and 4096, down-projection inputs 8192 and 14336) and the ragged 9728 of the paper's tables.
"""
import math

import torch

own = False

INT4, INT4_ASYM, INT8 = "int4", "int4_asym", "int8"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HIDDEN = (2048, 4096)
WIDTHS = (2048, 4096, 6144, 8192, 9728, 14336)
MAX_TOKENS = 16384
MAX_PRODUCT = MAX_TOKENS * 4096 * 14336
MAX_EXPERT_WEIGHTS = 32 * 2048 * 4096


def _quant(name, T, d, b, perm):
    return {"name": name, "op": "quant", "T": T, "d": d, "b": b, "perm": perm}


def _linear(name, T, N, d, a, w, out):
    return {"name": name, "op": "linear", "T": T, "N": N, "d": d, "a": a, "w": w, "out": out}


def _moe(name, T, E, N, d, a, w, out, skew, spare):
    return {"name": name, "op": "moe", "T": T, "E": E, "N": N, "d": d, "a": a, "w": w, "out": out, "skew": skew, "spare": spare}


def listed():
    return [
        # one token of a decode step, rotated to 8-bit codes: latency
        _quant("quant_1x4096_b32", 1, 4096, 32, False),
        # a ragged prompt at a ragged down-projection width, channels permuted
        _quant("quant_1531x9728_b128_perm", 1531, 9728, 128, True),
        # the hidden states of a full prefill batch
        _quant("quant_16384x4096_b32", 16384, 4096, 32, False),
        # one token through a down projection of 4-bit codes: latency, bound by the weights
        _linear("linear_1x4096x14336_w4a4", 1, 4096, 14336, INT4, INT4, "bf16"),
        # a decode batch through an up projection, 8-bit tokens with 4-bit weights
        _linear("linear_16x14336x4096_w4a8", 16, 14336, 4096, INT8, INT4, "bf16"),
        # a short prompt at a small hidden size, fp32 results
        _linear("linear_256x2048x2048_w8a8_f32", 256, 2048, 2048, INT8, INT8, "f32"),
        # a prompt with the paper's asymmetric 4-bit activations
        _linear("linear_2048x4096x4096_w4a4_asym", 2048, 4096, 4096, INT4_ASYM, INT4, "bf16"),
        # a ragged prompt, a ragged width and an odd number of channels
        _linear("linear_1531x1001x9728_w8a8_f16", 1531, 1001, 9728, INT8, INT8, "f16"),
        # the down projection of a full prefill batch: the largest call
        _linear("linear_16384x4096x14336_w8a8", 16384, 4096, 14336, INT8, INT8, "bf16"),
        # a decode batch over many experts, a row or two to each and some without any: bound by the weights
        _moe("moe_64x32e_2048x4096_w4a4", 64, 32, 2048, 4096, INT4, INT4, "bf16", 1.0, 0),
        # a prompt over many experts, ragged
        _moe("moe_4099x32e_2048x4096_w8a8", 4099, 32, 2048, 4096, INT8, INT8, "bf16", 0.7, 0),
        # a large prompt over few experts in 4-bit codes, in a buffer with rows to spare
        _moe("moe_8192x8e_4096x2048_w4a4", 8192, 8, 4096, 2048, INT4, INT4, "bf16", 0.5, 64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _formats(rng):
    return rng.choice(((INT8, INT8), (INT8, INT8), (INT4, INT4), (INT4, INT4), (INT4_ASYM, INT4), (INT8, INT4), (INT4_ASYM, INT8), (INT4, INT8)))


def draw(rng):
    op = rng.choices(("quant", "linear", "moe"), (3, 6, 4))[0]
    # one width in four is ragged: any multiple of 32
    d = rng.choice(WIDTHS) if rng.random() < 0.75 else 32 * rng.randint(2, 448)
    if op == "quant":
        b = rng.choice([v for v in (1, 16, 32, 64, 128, 256, 512) if d % v == 0])
        return {"op": op, "T": _log_int(rng, 1, min(MAX_TOKENS, MAX_TOKENS * 8192 // d)), "d": d, "b": b, "perm": rng.random() < 0.3}
    a, w = _formats(rng)
    out = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op == "linear":
        N = rng.choice(WIDTHS) if rng.random() < 0.6 else _log_int(rng, 1, 14336)
        return {"op": op, "T": _log_int(rng, 1, max(1, min(MAX_TOKENS, MAX_PRODUCT // (N * d)))), "N": N, "d": d, "a": a, "w": w, "out": out}
    d = rng.choice(HIDDEN) if rng.random() < 0.6 else 32 * rng.randint(2, 128)
    E = rng.choice((2, 4, 7, 8, 16, 32, 60, 64))
    N = min(_log_int(rng, 64, 4096), max(1, MAX_EXPERT_WEIGHTS // (E * d)))
    return {"op": op, "T": _log_int(rng, 1, 8192), "E": E, "N": N, "d": d, "a": a, "w": w, "out": out,
            "skew": round(rng.uniform(0.0, 2.5), 2), "spare": rng.choice((0, 0, 1, 40))}


# ------------------------------------------------------------------------------------------------------- inputs

def _activations(T, d, gen):
    """bf16 rows as the workload generator has them: laplace values, one channel in a thousand 200 times larger."""
    u = torch.rand(T, d, generator=gen, device="cuda") - 0.5
    v = -u.sign() * torch.log1p(-2 * u.abs()).clamp_min(-20.0)
    v[:, torch.randperm(d, generator=gen, device="cuda")[:max(1, d // 1000)]] *= 200.0
    return v.to(torch.bfloat16)


def _packed(codes):
    """Two codes to a byte, the even one in the low nibble."""
    c = codes.to(torch.int16) & 15
    return (c[..., 0::2] | (c[..., 1::2] << 4)).to(torch.uint8)


def _codes(fmt, rows, d, gen, spread):
    """Codes and scales of `rows` rotated rows, which are close to gaussian, each with a magnitude of its own."""
    codes = torch.empty((rows, d if fmt == INT8 else d // 2), dtype=torch.int8 if fmt == INT8 else torch.uint8, device="cuda")
    scales = torch.empty((rows, 2 if fmt == INT4_ASYM else 1), device="cuda")
    for at in range(0, rows, 16384):
        y = torch.randn(min(16384, rows - at), d, generator=gen, device="cuda")
        y *= spread * torch.exp(0.5 * torch.randn(len(y), 1, generator=gen, device="cuda"))
        part = slice(at, at + len(y))
        if fmt == INT4_ASYM:
            low, high = y.amin(1, keepdim=True), y.amax(1, keepdim=True)
            s = (high - low) / 15
            z = torch.round(low / s)
            codes[part] = _packed(torch.clamp(torch.round(y / s) - z, 0, 15))
            scales[part] = torch.cat((s, z), 1)
            continue
        top = 127 if fmt == INT8 else 7
        s = y.abs().amax(1, keepdim=True) / top
        q = torch.clamp(torch.round(y / s), -top, top)
        codes[part] = q.to(torch.int8) if fmt == INT8 else _packed(q)
        scales[part] = s
    return codes, scales


def _unpacked(fmt, codes):
    """Codes as fp32 whole numbers."""
    if fmt == INT8:
        return codes.float()
    c = codes.view(torch.uint8)
    q = torch.stack((c & 15, c >> 4), -1).flatten(-2).float()
    return q if fmt == INT4_ASYM else q - 16.0 * (q >= 8)


def _rows_of_experts(case):
    """How many rows each expert gets, the same for every seed: rows choose by shares whose logarithms are gaussian."""
    gen = torch.Generator()
    gen.manual_seed(1000 * case["T"] + case["E"])
    share = torch.softmax(case["skew"] * torch.randn(case["E"], generator=gen), 0)
    return torch.bincount(torch.multinomial(share, case["T"], replacement=True, generator=gen), minlength=case["E"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    T, d = case["T"], case["d"]
    if case["op"] == "quant":
        x = _activations(T, d, gen)
        perm = torch.randperm(d, generator=gen, device="cuda").to(torch.int32) if case["perm"] else None
        return {"op": "quant", "x": x, "b": case["b"], "perm": perm}
    N, E = case["N"], case.get("E", 1)
    s = {"op": case["op"], "a_fmt": case["a"], "w_fmt": case["w"], "dtype": DTYPES[case["out"]]}
    total = T + case.get("spare", 0)
    s["a"], s["a_scales"] = _codes(case["a"], total, d, gen, 1.0)
    s["w"], s["w_scales"] = _codes(case["w"], E * N, d, gen, 0.02)
    s["w_scales"] = s["w_scales"].reshape(E, N)
    # the sums of the weights' codes belong to asymmetric tokens; they are made once, with the weights
    s["w_sums"] = _unpacked(case["w"], s["w"]).sum(1).to(torch.int32).reshape(E, N) if case["a"] == INT4_ASYM else None
    if case["op"] == "linear":
        s["w_scales"] = s["w_scales"].reshape(N)
        s["w_sums"] = None if s["w_sums"] is None else s["w_sums"].reshape(N)
        return s
    rows = _rows_of_experts(case)
    s["w"] = s["w"].reshape(E, N, -1)
    s["offsets"] = torch.cat((torch.zeros(1, dtype=torch.int64), rows.cumsum(0))).to(torch.int32).cuda()
    s["most"] = int(rows.max())                                        # of one expert: the plain form's batch
    s["out"] = torch.zeros((total, N), dtype=s["dtype"], device="cuda")
    return s


# --------------------------------------------------------------------------------------------------- plain forms

def _hadamard(b):
    i = torch.arange(b, device="cuda")
    v = i[:, None] & i[None, :]
    v = v ^ (v >> 8)
    v = v ^ (v >> 4)
    v = v ^ (v >> 2)
    return 1.0 - 2.0 * ((v ^ (v >> 1)) & 1).double()


def _plain_quant(s):
    """In 64 bits, because codes are decided at borders."""
    x = s["x"] if s["perm"] is None else s["x"][:, s["perm"].long()]
    T, d = x.shape
    u = (x.double().reshape(-1, s["b"]) @ _hadamard(s["b"])).reshape(T, d)         # sqrt(b) times the rotated row
    top = u.abs().amax(1, keepdim=True)
    q = torch.round(127.0 * u / torch.where(top > 0, top, 1.0))
    return q.to(torch.int8), (top / (127.0 * math.sqrt(s["b"]))).float()


def _scaled(acc, s, a_scales, w_scales, w_sums):
    if s["a_fmt"] == INT4_ASYM:
        acc = acc + a_scales[..., 1:2] * w_sums.float()
    return (acc * a_scales[..., 0:1] * w_scales).to(s["dtype"])


def _plain_linear(s):
    acc = _unpacked(s["a_fmt"], s["a"]) @ _unpacked(s["w_fmt"], s["w"]).t()
    return _scaled(acc, s, s["a_scales"], s["w_scales"], s["w_sums"])


def _plain_moe(s):
    """Rows of every expert in a batch as long as the largest one's, one batched product."""
    offsets = s["offsets"].long()
    a, (E, N) = s["a"], s["w_scales"].shape
    row = torch.arange(len(a), device="cuda")
    expert = torch.searchsorted(offsets, row, right=True) - 1
    used = row < offsets[-1]
    expert = torch.where(used, expert, 0)
    # rows of no expert go to a place behind the batches
    place = torch.where(used, expert * s["most"] + row - offsets[expert], E * s["most"])
    batch = torch.zeros((E * s["most"] + 1, a.shape[1] if s["a_fmt"] == INT8 else 2 * a.shape[1]), device="cuda")
    batch[place] = _unpacked(s["a_fmt"], a)
    w = _unpacked(s["w_fmt"], s["w"])
    acc = torch.bmm(batch[:-1].reshape(E, s["most"], -1), w.transpose(1, 2)).reshape(-1, N)
    acc = acc[torch.where(used, place, 0)]
    out = _scaled(acc, s, s["a_scales"], s["w_scales"][expert], None if s["w_sums"] is None else s["w_sums"][expert])
    return torch.where(used[:, None], out, s["out"])


def run(s):
    if not own:
        return _plain_quant(s) if s["op"] == "quant" else _plain_linear(s) if s["op"] == "linear" else _plain_moe(s)
    from paper_2601_22347_b200 import binding as B
    if s["op"] == "quant":
        return B.perq_rotate_quantize_i8(s["x"], s["perm"], s["b"])
    a_fmt, w_fmt = B.FMT_BY_NAME[s["a_fmt"]], B.FMT_BY_NAME[s["w_fmt"]]
    if s["op"] == "linear":
        return B.perq_matmul_i8(s["a"], s["a_scales"], a_fmt, s["w"], s["w_scales"], w_fmt, s["w_sums"], out_dtype=s["dtype"])
    return B.perq_grouped_matmul_i8(s["a"], s["a_scales"], a_fmt, s["w"], s["w_scales"], w_fmt, s["offsets"], s["w_sums"], out=s["out"])


# ---------------------------------------------------------------------------------------------------------- work

def _bytes_of(fmt, rows, d):
    return rows * (d if fmt == INT8 else d // 2) + rows * (8 if fmt == INT4_ASYM else 4)


def work(case):
    T, d = case["T"], case["d"]
    if case["op"] == "quant":
        return {"bytes": T * (3 * d + 4) + (4 * d if case["perm"] else 0), "flops": T * d * (math.log2(case["b"]) + 3)}
    N = case["N"]
    weights = N if case["op"] == "linear" else N * int((_rows_of_experts(case) > 0).sum())      # of experts that have rows
    extra = 4 * weights if case["a"] == INT4_ASYM else 0
    return {"bytes": _bytes_of(case["a"], T, d) + _bytes_of(case["w"], weights, d) + extra + T * N * DTYPES[case["out"]].itemsize,
            "flops": 2 * T * N * d}


# --------------------------------------------------------------------------------------------------------- exact

def _whole(fmt, codes):
    """Codes as 64-bit floats, from their bits."""
    if fmt == INT8:
        return codes.to(torch.float64)
    byte = codes.to(torch.int64)
    q = torch.empty(*byte.shape[:-1], 2 * byte.shape[-1], dtype=torch.float64, device=byte.device)
    low, high = byte % 16, byte // 16
    q[..., 0::2] = (low if fmt == INT4_ASYM else (low + 8) % 16 - 8).to(torch.float64)
    q[..., 1::2] = (high if fmt == INT4_ASYM else (high + 8) % 16 - 8).to(torch.float64)
    return q


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quant":
        x = s["x"].to(torch.float64)
        y = x if s["perm"] is None else x.index_select(1, s["perm"].to(torch.int64))
        y = y.reshape(case["T"], case["d"] // case["b"], case["b"])
        half = case["b"] // 2
        while half >= 1:                                # butterflies: the halves of every run of 2 * half
            z = y.reshape(case["T"], -1, 2, half)
            y = torch.stack((z[:, :, 0] + z[:, :, 1], z[:, :, 0] - z[:, :, 1]), 2)
            half //= 2
        # codes are whole numbers, which have to be equal as they are
        return None, y.reshape(case["T"], -1).abs().amax(1, keepdim=True) / (127 * case["b"] ** 0.5)
    value = _whole(case["a"], s["a"])
    if case["a"] == INT4_ASYM:
        value = value + s["a_scales"][:, 1:2].to(torch.float64)
    value = value * s["a_scales"][:, 0:1].to(torch.float64)
    if case["op"] == "linear":
        return value @ (_whole(case["w"], s["w"]) * s["w_scales"].to(torch.float64)[:, None]).t()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    at = s["offsets"].tolist()
    for e in range(case["E"]):
        w = _whole(case["w"], s["w"][e]) * s["w_scales"][e].to(torch.float64)[:, None]
        out[at[e]:at[e + 1]] = value[at[e]:at[e + 1]] @ w.t()
    return out
