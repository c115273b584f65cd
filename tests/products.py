"""Products of codes in 64 bits, and how far a correct result may be from them."""
import torch

INT8, INT4, ASYM = "int8", "int4", "int4_asym"


def random_codes(fmt, rows, d, gen, device="cuda"):
    """Codes over their whole range (the lowest ones too), scales of both signs and many sizes, zero points on both sides."""
    if fmt == INT8:
        codes = torch.randint(-128, 128, (rows, d), generator=gen, dtype=torch.int32).to(torch.int8)
    else:
        codes = torch.randint(0, 256, (rows, d // 2), generator=gen, dtype=torch.int32).to(torch.uint8)
    scales = torch.exp(torch.randn(rows, 2 if fmt == ASYM else 1, generator=gen)) * 0.01
    if fmt == ASYM:
        scales[:, 1] = torch.randint(-40, 12, (rows,), generator=gen).float()
    return codes.to(device), scales.to(device)


def whole(fmt, codes):
    """Codes as whole numbers in 64-bit floats: nibbles, the even code in the low one."""
    if fmt == INT8:
        return codes.double()
    c = codes.to(torch.int64)
    q = torch.stack((c & 15, c >> 4), -1).flatten(-2)
    return (q if fmt == ASYM else torch.where(q >= 8, q - 16, q)).double()


def code_sums(fmt, codes):
    return whole(fmt, codes).sum(-1).to(torch.int32)


def product(a_fmt, a, a_scales, w_fmt, w, w_scales):
    """(y, acc): the results, and s_t s_n |acc| of the sums before the zero points, whose rounding the results inherit.
    Sums are below 2^31, so 64-bit floats hold them exactly in any order."""
    acc = whole(a_fmt, a) @ whole(w_fmt, w).t()
    scale = a_scales[:, 0:1].double() * w_scales.double().reshape(1, -1)
    full = acc + (a_scales[:, 1:2].double() * whole(w_fmt, w).sum(1) if a_fmt == ASYM else 0.0)
    return full * scale, (acc * scale).abs()


def tolerance(y, acc, dtype):
    """Roundings by half a step of fp32, u = 2^-24: of the sum (of |acc|), the corrected sum and two products (of |y|), then one of
    the result's type; products of roundings are below a hundredth of u.  (fp16 below 2^-14: half its smallest step.)"""
    u = 2.0 ** -24
    fp32 = 1.01 * u * (acc + 3 * y.abs())
    return fp32 if dtype == torch.float32 else fp32 + torch.finfo(dtype).eps / 2 * (y.abs() + fp32) + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def compare(out, y, acc):
    error = (out.double() - y).abs()
    if out.dtype == torch.float16:
        # The largest fp16 is 65504 and its step 32, so what is 65520 or more before the last rounding becomes infinite, and nothing else does.
        before, infinite = tolerance(y, acc, torch.float32), torch.isinf(out)
        assert infinite[y.abs() - before >= 65520].all() and (y.abs() + before >= 65520)[infinite].all() and ((out > 0) == (y > 0))[infinite].all()
        error = torch.where(infinite, 0.0, error)
        out = torch.where(infinite, 0.0, out)
    over = error - tolerance(y, acc, out.dtype)
    assert torch.isfinite(out).all()
    worst = int(over.argmax())
    assert over.max() <= 0, "%d of %d too far, worst at %d: %r for %r" % (int((over > 0).sum()), over.numel(), worst, out.flatten()[worst].item(),
                                                                       y.flatten()[worst].item())
