"""The 8-bit cache and the attention over it in 64 bits, a sequence, a page and a head at a time, and how far a correct result may be from them."""
import math

import torch


def hadamard(b):
    i = torch.arange(b)
    parity = torch.tensor([bin(v).count("1") & 1 for v in range(b)])
    return 1.0 - 2.0 * parity[i[:, None] & i[None, :]].double()


def rotated(x, b):
    """Blocks of b channels times the normalised Hadamard matrix."""
    return x if b == 1 else (x.reshape(-1, b) @ hadamard(b)).reshape(x.shape) / math.sqrt(b)


class Cache:
    """Codes and steps on the CPU, written as the definition says."""

    def __init__(self, n_pages, heads, page, D, gen=None):
        self.page, self.D, self.heads, self.n_pages = page, D, heads, n_pages
        shape = (n_pages, heads, page, D)
        # (what pages held before says nothing)
        self.codes = [torch.randint(-127, 128, shape, generator=gen, dtype=torch.int32).to(torch.int8) for _ in range(2)]
        self.steps = [torch.rand((n_pages, heads), generator=gen) * 50 for _ in range(2)]

    def on_gpu(self):
        return tuple(t.cuda() for t in (self.codes[0], self.steps[0], self.codes[1], self.steps[1]))

    def write(self, k, v, offsets, lengths, pages, b):
        for kind, x in ((0, rotated(k.double(), b)), (1, v.double())):
            codes, steps = self.codes[kind], self.steps[kind]
            for i, length in enumerate(lengths):
                first = length - (offsets[i + 1] - offsets[i])
                for index in range(max(first, 0) // self.page, -(-length // self.page)):
                    at = int(pages[i, index])
                    if not 0 <= at < self.n_pages or length <= max(first, 0):
                        continue
                    begin, end = max(max(first, 0), index * self.page), min(length, (index + 1) * self.page)
                    rows = x[offsets[i] + begin - first:offsets[i] + end - first]                    # [n, heads, D]
                    slot = begin - index * self.page
                    for h in range(self.heads):
                        y = rows[:, h]
                        step = (y.abs().max() / 127).float()
                        if slot > 0:
                            old = steps[at, h].clone()
                            step = torch.maximum(step, old)
                            if step != old:
                                q = torch.clamp(torch.round(codes[at, h, :slot].double() * old.double() / step.double()), -127, 127)
                                codes[at, h, :slot] = torch.where(torch.isfinite(q) & bool(torch.isfinite(step)), q, 0.0).to(torch.int8)
                        q = torch.clamp(torch.round(y / step.double()), -127, 127) if bool(step > 0) and bool(torch.isfinite(step)) else torch.zeros_like(y)
                        codes[at, h, slot:slot + len(q)] = q.to(torch.int8)
                        steps[at, h] = step

    def tokens(self, kind, i, length, pages):
        """[length, heads, D] of sequence i."""
        j = torch.arange(length)
        at = pages[i, j // self.page].long()
        return self.codes[kind][at, :, j % self.page].double() * self.steps[kind][at].double()[..., None]


def visible(positions, length, window, sinks):
    """[rows, length]"""
    i, j = positions[:, None], torch.arange(length)
    seen = j <= i
    return seen & ((j > i - window) | (j < sinks)) if window else seen


def attention(cache, q, offsets, lengths, pages, b, scale, window=0, sinks=0):
    """(out, tolerance before the result's own rounding), [T, heads of queries, D]; rows of no sequence are NaN.

    Roundings that count: a query's channels, which move a logit by at most d_j = scale sum |dq| |k_j|.  Few rows: to whole multiples of the largest / 16256, so by 2^-15 of it; many
    rows: to fp16, 2^-11 of each where they are rotated (bf16 and fp16 are kept otherwise), or half of fp16's smallest step, 2^-25, of the largest; the sum of both covers either.  The
    rotation's, products', sums' and exponential's in fp32, (64 + |x_j|) 2^-22 in all; a probability times its step to
    fp16, 2^-11 of it, or 2^-25 of at least the largest.  out = sum p v / sum p, so it moves by sum p |v| (d + 2^-11) + |out| sum p d and, for the small ones, by at most
    length 2^-25 times the largest value."""
    T, Hq, D = q.shape
    g = Hq // cache.heads
    q = rotated(q.double(), b)
    out, tolerance = torch.full((T, Hq, D), math.nan, dtype=torch.float64), torch.zeros((T, Hq, D), dtype=torch.float64)
    for i, length in enumerate(lengths):
        rows, length = slice(offsets[i], offsets[i + 1]), max(length, 0)
        if rows.start == rows.stop:
            continue
        k, v = (cache.tokens(kind, i, length, pages) for kind in (0, 1))
        seen = visible(torch.arange(lengths[i] - (rows.stop - rows.start), lengths[i]), length, window, sinks)
        for h in range(Hq):
            kh, vh, qh = k[:, h // g], v[:, h // g], q[rows, h]
            x = ((qh @ kh.T) * scale).masked_fill(~seen, -math.inf)
            p = torch.nan_to_num(torch.softmax(x, 1), nan=0.0) * seen                    # (a row that sees nothing)
            y = p @ vh
            dq = (2.0 ** -11 if b > 1 else 0.0) * qh.abs() + 2.0 ** -15 * qh.abs().amax(1, keepdim=True)
            d = abs(scale) * (dq @ kh.abs().T) + (64 + torch.where(seen, x.abs(), 0.0) + abs(scale) * (qh.abs() @ kh.abs().T)) * 2.0 ** -22
            out[rows, h] = y
            most = torch.stack([vh[r].abs().amax() if bool(r.any()) else torch.zeros((), dtype=torch.float64) for r in seen]) if window else torch.cummax(
                torch.cat((torch.zeros(1), vh.abs().amax(1))), 0).values[(seen.sum(1))]
            tolerance[rows, h] = 1.05 * ((p * (d + 2.0 ** -11)) @ vh.abs() + y.abs() * (p * d).sum(1, keepdim=True)) + (seen.sum(1) * 2.0 ** -25 * most)[:, None]
    return out, tolerance


def half_step(y, dtype):
    return torch.finfo(dtype).eps / 2 * y.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def compare(out, y, tolerance):
    out = out.cpu()
    error, most = (out.double() - y).abs(), tolerance + half_step(y.abs() + tolerance, out.dtype)
    assert torch.isfinite(out).all()
    over = error - most
    worst = int(over.argmax())
    assert over.max() <= 0, "%d of %d too far, worst at %d: %r for %r, %r off, %r allowed" % (
        int((over > 0).sum()), over.numel(), worst, out.flatten()[worst].item(), y.flatten()[worst].item(), error.flatten()[worst].item(), most.flatten()[worst].item())


def table(lengths, page, n_pages, gen, width=None):
    """Pages of the pool in any order, none twice; those behind a sequence's last are none of the pool's."""
    used = [-(-max(n, 0) // page) for n in lengths]
    width = width or max(1, max(used))
    order = torch.randperm(n_pages, generator=gen)
    pages = torch.full((len(lengths), width), n_pages + 7, dtype=torch.int32)
    at = 0
    for i, n in enumerate(used):
        pages[i, :n] = order[at:at + n].to(torch.int32)
        at += n
    assert at <= n_pages
    return pages


def starts(rows):
    offsets = [0]
    for n in rows:
        offsets.append(offsets[-1] + n)
    return offsets


def ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()
