"""The operations around a paged cache in 64 bits, written from their definitions, and caches to try them on."""
import math

import torch


def turned(x, positions, frequencies, layout, amplitude=1.0, inverse=False):
    """x [..., d] with positions broadcast to x's leading dimensions; float64."""
    x = x.double().clone()
    r = 2 * frequencies.numel()
    first, second = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    angle = positions.double()[..., None] * frequencies.to(x.device) * (-1.0 if inverse else 1.0)
    a, b = x[..., first].clone(), x[..., second].clone()
    x[..., first] = amplitude * (a * angle.cos() - b * angle.sin())
    x[..., second] = amplitude * (b * angle.cos() + a * angle.sin())
    return x


class Paged:
    """A pool of pages in random order with the given (new tokens, length) pairs.  Places that no key uses hold NaN; new tokens lie behind
    `front` and in front of `behind` tokens of nobody."""

    def __init__(self, pairs, Hkv, d, page, seed=0, device="cuda", spare=3, front=0, behind=0, sigma=1.0, width=None):
        gen = torch.Generator().manual_seed(seed)
        self.pairs, self.Hkv, self.d, self.page, self.device = pairs, Hkv, d, page, device
        B = len(pairs)
        self.width = width or max(1, max(-(-max(n, 1) // page) for _, n in pairs))
        used = [-(-min(max(length, 0), self.width * page) // page) for _, length in pairs]
        self.pages = sum(used) + spare
        order = torch.randperm(self.pages, generator=gen).tolist()
        table = torch.full((B, self.width), -12345, dtype=torch.int32)  # entries behind a sequence name no page
        K = torch.full((self.pages, Hkv, page, d), float("nan"))
        V = torch.full((self.pages, Hkv, page, d), float("nan"))
        for b, (_, length) in enumerate(pairs):
            for i in range(used[b]):
                p = order.pop()
                table[b, i] = p
                n = min(page, min(length, self.width * page) - i * page)
                K[p, :, :n] = torch.randn(Hkv, n, d, generator=gen) * sigma
                V[p, :, :n] = torch.randn(Hkv, n, d, generator=gen)
        self.K, self.V = K.bfloat16().to(device), V.bfloat16().to(device)
        self.table = table.to(device)
        self.spare = order
        self.lengths = torch.tensor([length for _, length in pairs], dtype=torch.int32, device=device)
        starts = [front]
        for n, _ in pairs:
            starts.append(starts[-1] + n)
        self.starts = torch.tensor(starts, dtype=torch.int32, device=device)
        self.tokens = starts[-1] + behind
        self.gen = gen

    def normal(self, *shape, sigma=1.0):
        return (torch.randn(*shape, generator=self.gen) * sigma).bfloat16().to(self.device)

    def rows(self, cache, b, length):
        """The first `length` keys of sequence b, [Hkv, length, d] in float64; zeros where the table names no page."""
        at = torch.arange(length)
        pages = self.table[b].cpu().long()[at // self.page]
        good = (pages >= 0) & (pages < self.pages)
        x = cache.cpu().double()[pages.where(good, torch.tensor(0)), :, at % self.page].transpose(0, 1)
        return x * 1.0 if bool(good.all()) else x.where(good[None, :, None], torch.tensor(0.0, dtype=torch.float64))

    def attention(self, Q, scale):
        """O, lse, the weights each key receives, and for the tolerances: sum p |v| of each output and the largest |q . k|; rows of
        nobody stay NaN."""
        T, H, d = Q.shape
        G = H // self.Hkv
        O = torch.full((T, H, d), float("nan"), dtype=torch.float64)
        spread, lse = O.clone(), torch.full((T, H), float("nan"), dtype=torch.float64)
        mass = torch.zeros(len(self.pairs), self.Hkv, self.width * self.page, dtype=torch.float64)
        most = 0.0
        starts, lengths = self.starts.tolist(), self.lengths.tolist()
        q64 = Q.cpu().double()
        for b in range(len(self.pairs)):
            length = min(max(lengths[b], 0), self.width * self.page)
            n = starts[b + 1] - starts[b]
            if n <= 0:
                continue
            k, v = self.rows(self.K, b, length), self.rows(self.V, b, length)
            q = q64[starts[b]:starts[b + 1]].view(n, self.Hkv, G, d)
            raw = torch.einsum("ngrd,gjd->ngrj", q, k)
            z = raw * scale
            seen = torch.arange(length)[None, :] <= (length - n + torch.arange(n))[:, None]
            z = z.masked_fill(~seen[:, None, None, :], -math.inf)
            if length:
                most = max(most, float(raw.abs().max()))
                top = z.amax(-1, keepdim=True).clamp_min(-1e300)
                e = (z - top).exp()
                total = e.sum(-1, keepdim=True)
                p = e / total.clamp_min(1e-300)
                logs = torch.where(total > 0, top + total.log(), -math.inf).squeeze(-1)
            else:
                p, logs = z, torch.full((n, self.Hkv, G), -math.inf, dtype=torch.float64)
            O[starts[b]:starts[b + 1]] = torch.einsum("ngrj,gjd->ngrd", p, v).reshape(n, H, d)
            spread[starts[b]:starts[b + 1]] = torch.einsum("ngrj,gjd->ngrd", p, v.abs()).reshape(n, H, d)
            lse[starts[b]:starts[b + 1]] = logs.reshape(n, H)
            mass[b, :, :length] = p.sum((0, 2))
        return O, lse, mass, spread, most


def score_error(most, scale, d):
    """How far a scaled score may be off: the tensor cores add the 16 products of a step, and the sum so far, aligned to the largest of them and
    cut off below 24 bits, d / 16 times (17 terms each), and nothing in between is larger than some |q||k|, taken as 4 times the largest
    score; the float32 product with the scale adds a rounding."""
    return scale * 4 * most * ((d / 16) * 17 + 2) * 2.0 ** -24
