"""A plain model of the paged 8-bit cache in 64 bits: what the tests of its operators compare with.  It keeps every sequence's
tokens as they went in and says what a cache has to hold and what attention over it has to give; where the cache's rounding
(to the 16-bit type, to a code) decides, it takes the codes and tails that the cache holds."""
import math

import torch

BT = 64
F64 = torch.float64


def rotate(x, cos_sin, pos, interleaved=False, sections=None):
    """x [n, heads, D] float64, cos_sin [positions, rot] as handed over, pos [axes, n]; also the size of what was added up."""
    rot = cos_sin.shape[1]
    pairs = rot // 2
    sections = [pairs] if sections is None else sections
    y, size, at = x.clone(), x.abs().clone(), 0
    for axis, width in enumerate(sections):
        p = torch.arange(at, at + width)
        at += width
        rows = cos_sin.double()[pos[axis].long()]
        c, s = rows[:, p][:, None], rows[:, pairs + p][:, None]
        i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + pairs)
        a, b = x[..., i], x[..., j]
        y[..., i], y[..., j] = a * c - b * s, b * c + a * s
        size[..., i] = size[..., j] = (a * c).abs() + (b * s).abs() + (b * c).abs() + (a * s).abs()
    return y, size


class Sequences:
    """Tokens that went into a cache, per sequence: lists of K (rotated, float64) with the size of its terms, and V."""

    def __init__(self, batch):
        self.k, self.size, self.v = ([[] for _ in range(batch)] for _ in range(3))

    def add(self, b, k, size, v):
        self.k[b].extend(k)
        self.size[b].extend(size)
        self.v[b].extend(v)


class Snapshot:
    """What a cache holds now, on the CPU."""

    def __init__(self, cache):
        self.codes = [x.cpu() for x in (cache.k_codes, cache.v_codes)]
        self.tails = [x.cpu() for x in (cache.k_tail, cache.v_tail)]
        self.scales, self.H, self.D = cache.scales.cpu().double(), cache.H, cache.D

    def held(self, page_row, tail, length):
        """K and V [length, H, D] float64 that the codes and the tail stand for."""
        out = []
        for which in (0, 1):
            parts = []
            for j in range(length // BT):
                page = int(page_row[j])
                tile = self.codes[which][page].float().double() * self.scales[page, :, which][:, None, None]
                parts.append((tile.transpose(1, 2) if which else tile).transpose(0, 1))
            if length % BT:
                parts.append(self.tails[which][int(tail)].double().transpose(0, 1)[:length % BT])
            out.append(torch.cat(parts) if parts else torch.zeros((0, self.H, self.D), dtype=F64))
        return out


def check_stored(cache, seqs, table, tails, lens):
    """What the cache holds against the tokens that went in, value by value.

    A key is rotated in binary32: two products and a sum, each off by at most 2^-24 of what it gives, so by at most
    3 * 2^-24 * size in all, and then rounded to the 16-bit type, at most eps / 2 of it (or half its smallest step).  A code is off
    by at most half a step: int8 scale / 2, e4m3 2^-4 of the value or half of 2^-9 scale; the factor that is multiplied with and the
    scale are each rounded once, and so is the product: 3 * 2^-24 of the value.  amax itself is off by what its value is."""
    eps = torch.finfo(cache.dtype).eps / 2
    tiny = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}[cache.dtype]
    int8 = cache.k_codes.dtype is torch.int8
    now = Snapshot(cache)
    for b, length in enumerate(lens):
        got = now.held(table[b], tails[b], length)
        if not length:
            continue
        for which, name in ((0, "K"), (1, "V")):
            want = torch.stack((seqs.v if which else seqs.k)[b][:length])
            slack = torch.zeros_like(want) if which else 3 * 2.0 ** -24 * torch.stack(seqs.size[b][:length])
            near = torch.zeros_like(want) if which else slack + eps * (want.abs() + slack) + tiny
            tol = near.clone()
            whole = length // BT * BT
            if whole:
                w = want[:whole].view(-1, BT, *want.shape[1:])
                amax = w.abs().amax(dim=(1, 3), keepdim=True)
                off = near[:whole].view_as(w).amax(dim=(1, 3), keepdim=True)
                scale = (amax + off) / (127 if int8 else 448)
                most = w.abs() + near[:whole].view_as(w)
                step = scale / 2 if int8 else torch.maximum(most * 2.0 ** -4, scale * 2.0 ** -10)
                step = torch.where(amax - off < 2.0 ** -100, torch.maximum(step.expand_as(w), most), step.expand_as(w))
                tol[:whole] += (step + 3 * 2.0 ** -24 * most * (1 + 2.0 ** -4)).view_as(tol[:whole])
            err = (got[which] - want).abs()
            assert bool((err <= tol).all()), (name, b, length, float((err - tol).max()), float((err / tol.clamp(min=1e-300)).max()))


def attention(q, k, v, scale, pos, window):
    """q [rows, Hq, D] at positions pos [rows] over k, v [length, H, D], float64: out, the mean of |v| under the weights,
    the largest sum of magnitudes that a score is made of, and the sum of |v| over the keys that a row sees."""
    rows, Hq, D = q.shape
    H = k.shape[1]
    G = Hq // H
    out, size = torch.zeros((rows, Hq, D), dtype=F64), torch.zeros((rows, Hq, D), dtype=F64)
    spread, plain = torch.zeros((rows, Hq, 1), dtype=F64), torch.zeros((rows, Hq, D), dtype=F64)
    if k.shape[0] == 0:
        return out, size, spread, plain
    j = torch.arange(k.shape[0])
    seen = j <= pos[:, None]
    if window:
        seen &= j > pos[:, None] - window
    any_ = seen.any(1)
    for g in range(Hq):
        s = q[:, g] @ k[:, g // G].t() * scale
        mass = q[:, g].abs() @ k[:, g // G].abs().t() * abs(scale)
        s = torch.where(seen, s, torch.full_like(s, -math.inf))
        p = torch.softmax(s, dim=-1)
        p = torch.where(any_[:, None], p, torch.zeros_like(p))
        vv = torch.where(seen.any(0)[:, None], v[:, g // G], torch.zeros_like(v[:, g // G]))
        out[:, g], size[:, g], plain[:, g] = p @ vv, p @ vv.abs(), seen.double() @ vv.abs()
        spread[:, g, 0] = torch.where(seen & torch.isfinite(mass), mass, torch.zeros_like(mass)).amax(1)
    return out, size, spread, plain
