"""How far span attention may be off, element by element, and an emulation of its number formats on the CPU that shows that the bound
sees what it has to see.  Shares nothing with the library.

Counted, with independent roundings taken at four standard deviations (a rounding of at most u has a deviation of u / sqrt(3)):
  score     q as two half terms (2^-22 of every element, 2^-24 for its scaling), hd products of two terms summed in fp32, each sum off by 2^-24 of
            sums up to |q o k| + |q . k|; the factor 1 / sqrt(hd) log2(e), a row scale and the exponential's argument 2^-22 of the score each side
  weight    the exponential 2^-21; a probability as two half terms, the second one rounded to nearest: 2^-21 of itself, and 2^-32 of the
            largest probability (a half's smallest step 2^-24, the reference 2^7, half a step); block-scaled, of the largest probability times the row's largest |v|
  sums      n additions in fp32, 2^-24 of the sum of magnitudes each (the kernel adds up a lane's 8 keys of a tile before it adds them to a sum that may
            be large: additions of equal small numbers to a large one are no independent roundings)
  result    2^-11 of itself as a half, 2^-22 as two; 2^-25, half of the smallest step, where it is small
A relative error r_j of every weight moves a softmax's mean by sum_j p_j r_j |v_j - out|."""
import math

import torch

SIGMA4 = 4 / math.sqrt(3)


def bound(q, k, v, scales=None):
    """One query head: (out, p, tolerance of the first half term, tolerance of both) for q [hd], k, v [n, hd] (fp64 values); scales: the largest
    |v| of every row where rows are block-scaled."""
    n, hd = k.shape
    x = k * q
    s = x.sum(-1) / math.sqrt(hd)
    norm = x.norm(dim=-1)
    p = torch.softmax(s, -1)
    out = p @ v
    r = SIGMA4 * (1.25 * 2.0 ** -22 * norm + 2.0 ** -24 * math.sqrt(2 * hd) * (norm + s.abs() * math.sqrt(hd))) / math.sqrt(hd)
    r = r + (s.abs() + s.abs()[p.argmax()]) * 2.0 ** -22 + 2.0 ** -21
    tol = (p * r) @ (v - out).abs()
    tol = tol + SIGMA4 * 2.0 ** -21 * ((p ** 2) @ (v ** 2)).sqrt()
    if scales is None:
        tol = tol + SIGMA4 * 2.0 ** -32 * p.max() * (v ** 2).sum(0).sqrt()
    else:
        tol = tol + SIGMA4 * 2.0 ** -32 * (p * scales).max() * math.sqrt(n)
    tol = tol + SIGMA4 * 2.0 ** -24 * math.sqrt(n) * (p @ v.abs()) + 2.0 ** -21 * out.abs() + 2.0 ** -25
    return out, p, tol + 2.0 ** -11 * out.abs(), tol + 2.0 ** -22 * out.abs()


def attend(q, k, v, lens, T, block_scaled=False, span=None):
    """(out, tolerance of the half, tolerance of both halves, added weight, its tolerance) for q [B, T, Hq, hd], k, v [B, Hkv, S, hd]; NaN where
    there is no query."""
    B, _, Hq, hd = q.shape
    Hkv, S = k.shape[1:3]
    out, hi, both = (torch.full_like(q, float("nan")) for _ in range(3))
    add, add_tol = torch.zeros((B, Hkv, S), dtype=torch.float64), torch.zeros((B, Hkv, S), dtype=torch.float64)
    for b in range(B):
        n0 = min(max(int(lens[b]), 0), S)
        for t in range(T if span is None else min(max(int(span[b]), 0), T)):
            n = min(n0 + t + 1, S)
            for h in range(Hq):
                kv = h // (Hq // Hkv)
                kk, vv = k[b, kv, :n], v[b, kv, :n]
                out[b, t, h], p, hi[b, t, h], both[b, t, h] = bound(q[b, t, h], kk, vv, vv.abs().amax(-1) if block_scaled else None)
                add[b, kv, :n] += p
                # a weight: its score's error and that of the others' mean, the exponentials, the sum
                x = kk * q[b, t, h]
                r = SIGMA4 * (2.0 ** -21 * x.norm(dim=-1) + 2.0 ** -24 * math.sqrt(2 * hd) * (x.norm(dim=-1) + x.sum(-1).abs())) / math.sqrt(hd)
                r = r + 2.0 ** -20 + 2.0 ** -21 * (x.sum(-1).abs() + x.sum(-1).abs().max()) / math.sqrt(hd)
                add_tol[b, kv, :n] += p * (r + (p * r).sum() + SIGMA4 * 2.0 ** -24 * math.sqrt(n))
    return out, hi, both, add, add_tol


def _half(x, toward_zero=False):
    h = x.to(torch.float16)
    if toward_zero:
        over = h.float().abs() > x.abs()
        bits = h.view(torch.int16)
        h = torch.where(over, bits - 1, bits).view(torch.float16)       # one step towards zero, also from infinity
    return h.float()


def emulate(q, k, v, n, rows=None, mistake=None):
    """Span attention of one kv head in the kernel's formats: q [R, hd] over k, v [n, hd], four wavefronts' shares of tiles of 32.  rows:
    (integers, scales) of K and of V instead of k, v.  mistake: one of "q", "p", "rows" (a second half term left out), "tail"
    (probabilities split as they are), "reference" (the reference of block-scaled rows stays behind the maximum).  Returns out as fp32."""
    R, hd = q.shape
    scaled = rows is not None
    qs = q.float() * float(torch.tensor(hd ** -0.5 * math.log2(math.e), dtype=torch.float32))
    qh = _half(qs)
    ql = _half(qs - qh) if mistake != "q" else torch.zeros_like(qs)
    shift = 0.0 if scaled or mistake == "tail" else 7.0

    def terms(x):
        if not scaled:
            return x.to(torch.float16).float()
        i = x.to(torch.int32)
        return ((i >> 6).float() + ((i & 63).float() / 64 if mistake != "rows" else 0.0))

    ks, vs = (rows[0][1].float() * 64, rows[1][1].float()) if scaled else (None, None)
    kx, vx = (terms(rows[0][0]), terms(rows[1][0])) if scaled else (terms(k), terms(v))
    chunk = -(-(-(-n // 4)) // 32) * 32
    parts = []
    for w in range(4):
        m = torch.full((R, 1), -math.inf)
        den, ref, acc = torch.zeros(R, 1), torch.zeros(R, 1), torch.zeros(R, hd)
        for j in range(min(w * chunk, n), min((w + 1) * chunk, n), 32):
            e = min(j + 32, (w + 1) * chunk, n)
            s = qh @ kx[j:e].t() + ql @ kx[j:e].t()
            if scaled:
                s = s * ks[j:e]
            top = s.amax(-1, keepdim=True)
            if bool((top > m + 8).any()):
                new = torch.maximum(m, top)
                alpha = torch.where(m == -math.inf, torch.zeros_like(m), torch.exp2(m - new))
                m, den = new, den * alpha
                if scaled and mistake != "reference":
                    ref = ref * alpha
                else:
                    acc = acc * alpha
            x = torch.exp2(s - (m - shift))
            den = den + x.sum(-1, keepdim=True)
            if scaled:
                x = x * vs[j:e]
                big = x.amax(-1, keepdim=True)
                if bool((big > ref * 256).any()):
                    new = torch.maximum(ref, big)
                    acc = acc * torch.where(new > 0, ref / new, torch.zeros_like(ref))
                    ref = new
                x = torch.where(ref > 0, x * ((1.0 if mistake == "tail" else 128.0) / ref), torch.zeros_like(x))
            hi = _half(x, True)
            lo = _half(x - hi, mistake == "tail") if mistake != "p" else torch.zeros_like(x)
            acc = acc + (hi @ vx[j:e] + lo @ vx[j:e])
        if scaled:
            acc = acc * (ref * (64.0 if mistake == "tail" else 0.5))
        parts.append((m, den, acc))
    top = torch.stack([m for m, _, _ in parts]).amax(0)
    f = [torch.where(m == -math.inf, torch.zeros_like(m), torch.exp2(m - top)) for m, _, _ in parts]
    return sum(a * x for (_, _, a), x in zip(parts, f)) / sum(d * x for (_, d, _), x in zip(parts, f))
