"""Plain 64-bit forms of the span operators (torch on the CPU), and helpers that lay caches out.  Shares nothing with the library."""
import math

import torch

HALF_STEP = 2.0 ** -11          # rounding to IEEE half, relative
F32_STEP = 2.0 ** -24           # rounding to fp32, relative


class Cache:
    """Cache rows of one layer as values: k, v [B, Hkv, S, hd] (fp64), and the device tensors that hold them in one of the library's
    forms: half or block-scaled int16, contiguous or a pool of pages in no order."""

    def __init__(self, k, v, block_scaled=False, page=0, device="cuda:0", seed=0, spare=2, fill=float("nan")):
        self.B, self.Hkv, self.S, self.hd = k.shape
        self.page, self.block_scaled, self.device = page, block_scaled, device
        g = torch.Generator().manual_seed(seed)
        if page:
            assert self.S % page == 0
            n = self.B * (self.S // page)
            self.table = torch.randperm(n + spare, generator=g)[:n].to(torch.int32).view(self.B, self.S // page)
            self.lead = (n + spare, self.Hkv, page)
        else:
            self.table, self.lead = None, (self.B, self.Hkv, self.S)
        self.scales = [None, None]
        self.rows = []
        for i, x in enumerate((k, v)):
            if block_scaled:
                scale = (x.abs().amax(-1) / 32767).to(torch.float32)
                q = torch.where(scale[..., None] > 0, (x / scale[..., None].double()).round().clamp(-32767, 32767), 0.0).to(torch.int16)
                self.rows.append(self.place(q, torch.zeros(self.lead + (self.hd,), dtype=torch.int16) + 77))
                self.scales[i] = self.place(scale, torch.full(self.lead, fill))
            else:
                self.rows.append(self.place(x.to(torch.float16), torch.full(self.lead + (self.hd,), fill, dtype=torch.float16)))
        self.rows = [r.to(device) for r in self.rows]
        self.scales = [None if s is None else s.to(device) for s in self.scales]
        self.d_table = None if self.table is None else self.table.to(device)

    def index(self):
        """Flat row number of (b, h, j)."""
        b, h, j = (torch.arange(n) for n in (self.B, self.Hkv, self.S))
        if not self.page:
            return (b[:, None, None] * self.Hkv + h[:, None]) * self.S + j
        pages = self.table.long()[:, j // self.page]
        return (pages[:, None] * self.Hkv + h[:, None]) * self.page + (j % self.page)

    def place(self, x, into):
        flat = into.view((-1,) + x.shape[3:])
        flat[self.index().reshape(-1)] = x.reshape((-1,) + x.shape[3:])
        return into

    def values(self, i):
        """Rows as fp64 values [B, Hkv, S, hd], as the device holds them now (0: K, 1: V)."""
        r = self.rows[i].cpu().view(-1, self.hd)[self.index()].double()
        return r if self.scales[i] is None else r * self.scales[i].cpu().view(-1)[self.index()].double()[..., None]

    def raw(self, i):
        return self.rows[i].cpu().view(-1, self.hd)[self.index()]

    def args(self):
        return dict(kscale=self.scales[0], vscale=self.scales[1], table=self.d_table, page_size=self.page)


def attend(q, k, v, lens, T, span=None):
    """(out [B, T, Hq, hd], added weight [B, Hkv, S], valid [B, T]); q [B, T, Hq, hd], k, v [B, Hkv, S, hd], all fp64."""
    B, _, Hq, hd = q.shape
    Hkv, S = k.shape[1:3]
    out, add = torch.zeros_like(q), torch.zeros((B, Hkv, S), dtype=torch.float64)
    valid = torch.zeros((B, T), dtype=torch.bool)
    for b in range(B):
        n0 = min(max(int(lens[b]), 0), S)
        for t in range(T if span is None else min(max(int(span[b]), 0), T)):
            n = min(n0 + t + 1, S)
            valid[b, t] = True
            s = torch.einsum("hgd,hjd->hgj", q[b, t].view(Hkv, -1, hd), k[b, :, :n]) / math.sqrt(hd)
            p = torch.softmax(s, -1)
            out[b, t] = torch.einsum("hgj,hjd->hgd", p, v[b, :, :n]).reshape(Hq, hd)
            add[b, :, :n] += p.sum(1)
    return out, add, valid


def score_error(q, k, hd):
    """Absolute error of a score: q as a two-term half sum (2^-22 relative), products summed in fp32 in hd terms whose roundings
    have random signs (4 sigma), relative to the sum of magnitudes."""
    mags = float(q.abs().amax(-1).max() * k.abs().nan_to_num(0, 0, 0).sum(-1).max()) / math.sqrt(hd)
    return mags * (2.0 ** -22 + 4 * math.sqrt(hd) * F32_STEP)


def frequencies(rot, base, kind=0, factor=1.0, orig=0, low=1.0, high=32.0):
    if kind == 2:
        base = base * factor ** (rot / (rot - 2.0))
    f = [base ** (-2.0 * r / rot) for r in range(rot // 2)]
    if kind == 1:
        f = [x / factor for x in f]
    if kind == 3:
        def part(x):
            turns = orig * x / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - low) / (high - low)))
            return keep * x + (1 - keep) * x / factor
        f = [part(x) for x in f]
    return f


def rotate(x, pos, freq, rot, style):
    """x [..., hd] fp64 at positions pos (broadcast over the leading axes)."""
    y = x.clone()
    f = torch.tensor(freq, dtype=torch.float64)
    ang = pos[..., None].double() * f
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if style == 0 else (x[..., :rot // 2], x[..., rot // 2:rot])
    ra, rb = a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()
    if style == 0:
        y[..., 0:rot:2], y[..., 1:rot:2] = ra, rb
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = ra, rb
    return y


def evict(weight, pos, n, S, keep, recent):
    """source[slot] for slots 0 .. min(n, keep) - 1 of one slab (lists in, list out)."""
    n = min(max(n, 0), S)
    if n <= keep:
        return list(range(n))
    age = list(range(n)) if pos is None else pos[:n]
    newest = max(age)
    def rank(j):
        w = weight[j]
        return (0 if age[j] > newest - recent else 1, 0.0 if age[j] > newest - recent else (math.inf if w != w else -w), j)
    chosen = set(sorted(range(n), key=rank)[:keep])
    fillers = iter(sorted(j for j in chosen if j >= keep))
    return [j if j in chosen else next(fillers) for j in range(keep)]


def verify(target, draft, drafts, u, n, temperature):
    """One sequence: (accepted, tokens, logp) as lists; target [T+1, V], draft [T, V] or None, fp64."""
    T, V = target.shape[0] - 1, target.shape[1]
    greedy = not temperature > 0

    def probs(row):
        x = row / (1.0 if greedy else temperature)
        return torch.softmax(x, -1), torch.log_softmax(x, -1)

    def usable(row):
        return not bool(row.isnan().any()) and (greedy or math.isfinite(float(row.max())))

    tokens, logp, i, weight = [], [], 0, None
    while True:
        if not usable(target[i]):
            return i, tokens + [-1] * (T + 1 - i), logp + [0.0] * (T + 1 - i)
        p, lp = probs(target[i])
        best = int((target[i] == target[i].max()).nonzero()[0])
        if i == n:
            break
        x = int(drafts[i])
        inside = 0 <= x < V
        if greedy:
            ok = x == best
        else:
            if draft is None:
                q = torch.zeros(V, dtype=torch.float64)
                if inside:
                    q[x] = 1
            else:
                if not usable(draft[i]):
                    return i, tokens + [-1] * (T + 1 - i), logp + [0.0] * (T + 1 - i)
                q = probs(draft[i])[0]
            ok = inside and float(u[i]) * float(q[x]) < float(p[x])
            weight = (p - q).clamp(min=0)
        if not ok:
            break
        tokens.append(x)
        logp.append(float(lp[x]))
        i, weight = i + 1, None
    if greedy:
        new = best
    else:
        w = p if weight is None or not float(weight.sum()) > 0 else weight
        c = w.cumsum(0)
        above = (c > float(u[T]) * float(c[-1])) & (w > 0)
        new = int(above.nonzero()[0]) if bool(above.any()) else int((w > 0).nonzero()[-1])
    return i, tokens + [new] + [-1] * (T - i), logp + [float(lp[new])] + [0.0] * (T - i)
