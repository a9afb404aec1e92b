"""The token operators from their definitions, in 64 bits on the CPU, and how far a kernel that holds its
sums in 32 bits may be from them.

Bounds, with u = 2^-24 (half a step of 32 bits, relative):
  z = scale * (x - m): three roundings, one of them the scale's product with a constant, so |z| 4u at most;
  exp(z): relative 4u |z| + 4u (the function's own error of a step or two);
  a sum of V such terms, all positive: at most V / 64 + 8 additions in a row (a wavefront shares a
  row, or more lanes do), each u relative to the whole;
  log of it: the sum's relative error + u |log| + 2u; the difference of two such numbers one rounding more.
With w = the mean of |z| under the row's probabilities the sum's relative error is
  S = u (4 w + V / 64 + 16)."""
import numpy as np
import torch

U = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}   # half the smallest step there is
NONE = -np.inf


def mask_bits(mask, n, v):
    """bool [n, v] from int32 words [n, words] or [words], None: all"""
    if mask is None:
        return np.ones((n, v), bool)
    w = np.atleast_2d(mask.cpu().numpy().view(np.uint32))
    bits = ((w[:, :, None] >> np.arange(32, dtype=np.uint32)) & 1).reshape(len(w), -1)[:, :v].astype(bool)
    return np.broadcast_to(bits, (n, v))


def words_of(bits):
    """int32 words [n, words] on the CPU of bool [n, v]"""
    n, v = bits.shape
    full = np.zeros((n, (v + 31) // 32 * 32), np.uint64)
    full[:, :v] = bits
    w = (full.reshape(n, -1, 32) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32)
    return torch.from_numpy(w.view(np.int32))


class Rows:
    """everything about rows of logits; `top` alternatives are listed"""

    def __init__(self, logits, token=None, mask=None, scale=1.0, top=0):
        x = logits.detach().cpu().double().numpy()
        n, v = x.shape
        scale = float(np.float32(scale))
        allowed = mask_bits(mask, n, v)
        self.token = None if token is None else token.cpu().numpy()
        self.padding = np.zeros(n, bool) if token is None else self.token < 0
        self.scale, self.allowed = scale, allowed
        with np.errstate(all="ignore"):
            self.bad = (allowed & (np.isnan(x) | (x == np.inf))).any(1) & ~self.padding
            x = np.where(allowed & ~self.bad[:, None] & ~self.padding[:, None], x, NONE)
            m = x.max(1)
            self.empty = m == NONE
            base = np.where(self.empty, 0.0, m)
            z = (x - base[:, None]) * scale
            e = np.exp(z)
            s = e.sum(1)
            log_sum = np.log(s)
            p = e / np.where(self.empty, 1.0, s)[:, None]
            zf = np.where(e > 0, z, 0.0)
            mean = (p * zf).sum(1)
            self.entropy = np.where(self.empty, 0.0, log_sum - mean)
            self.w, self.w2 = -mean, (p * zf * zf).sum(1)
            self.z, self.p, self.log_sum, self.x = z, p, log_sum, x
            self.stat = np.stack([m, log_sum], 1)
            self.sum_err = U * (4 * self.w + v / 64 + 16)
            fine = np.where(self.empty, 0.0, log_sum)
            self.log_err = self.sum_err + U * np.abs(fine) + 2 * U
            self.stat_err = np.stack([np.zeros(n), self.log_err], 1)
            # both parts of the difference: terms u (4 z^2 + 4 |z|) under p, the quotient 3u of it
            self.entropy_err = self.log_err + U * (4 * self.w2 + 4 * self.w) + self.w * (2 * self.sum_err + 3 * U) + U * np.abs(self.entropy)
            if token is not None:
                t = np.clip(self.token, 0, v - 1)
                self.inside = (self.token >= 0) & (self.token < v)
                zt = np.where(self.inside, z[np.arange(n), t], NONE)
                self.logprob = np.where(self.empty, NONE, zt - log_sum)
                self.logprob_err = np.where(np.isfinite(zt), 4 * U * np.abs(np.where(np.isfinite(zt), zt, 0)), 0) + self.log_err + U * np.where(np.isfinite(self.logprob), np.abs(self.logprob), 0)
                self.logprob[self.padding] = 0.0
                self.logprob[self.bad] = np.nan
            if top:
                k = min(top, v)
                order = np.argsort(-x, axis=1, kind="stable")[:, :k]
                best = np.take_along_axis(x, order, 1)
                none = best == NONE
                lq = np.take_along_axis(z, order, 1) - log_sum[:, None]
                fill = ((0, 0), (0, top - k))
                self.top_token = np.pad(np.where(none | self.bad[:, None], -1, order), fill, constant_values=-1)
                self.top_logprob = np.pad(np.where(none, NONE, lq), fill, constant_values=NONE)
                self.top_logprob[self.bad] = np.nan
                fin = np.where(np.isfinite(self.top_logprob), np.abs(self.top_logprob), 0)
                self.top_err = 5 * U * (fin + np.abs(fine)[:, None]) + self.log_err[:, None]
        for a in (self.entropy, self.stat):
            a[self.padding] = 0.0
            a[self.bad] = np.nan

    def grad(self, dtype, g=None, e=None):
        """(gradient, how far it may be)"""
        n, v = self.z.shape
        g = np.zeros(n) if g is None else g.cpu().double().numpy()
        e = np.zeros(n) if e is None else e.cpu().double().numpy()
        idle = self.padding | (self.empty & ~self.bad)
        with np.errstate(all="ignore"):
            ls = np.where(self.empty, 0.0, self.log_sum)[:, None]
            lp = np.where(self.p > 0, np.where(np.isfinite(self.z), self.z, 0) - ls, 0.0)
            h = np.where(np.isnan(self.entropy), 0, self.entropy)[:, None]
            hot = np.zeros((n, v))
            if self.token is not None:
                r = np.flatnonzero(self.inside)
                hot[r, self.token[r]] = 1.0
            inner = lp + h
            d = self.scale * (g[:, None] * (hot - self.p) - e[:, None] * self.p * inner)
            # p: exp of a number that is off by 4u |z| + the log's error, + 4u; each product and sum a rounding
            lp_err = 4 * U * np.abs(np.where(np.isfinite(self.z), self.z, 0)) + self.log_err[:, None] + 2 * U * np.abs(lp)
            p_err = self.p * (lp_err + 8 * U)
            h_err = np.where(np.isnan(self.entropy_err), 0, self.entropy_err)[:, None]
            err = np.abs(g)[:, None] * (p_err + U * (hot + self.p)) + np.abs(e)[:, None] * (p_err * np.abs(inner) + self.p * (lp_err + h_err + 2 * U * (np.abs(lp) + h)))
            err = self.scale * (err + 4 * U * (np.abs(g)[:, None] * (hot + self.p) + np.abs(e)[:, None] * self.p * np.abs(inner)))
            # what 32 bits hold of tiny probabilities: exp2 gives 0 below 2^-126
            err = err + self.scale * (np.abs(g)[:, None] + np.abs(e)[:, None] * (np.abs(inner) + 1)) * 2.0 ** -125
            err = err + HALF_STEP[dtype] * (np.abs(d) + err) + LEAST[dtype]
        d[idle] = 0.0
        err[idle] = 0.0
        d[self.bad] = np.nan
        d[~self.allowed] = 0.0
        err[~self.allowed] = 0.0
        return d, err


def near(got, want, err, what=""):
    got = got.detach().cpu().double().numpy()
    assert got.shape == want.shape, what
    want = np.where(np.abs(want) > 3.4028236e38, np.copysign(np.inf, want), want)   # what 32 bits do not hold
    odd = ~np.isfinite(want)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    assert same[odd].all(), f"{what}: {np.argwhere(odd & ~same)[:5].tolist()} got {got[odd & ~same][:5]} want {want[odd & ~same][:5]}"
    with np.errstate(all="ignore"):
        off = np.where(odd, 0.0, np.abs(got - want)) - np.where(odd, 0.0, err)
    assert not (off > 0).any() and not np.isnan(off).any(), \
        f"{what}: at {np.argwhere(~(off <= 0))[:5].tolist()} got {got[~(off <= 0)][:5]} want {want[~(off <= 0)][:5]} err {np.broadcast_to(err, want.shape)[~(off <= 0)][:5]}"


def advantages(counts, extra, off, weights, eps):
    """(reward, advantage) per sample, NaN where no group has it"""
    w = np.float32(weights).astype(float)
    n = len(extra) if counts is None else len(counts)
    r = np.zeros(n) if extra is None else extra.astype(float).copy()
    if counts is not None:
        r += (counts[:, 0] == 0) * w[0] + counts[:, 1] * w[1] + counts[:, 2] * w[2] + counts[:, 3] * w[3]
    reward, adv = np.full(n, np.nan), np.full(n, np.nan)
    for a, b in zip(off[:-1], off[1:]):
        a, b = min(a, n), min(b, n)
        if a < b:
            g = r[a:b] - r[a]
            reward[a:b] = r[a:b]
            adv[a:b] = (g - g.mean()) / (g.std() + float(np.float32(eps)))
    return reward, adv


def policy(lp, old, ref, start, length, adv, weight, lo, hi, kl):
    """gradient (NaN where no sample is), its error, loss, kl and their errors, tokens, clipped"""
    lp, old = lp.astype(float), old.astype(float)
    lo, hi, kl = (float(np.float32(v)) for v in (lo, hi, kl))
    n = len(lp)
    grad, err = np.full(n, np.nan), np.zeros(n)
    loss = kls = loss_err = kl_err = 0.0
    tokens = clipped = 0
    for c in range(len(start)):
        i = np.arange(min(int(start[c]), n), min(int(start[c]) + int(length[c]), n))
        if not len(i):
            continue
        a, w = float(adv[c]), float(weight[c])
        with np.errstate(all="ignore"):
            d = lp[i] - old[i]
            clip = (d > hi) if a > 0 else (d < lo) if a < 0 else np.zeros(len(i), bool)
            t = np.where(clip, hi if a > 0 else lo, d)
            part = -a * np.exp(t)
            # d is rounded to 32 bits (u |d|), exp is off by two steps, the products by a rounding each
            part_err = np.abs(part) * U * (np.abs(t) + 8)
            g, g_err = np.where(clip, 0.0, part), np.where(clip, 0.0, part_err)
            gap = np.zeros(len(i))
            if ref is not None:
                q = ref[i].astype(float) - lp[i]
                # q rounded: u |q| |exp(q) - 1|; the value itself: exp within 4u, minus q and 1, from |q| = 1/4 on; below it a sum of
                # terms of which the first is the largest
                gap = np.expm1(q) - q
                gap_err = U * (np.abs(q) * np.abs(np.expm1(q)) + np.where(np.abs(q) < 0.26, 16 * gap, 6 * (np.exp(q) + np.abs(q) + 1)))
                g = g - kl * np.expm1(q)
                g_err = g_err + abs(kl) * U * (np.abs(q) * np.exp(q) + 8 * np.abs(np.expm1(q)))
                part, part_err = part + kl * gap, part_err + abs(kl) * (gap_err + 2 * U * gap)
                kls += w * gap.sum()
                kl_err += abs(w) * gap_err.sum()
            grad[i] = w * g
            err[i] = np.abs(w) * (g_err + 4 * U * np.abs(g)) + 2.0 ** -148
            loss += w * part.sum()
            loss_err += abs(w) * (part_err + 2 * U * np.abs(part)).sum()
        tokens += len(i)
        clipped += int(clip.sum())
    return grad, err, loss, loss_err + U * abs(loss), kls, kl_err + U * abs(kls), tokens, clipped
