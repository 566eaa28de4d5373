"""The layer operators' definitions in float64 (plain torch; attention on the GPU where there is one), for their tests, with the bounds that their
results have to keep.

u = 2^-24 is half a step of fp32, H half a step of the results' type (2^-8 for bf16, u for fp32).  A sum of n
fp32 terms in any order is off by at most n u times the sum of their magnitudes; products of bf16 values are
exact in fp32.  Every bound is |error| <= H |result| + what the sums and, for bf16 attention, the operands
rounded between two products may do; the sums of magnitudes that they need are formed beside the results.
"""
import math

import torch

U = 2.0 ** -24
F64 = torch.float64


def half(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def within(got, ref, bound, what):
    """|got - ref| <= bound in every element (NaN only where ref has it)."""
    got = got.detach().cpu().to(F64)
    assert got.shape == ref.shape, (what, tuple(got.shape), tuple(ref.shape))
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN elsewhere than in the definition"
    fine = ~torch.isnan(ref)
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]), f"{what}: infinities"
    fine &= ~inf
    over = ((got - ref).abs() - bound)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, \
        f"{what}: off by up to {float((got - ref).abs()[fine].max()):.3e}, {float(over.max()):.3e} over its bound"


# ---- LayerNorm ---------------------------------------------------------------

def norm(x, gamma, beta, residual, eps, dtype):
    """(y, bound), (h, bound)"""
    x, gamma, beta = x.to(F64), gamma.to(F64), beta.to(F64)
    h = x if residual is None else x + residual.to(F64)
    w = h.shape[1]
    mean = h.mean(1, keepdim=True)
    var = ((h - mean) ** 2).mean(1, keepdim=True)
    rstd = 1 / (var + eps).sqrt()
    xhat = (h - mean) * rstd
    y = xhat * gamma + beta
    H = half(dtype)
    # h, its mean (w terms), the centred value; rstd is off relatively by half the variance's relative error
    e_c = U * ((w + 2) * h.abs().mean(1, keepdim=True) + 3 * h.abs())
    e_v = 2 * rstd ** 2 * ((h - mean).abs() * e_c).mean(1, keepdim=True) + (w + 4) * U
    e_x = rstd * e_c + xhat.abs() * (e_v / 2 + 4 * U)
    return (y, H * y.abs() + (gamma.abs() * e_x + 4 * U * (xhat * gamma).abs() + 2 * U * beta.abs()) * (1 + 2 * H)), \
        (h, H * h.abs() * (1 + 2 * U) + U * h.abs())


def norm_backward(h, gamma, dy, dsum, eps, dtype):
    """(dh, bound), (dgamma, bound), (dbeta, bound)"""
    h, gamma, dy = h.to(F64), gamma.to(F64), dy.to(F64)
    rows, w = h.shape
    mean = h.mean(1, keepdim=True)
    var = ((h - mean) ** 2).mean(1, keepdim=True)
    rstd = 1 / (var + eps).sqrt()
    xhat = (h - mean) * rstd
    g = dy * gamma
    m1, m2 = g.mean(1, keepdim=True), (g * xhat).mean(1, keepdim=True)
    dh = rstd * (g - m1 - xhat * m2)
    if dsum is not None:
        dh = dh + dsum.to(F64)
    H = half(dtype)
    e_c = U * ((w + 2) * h.abs().mean(1, keepdim=True) + 3 * h.abs())
    e_v = 2 * rstd ** 2 * ((h - mean).abs() * e_c).mean(1, keepdim=True) + (w + 4) * U
    e_x = rstd * e_c + xhat.abs() * (e_v / 2 + 4 * U)
    a1, a2 = g.abs().mean(1, keepdim=True), (g * xhat).abs().mean(1, keepdim=True)
    e_m2 = (w + 3) * U * a2 + (g.abs() * e_x).mean(1, keepdim=True)
    inner = g.abs() + a1 + xhat.abs() * a2
    e_h = rstd * ((w + 3) * U * a1 + e_x * a2 + xhat.abs() * e_m2 + (e_v / 2 + 8 * U) * inner)
    out = H * dh.abs() + (e_h + 2 * U * dh.abs()) * (1 + 2 * H)
    n = max(rows, 1)
    return (dh, out), ((dy * xhat).sum(0), ((dy.abs() * e_x).sum(0) + (n + 2) * U * (dy * xhat).abs().sum(0))), \
        (dy.sum(0), (n + 2) * U * dy.abs().sum(0))


# ---- FC --------------------------------------------------------------------------

def fc(x, w, b, act, residual, dtype):
    """(y, bound), (a, bound)"""
    x, w = x.to(F64), w.to(F64)
    k = x.shape[1]
    a, size = x @ w.t(), x.abs() @ w.abs().t()
    if b is not None:
        a, size = a + b.to(F64), size + b.to(F64).abs()
    if act == "relu":
        a = a.clamp_min(0)
    H = half(dtype)
    e = (k + 8) * U * size                                 # fp32: six plane products leave up to 2^-24 of each
    y = a if residual is None else a + residual.to(F64)
    extra = 0 if residual is None else U * (a.abs() + residual.to(F64).abs())
    return (y, H * y.abs() + (e + extra) * (1 + H)), (a, H * a.abs() + e * (1 + H))


def fc_backward(dy, x, w, act, act_out, dx_add, dtype):
    """(dx, bound), (dw, bound), (db, bound)"""
    dp = dy.to(F64)
    if act == "relu":
        dp = torch.where(act_out.to(F64) > 0, dp, 0.0)
    x, w = x.to(F64), w.to(F64)
    rows, n = dp.shape
    dx, H = dp @ w, half(dtype)
    e = (n + 8) * U * (dp.abs() @ w.abs())
    if dx_add is not None:
        dx = dx + dx_add.to(F64)
        e = e + U * dx_add.to(F64).abs()
    return (dx, H * dx.abs() + e * (1 + H)), (dp.t() @ x, (rows + 8) * U * (dp.abs().t() @ x.abs())), \
        (dp.sum(0), (rows + 8) * U * dp.abs().sum(0))


# ---- attention ---------------------------------------------------------------------

class Attention:
    """gdp.RelAttention's definition for the same arguments."""

    def __init__(self, lengths, heads, d_head, bounds, kv_heads=None, seg_len=None, mem_len=0, causal=False,
                 queries=None, starts=None, scale=None):
        self.lengths, self.heads, self.d = list(lengths), heads, d_head
        self.kv = kv_heads or heads
        self.bounds = torch.tensor(list(bounds), dtype=torch.int64)
        self.seg, self.mem, self.causal = seg_len or max(1, max(lengths, default=1)), mem_len, causal
        self.queries = list(lengths) if queries is None else list(queries)
        if starts is None:
            starts, at = [], 0
            for n in self.lengths:
                starts.append(at)
                at += n
        self.starts = list(starts)
        self.scale = d_head ** -0.5 if scale is None else scale
        self.buckets = (len(self.bounds) + 1) * (1 if causal else 2)

    def bucket(self, rel):
        f = torch.zeros_like(rel)
        for b in self.bounds.tolist():
            f = f + (rel.abs() >= b)
        return f if self.causal else f + torch.where(rel > 0, len(self.bounds) + 1, 0)

    def run(self, q, k, v, table, key_mask=None, dout=None, dtype=torch.float32):
        """{name: (value, bound)} for o and lse, with dout also dq, dk, dv and dtable."""
        H, hd, share = half(dtype), self.d, self.heads // self.kv
        # a probability's or dS's rounding as the next product's operand (fp32: three planes, what they leave)
        R = H if dtype == torch.bfloat16 else 2 * U
        dev = torch.device("cuda" if torch.cuda.is_available() else "cpu")
        q, k, v, table = (t.to(dev, F64) for t in (q, k, v, table))
        dout = None if dout is None else dout.to(dev, F64)
        key_mask = None if key_mask is None else key_mask.to(dev)
        table = torch.where(table < -1e30, -math.inf, table)
        zero = lambda t: (torch.zeros_like(t), torch.zeros_like(t))
        o, dq, dk, dv, dt = zero(q), zero(q), zero(k), zero(v), zero(table)
        lse = zero(q.new_zeros(q.shape[0], self.heads))
        lse[0].fill_(-math.inf)
        first = 0
        for n, nq, start in zip(self.lengths, self.queries, self.starts):
            if nq == 0:
                first += nq
                continue
            p, j = torch.arange(n - nq, n, device=dev)[:, None], torch.arange(n, device=dev)[None, :]
            s0 = p // self.seg * self.seg
            seen = (j >= s0 - self.mem) & (j < s0 + self.seg)
            if self.causal:
                seen = seen & (j <= p)
            if key_mask is not None:
                seen = seen & (key_mask[start:start + n] != 0)[None, :]
            bucket = self.bucket(j - p)
            rows = slice(first, first + nq)
            keys = slice(start, start + n)
            for h in range(self.heads):
                c, ck = slice(h * hd, (h + 1) * hd), slice(h // share * hd, (h // share + 1) * hd)
                Q, K, V = q[rows, c], k[keys, ck], v[keys, ck]
                live = seen.any(0)
                K, V = torch.where(live[:, None], K, 0.0), torch.where(live[:, None], V, 0.0)   # never read
                bias = table[h][bucket.clamp_max(self.buckets - 1)]
                z = torch.where(seen, Q @ K.t() * self.scale + bias, -math.inf)
                top = z.amax(1, keepdim=True)
                e = torch.exp(z - torch.where(torch.isinf(top), 0.0, top))
                total = e.sum(1, keepdim=True)
                P = e / torch.where(total == 0, 1.0, total)
                # z: hd products, the scale, the bias, its change of base, the maximum's subtraction (at most 2^8 past it)
                size = torch.where(seen, abs(self.scale) * (Q.abs() @ K.abs().t()) + torch.where(torch.isinf(bias), 0.0, bias.abs()), 0.0)
                e_z = torch.where(seen & ~torch.isinf(z), U * ((hd + 8) * size + 6 * z.abs() + 6 * top.abs() + 12), 0.0)
                e_z = torch.where(torch.isnan(e_z) | torch.isinf(e_z), 0.0, e_z)
                keep = P * e_z
                # relative error of a probability: its own score's and the sum's (n terms)
                # and fp32 has no normal number below 2^-126: a smaller probability (and a smaller product
                # of one) is taken as 0, which is off by less than that
                e_P = P * (e_z + keep.sum(1, keepdim=True) + (n + 8) * U) + torch.where(seen, 2.0 ** -125, 0.0)
                O = P @ V
                o[0][rows, c] = O
                o[1][rows, c] = H * O.abs() + ((e_P + R * P) @ V.abs() + (n + 4) * U * (P @ V.abs())) * (1 + 2 * H)
                lse[0][rows, h] = torch.where(total == 0, -math.inf, top + torch.log(total))[:, 0] / math.log(2)
                lse[1][rows, h] = 2 * (keep.sum(1) + (n + 8) * U + 2 * U * torch.nan_to_num(lse[0][rows, h], neginf=0.0).abs())
                if dout is None:
                    continue
                G = dout[rows, c]
                dP = torch.where(seen, G @ V.t(), 0.0)
                D = (P * dP).sum(1, keepdim=True)
                S = P * (dP - D)
                aP = torch.where(seen, G.abs() @ V.abs().t(), 0.0)          # magnitudes of dP's products
                e_dP = (hd + 4) * U * aP
                aD = (P * aP).sum(1, keepdim=True)
                e_D = (n + 8) * U * aD + (e_P * dP.abs()).sum(1, keepdim=True) + (P * e_dP).sum(1, keepdim=True)
                # what the backward forms again from a stored lse: the same bounds once more
                e_S = 2 * e_P * (dP - D).abs() + P * (e_dP + e_D) + 4 * U * P * (aP + aD)
                # dq starts from the rounded o (off by R and H of it) and takes the rest in rounded operands
                rest = (R + H) * (P @ V.abs() * G.abs()).sum(1, keepdim=True) + e_D
                w = abs(self.scale)
                dq[0][rows, c] = S @ K * self.scale
                dq[1][rows, c] = H * dq[0][rows, c].abs() + w * ((R * (S.abs() + rest * P * 2) + e_S) @ K.abs() + (n + 4) * U * ((S.abs() + 2 * rest * P) @ K.abs())) * (1 + 2 * H)
                add_k, add_v = S.t() @ Q * self.scale, P.t() @ G
                dk[0][keys, ck] += add_k
                dv[0][keys, ck] += add_v
                dk[1][keys, ck] += w * ((R * S.abs() + e_S).t() @ Q.abs() + (nq * share + 4) * U * (S.abs().t() @ Q.abs())) * (1 + 2 * H)
                dv[1][keys, ck] += ((R * P + 2 * e_P).t() @ G.abs() + (nq * share + 4) * U * (P.t() @ G.abs())) * (1 + 2 * H)
                flat = bucket.clamp_max(self.buckets - 1).reshape(-1)
                dt[0][h].index_add_(0, flat, S.reshape(-1))
                dt[1][h].index_add_(0, flat, (e_S + (nq + 2 * n + 64) * U * S.abs()).reshape(-1))
            first += nq
        out = {"o": o, "lse": lse}
        if dout is not None:
            dk[1].add_(H * dk[0].abs())
            dv[1].add_(H * dv[0].abs())
            out.update(dq=dq, dk=dk, dv=dv, dtable=dt)
        return {n: (a.cpu(), b.cpu()) for n, (a, b) in out.items()}
