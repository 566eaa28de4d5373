"""The layer operators of paper_1910_01578_amd.gdp as measurable cases.

  norm             layer_norm: LayerNorm of a sum, as after a sublayer
  norm_backward    layer_norm_backward: its gradients, the weights' among them
  fc               fc: product with bias, activation and residual
  fc_backward      fc_backward: gradients of input, weights and bias
  attention        RelAttention.forward: segment attention with a learned bias
                   by buckets of the relative position; with few queries a
                   graph, the form for ops appended to a graph
  attention_train  the same with its backward: one training pass

With `own` false a case is computed from elementary torch operations in fp32,
rounded once; with `own` true by the library's calls.  exact() is a separate
statement in float64.
"""
import math

import torch

own = False

F32, F64 = torch.float32, torch.float64
EPS = 1e-5


# ----------------------------------------------------------------------------
# The cases.
# ----------------------------------------------------------------------------

def _norm(do, rows, width, dtype="bf16", residual=True):
    return {"do": do, "rows": rows, "width": width, "dtype": dtype, "residual": residual}


def _fc(do, rows, n_in, n_out, dtype="bf16", act="relu", residual=False):
    return {"do": do, "rows": rows, "in": n_in, "out": n_out, "dtype": dtype, "act": act, "residual": residual}


def _attn(do, nodes, graphs=1, new=0, heads=8, kv_heads=8, d_head=32, seg=512, mem=512, causal=False, buckets=16,
          reach=128, masked=False, dtype="bf16"):
    return {"do": do, "nodes": nodes, "graphs": graphs, "new": new, "heads": heads, "kv_heads": kv_heads,
            "d_head": d_head, "seg": seg, "mem": mem, "causal": causal, "buckets": buckets, "reach": reach,
            "masked": masked, "dtype": dtype}


def listed():
    return [
        # the smallest policy's LayerNorm after a sublayer: all launch latency
        {"name": "norm_256x64_f32", **_norm("norm", 256, 64, "f32")},
        # an odd width and odd row count, residual sum kept for the backward
        {"name": "norm_4099x1001", **_norm("norm", 4099, 1001)},
        # LayerNorm's backward at the headline graph's size
        {"name": "norm_backward_52000x256", **_norm("norm_backward", 52000, 256)},
        # one op appended to a placed graph: the first FC layer of its row alone
        {"name": "fc_1x256x1024", **_fc("fc", 1, 256, 1024)},
        # the feed-forward layer of the headline graph
        {"name": "fc_52000x256x1024", **_fc("fc", 52000, 256, 1024)},
        # a wide policy's projection added to its residual stream: bound by the matrix cores
        {"name": "fc_16384x2048x2048", **_fc("fc", 16384, 2048, 2048, act="none", residual=True)},
        # an odd fp32 layer: 2,503 ops, widths that no vector load fits
        {"name": "fc_2503x131x517_f32", **_fc("fc", 2503, 131, 517, "f32")},
        # the backward of the headline's feed-forward layer
        {"name": "fc_backward_52000x256x1024", **_fc("fc_backward", 52000, 256, 1024)},
        # the headline graph's attention with positions
        {"name": "attention_52000", **_attn("attention", 52000)},
        # eight growing graphs, one new op each, keys and values cached and shared by four heads
        {"name": "attention_new_op_8x12000", **_attn("attention", 96000, graphs=8, new=1, kv_heads=2, d_head=64,
                                                     seg=16384, mem=0, causal=True)},
        # a training pass over the four heterogeneous graphs
        {"name": "attention_train_29000", **_attn("attention_train", 29000, graphs=4, d_head=16, seg=256, mem=256)},
        # the smallest policy's training pass in fp32, some ops masked out
        {"name": "attention_train_256_f32", **_attn("attention_train", 256, heads=4, kv_heads=4, d_head=16, seg=64,
                                                    mem=64, causal=True, buckets=8, reach=48, masked=True,
                                                    dtype="f32")},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Spread over the logarithm; most are multiples of 8, some odd."""
    w = _log(rng, lo, hi)
    return max(lo, w - w % 8) if rng.random() < 0.7 else w


def draw(rng):
    do = rng.choice(["norm", "norm_backward", "fc", "fc", "fc_backward", "attention", "attention", "attention_train"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if do.startswith("norm"):
        width = _width(rng, 16, 4096)
        return _norm(do, _log(rng, 1, min(65536, 13312000 // width)), width, dtype, rng.random() < 0.6)
    if do.startswith("fc"):
        n_in, n_out = _width(rng, 16, 2048), _width(rng, 4, 2048)
        rows = _log(rng, 1, 65536) if do == "fc" else _log(rng, 64, 65536)
        # an fp32 product costs several times a bf16 one
        most = (1 << 36) // (8 if dtype == "f32" else 2 if do == "fc_backward" else 1)
        return _fc(do, max(1, min(rows, most // (n_in * n_out))), n_in, n_out, dtype, rng.choice(["none", "relu"]),
                   do == "fc" and rng.random() < 0.4)
    heads = rng.choice([2, 4, 8, 8])
    c = dict(heads=heads, kv_heads=rng.choice([heads, heads, heads // 2]), d_head=rng.choice([16, 32, 32, 64]),
             causal=rng.random() < 0.4, buckets=rng.choice([4, 8, 16, 16, 32]), reach=rng.choice([48, 128, 500]),
             masked=rng.random() < 0.25, dtype=dtype)
    if do == "attention" and rng.random() < 0.5:
        graphs, new = rng.choice([1, 1, 3, 8, 16]), rng.choice([1, 1, 1, 5])
        return _attn(do, max(_log(rng, 64, 16000) * graphs, new * graphs), graphs, new, seg=rng.choice([4096, 16384]),
                     mem=rng.choice([0, 4096]), **c)
    graphs = rng.choice([1, 1, 2, 4])
    seg = rng.choice([33, 64, 128, 200, 256, 512])
    nodes = max(_log(rng, 100, 20000 if do == "attention_train" or dtype == "f32" else 52000), 8 * graphs)
    return _attn(do, nodes, graphs, seg=seg, mem=rng.choice([0, seg // 2, seg, seg]), **c)


# ----------------------------------------------------------------------------
# Inputs.
# ----------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else F32


def _lengths(case):
    """The graphs' sizes: equal where ops are appended, else in proportion 1 : 2 : 3 ..."""
    n, g = case["nodes"], case["graphs"]
    if case["new"]:
        return [n // g] * g
    part = [n * (i + 1) // (g * (g + 1) // 2) for i in range(g)]
    part[-1] += n - sum(part)
    return part


def bounds(case):
    """Distances at which a bucket begins: every one up to half the buckets, then spread to `reach`."""
    n, reach = case["buckets"] - 1, case["reach"]
    near = min(n, case["buckets"] // 2)
    far = [near * (reach / near) ** ((i + 1) / (n - near)) for i in range(n - near)]
    out = list(range(1, near + 1))
    for f in far:
        out.append(max(out[-1] + 1, int(round(f))))
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = _dtype(case)

    def normal(*shape, scale=1.0, shift=0.0, dtype=dt):
        return (torch.randn(*shape, device="cuda", dtype=F32, generator=gen) * scale + shift).to(dtype)

    do = case["do"]
    s = {"case": case}
    if do.startswith("norm"):
        r, w = case["rows"], case["width"]
        s["gamma"], s["beta"] = normal(w, scale=0.1, shift=1.0), normal(w, scale=0.1)
        s["x"] = normal(r, w, shift=0.3)
        s["res"] = normal(r, w) if case["residual"] else None
        if do == "norm_backward":
            s["dy"] = normal(r, w)
        return s
    if do.startswith("fc"):
        r, k, n = case["rows"], case["in"], case["out"]
        s["x"] = normal(r, k)
        s["w"] = normal(n, k, scale=k ** -0.5)
        s["b"] = normal(n, scale=0.1)
        s["res"] = normal(r, n) if case["residual"] else None
        if do == "fc_backward":
            s["dy"] = normal(r, n)
            # what the forward left: the activation's output
            a = s["x"].float() @ s["w"].float().t() + s["b"].float()
            s["a"] = torch.relu(a).to(dt) if case["act"] == "relu" else None
        return s
    h, hk, d, new = case["heads"], case["kv_heads"], case["d_head"], case["new"]
    lengths = _lengths(case)
    total = sum(lengths)
    if new:                                        # queries of the new ops, keys and values from their caches
        s["q"] = normal(new * len(lengths), h * d)
        s["k"], s["v"] = normal(total, hk * d), normal(total, hk * d)
    else:                                          # one projection's columns
        qkv = normal(total, (h + 2 * hk) * d)
        s["q"], s["k"], s["v"] = qkv[:, :h * d], qkv[:, h * d:(h + hk) * d], qkv[:, (h + hk) * d:]
    s["bounds"] = bounds(case)
    n_buckets = case["buckets"] * (1 if case["causal"] else 2)
    s["table"] = normal(h, n_buckets, scale=0.5)
    s["mask"] = None
    if case["masked"]:
        s["mask"] = (torch.rand(total, device="cuda", generator=gen) < 0.8).to(torch.uint8)
    if do == "attention_train":
        s["do"] = normal(total, h * d)
    if own:
        from paper_1910_01578_amd import gdp
        s["plan"] = gdp.RelAttention(lengths, h, d, s["bounds"], kv_heads=hk, seg_len=case["seg"],
                                     mem_len=case["mem"], causal=case["causal"], queries=[new] * len(lengths) if new else None)
    else:
        s.update(_index(case, lengths))
    return s


def _index(case, lengths):
    """The plain form's plan: for every segment that holds queries, the rows of its queries and keys (-1: none) and
    the bucket of every pair."""
    longest = max(lengths)
    seg = min(case["seg"], longest)
    mem = min(case["mem"], longest) if case["seg"] < longest else 0
    new = case["new"]
    q_rows, k_rows, q_pos, k_pos = [], [], [], []
    start = first = 0
    for n in lengths:
        nq = new or n
        if new:                                    # the new ops as one row of queries, which may lie in two segments
            pos = torch.arange(n - nq, n)[None]
            kp = torch.arange(n)[None]
        else:
            s0 = torch.arange(0, n, seg)[:, None]
            pos = s0 + torch.arange(seg)[None]
            kp = s0 - mem + torch.arange(seg + mem)[None]
        q_rows.append(torch.where(pos < n, first + pos - (n - nq), -1))
        k_rows.append(torch.where((kp >= 0) & (kp < n), start + kp, -1))
        q_pos.append(pos)
        k_pos.append(kp)
        start, first = start + n, first + nq
    q_pos, k_pos = torch.cat(q_pos).cuda(), torch.cat(k_pos).cuda()
    rel = (k_pos[:, None, :] - q_pos[:, :, None])[:1 if not new else None]
    edge = torch.tensor(bounds(case), device="cuda")
    bucket = torch.bucketize(rel.abs(), edge, right=True) + (case["buckets"] * (rel > 0) if not case["causal"] else 0)
    if case["causal"]:
        bucket = torch.where(rel > 0, 0, bucket)   # never seen
    q_rows, k_rows = torch.cat(q_rows).cuda(), torch.cat(k_rows).cuda()
    return {"q_rows": q_rows, "k_rows": k_rows, "q_pos": q_pos, "k_pos": k_pos, "bucket": bucket}


# ----------------------------------------------------------------------------
# One pass.
# ----------------------------------------------------------------------------

def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_1910_01578_amd import gdp
    c = s["case"]
    do = c["do"]
    if do == "norm":
        if s["res"] is None:
            return gdp.layer_norm(s["x"], s["gamma"], s["beta"], eps=EPS)
        return gdp.layer_norm(s["x"], s["gamma"], s["beta"], residual=s["res"], eps=EPS, keep_sum=True)
    if do == "norm_backward":
        return gdp.layer_norm_backward(s["x"], s["gamma"], s["dy"], dsum=s["res"], eps=EPS)
    if do == "fc":
        return gdp.fc(s["x"], s["w"], s["b"], act=c["act"], residual=s["res"])
    if do == "fc_backward":
        return gdp.fc_backward(s["dy"], s["x"], s["w"], act=c["act"], act_out=s["a"])
    if do == "attention":
        return s["plan"].forward(s["q"], s["k"], s["v"], s["table"], key_mask=s["mask"])[0]
    o, lse = s["plan"].forward(s["q"], s["k"], s["v"], s["table"], key_mask=s["mask"])
    return (o, *s["plan"].backward(s["do"], s["q"], s["k"], s["v"], s["table"], o, lse, key_mask=s["mask"]))


def _plain(s):
    c = s["case"]
    do, dt = c["do"], _dtype(c)
    if do == "norm":
        h = s["x"].float() if s["res"] is None else s["x"].float() + s["res"].float()
        y = (_normal(h)[0] * s["gamma"].float() + s["beta"].float()).to(dt)
        return y if s["res"] is None else (y, h.to(dt))
    if do == "norm_backward":
        xhat, rstd = _normal(s["x"].float())
        dy = s["dy"].float()
        g = dy * s["gamma"].float()
        dh = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        if s["res"] is not None:
            dh = dh + s["res"].float()
        return dh.to(dt), (dy * xhat).sum(0), dy.sum(0)
    if do == "fc":
        y = s["x"].float() @ s["w"].float().t() + s["b"].float()
        if c["act"] == "relu":
            y = torch.clamp_min(y, 0)
        if s["res"] is not None:
            y = y + s["res"].float()
        return y.to(dt)
    if do == "fc_backward":
        dp = s["dy"].float()
        if c["act"] == "relu":
            dp = dp * (s["a"] > 0)
        return (dp @ s["w"].float()).to(dt), dp.t() @ s["x"].float(), dp.sum(0)
    return _plain_attention(s, c, dt)


def _normal(h):
    mean = h.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((h - mean) ** 2).mean(1, keepdim=True) + EPS)
    return (h - mean) * rstd, rstd


def _blocks(x, rows, heads, d):
    """Rows of x as [block, head, row, d] in fp32 (rows of -1: any)."""
    return x.float()[rows.clamp_min(0)].view(*rows.shape, heads, d).transpose(1, 2)


def _plain_attention(s, c, dt):
    h, hk, d, scale = c["heads"], c["kv_heads"], c["d_head"], c["d_head"] ** -0.5
    share = h // hk
    qr, kr = s["q_rows"], s["k_rows"]
    q = _blocks(s["q"], qr, h, d)
    k = _blocks(s["k"], kr, hk, d).repeat_interleave(share, 1)
    v = _blocks(s["v"], kr, hk, d).repeat_interleave(share, 1)
    s0 = s["q_pos"] // c["seg"] * c["seg"]
    kp, qp = s["k_pos"][:, None, :], s["q_pos"][:, :, None]
    seen = (kr[:, None, :] >= 0) & (kp >= s0[:, :, None] - c["mem"]) & (kp < s0[:, :, None] + c["seg"])
    if c["causal"]:
        seen = seen & (kp <= qp)
    if s["mask"] is not None:
        seen = seen & (s["mask"][kr.clamp_min(0)] != 0)[:, None, :]
    seen = seen[:, None]
    z = q @ k.transpose(2, 3) * scale + s["table"].float()[:, s["bucket"]].transpose(0, 1)
    z = torch.where(seen, z, -math.inf)
    top = z.amax(3, keepdim=True)
    e = torch.exp(z - torch.where(torch.isinf(top), 0.0, top))
    total = e.sum(3, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    live = qr >= 0
    o = (p @ v).transpose(1, 2)[live].reshape(-1, h * d)
    o = o.to(dt)                                   # blocks come in the order of the rows
    if c["do"] == "attention":
        return o
    do = _blocks(s["do"], qr, h, d) * live[:, None, :, None]
    dp = do @ v.transpose(2, 3)
    ds = p * (dp - (p * dp).sum(3, keepdim=True)) * live[:, None, :, None]
    dq = (ds @ k * scale).transpose(1, 2)[live].reshape(-1, h * d)
    dk = ds.transpose(2, 3) @ q * scale
    dv = p.transpose(2, 3) @ do
    pick = kr >= 0

    def to_rows(g):
        g = g.view(g.shape[0], hk, share, -1, d).sum(2).transpose(1, 2)
        return torch.zeros(s["k"].shape, device="cuda").index_add_(0, kr[pick], g[pick].reshape(-1, hk * d))

    # every segment has the same geometry: pairs of one distance lie at one place
    each = ds.sum(0).view(h, -1).double()
    one = torch.nn.functional.one_hot(s["bucket"].reshape(-1), s["table"].shape[1]).double()
    return o, dq.to(dt), to_rows(dk).to(dt), to_rows(dv).to(dt), (each @ one).float()


# ----------------------------------------------------------------------------
# What a pass cannot do without.
# ----------------------------------------------------------------------------

def _pairs(case):
    """(query, key) pairs of one head."""
    pairs = 0
    for n in _lengths(case):
        seg, mem, nq = case["seg"], case["mem"], case["new"] or n
        first = n - nq
        s0 = first // seg * seg
        while s0 < n:
            lo, hi = max(first, s0), min(s0 + seg, n)
            k0 = max(0, s0 - mem)
            pairs += (hi - lo) * (lo + hi + 1 - 2 * k0) // 2 if case["causal"] else (hi - lo) * (min(s0 + seg, n) - k0)
            s0 += seg
    return pairs


def work(case):
    do, e = case["do"], 2 if case["dtype"] == "bf16" else 4
    if do.startswith("norm"):
        n, w = case["rows"] * case["width"], case["width"]
        if do == "norm":
            return {"bytes": n * e * (4 if case["residual"] else 2) + 2 * w * e, "flops": 8 * n}
        return {"bytes": n * e * (4 if case["residual"] else 3) + w * e + 8 * w, "flops": 14 * n}
    if do.startswith("fc"):
        m, k, n = case["rows"], case["in"], case["out"]
        if do == "fc":
            return {"bytes": e * (m * k + n * k + n + m * n * (2 if case["residual"] else 1)), "flops": 2 * m * n * k}
        gate = 1 if case["act"] == "relu" else 0
        return {"bytes": e * (m * n * (1 + gate) + 2 * m * k + n * k) + 4 * (n * k + n), "flops": 4 * m * n * k}
    h, hk, d = case["heads"], case["kv_heads"], case["d_head"]
    nk = sum(_lengths(case))
    nq = case["new"] * case["graphs"] or nk
    tab = h * case["buckets"] * (1 if case["causal"] else 2)
    mask = nk if case["masked"] else 0
    pairs = _pairs(case)
    if do == "attention":
        return {"bytes": e * (2 * nq * h * d + 2 * nk * hk * d + tab) + mask, "flops": 4 * pairs * h * d}
    return {"bytes": e * (4 * nq * h * d + 4 * nk * hk * d + tab) + 4 * tab + mask, "flops": 14 * pairs * h * d}


# ----------------------------------------------------------------------------
# The definition in float64.
# ----------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    do = case["do"]
    wide = {k: t.to(F64) for k, t in s.items() if torch.is_tensor(t) and t.is_floating_point()}
    if do.startswith("norm"):
        x, gamma = wide["x"], wide["gamma"]
        if do == "norm":
            h = x + wide["res"] if "res" in wide else x
            var, mean = torch.var_mean(h, 1, correction=0, keepdim=True)
            y = (h - mean) * torch.rsqrt(var + EPS) * gamma + wide["beta"]
            return (y, h) if "res" in wide else y
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        r = torch.rsqrt(var + EPS)
        n, dy = (x - mean) * r, wide["dy"]
        g = dy * gamma
        # the projection of g off the directions 1 and n
        dh = r * (g - (g.sum(1, keepdim=True) + n * (g * n).sum(1, keepdim=True)) / x.shape[1])
        return dh + wide["res"] if "res" in wide else dh, torch.linalg.vecdot(dy, n, dim=0), dy.sum(0)
    if do == "fc":
        y = torch.nn.functional.linear(wide["x"], wide["w"], wide["b"])
        y = y.relu() if case["act"] == "relu" else y
        return y + wide["res"] if "res" in wide else y
    if do == "fc_backward":
        g = wide["dy"] if case["act"] == "none" else torch.where(s["a"] > 0, wide["dy"], 0.0)
        return torch.mm(g, wide["w"]), torch.mm(g.t(), wide["x"]), g.sum(0)
    return _exact_attention(case, s, wide)


def _exact_attention(case, s, w):
    """Head by head, segment by segment, over the keys that the segment admits."""
    h, d, share = case["heads"], case["d_head"], case["heads"] // case["kv_heads"]
    edges = torch.tensor(s["bounds"], device="cuda")
    train = case["do"] == "attention_train"
    o = torch.zeros(w["q"].shape, dtype=F64, device="cuda")
    grads = {x: torch.zeros(w[x].shape, dtype=F64, device="cuda") for x in ("q", "k", "v")}
    dtab = torch.zeros(w["table"].shape, dtype=F64, device="cuda")
    base = first = 0
    for n in _lengths(case):
        nq = case["new"] or n
        at = n - nq
        while at < n:
            s0 = at - at % case["seg"]
            end = min(s0 + case["seg"], n)
            lo = max(0, s0 - case["mem"])
            qp, kp = torch.arange(at, end, device="cuda"), torch.arange(lo, end, device="cuda")
            rel = kp[None] - qp[:, None]
            admit = torch.ones_like(rel, dtype=torch.bool) if not case["causal"] else rel <= 0
            if s["mask"] is not None:
                admit = admit & s["mask"][base + lo:base + end].bool()[None]
            bucket = torch.searchsorted(edges, rel.abs(), right=True)
            if not case["causal"]:
                bucket = bucket + torch.where(rel > 0, case["buckets"], 0)
            qs, ks = slice(first + at - (n - nq), first + end - (n - nq)), slice(base + lo, base + end)
            heads = lambda x, r, g: w[x][r].reshape(-1, h // g, d).permute(1, 0, 2).repeat_interleave(g, 0)  # noqa: E731
            q, k, v = heads("q", qs, 1), heads("k", ks, share), heads("v", ks, share)
            z = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(d) + w["table"][:, bucket.clamp_max(dtab.shape[1] - 1)]
            z = z.masked_fill(~admit[None], -math.inf)
            p = torch.softmax(z, 2).masked_fill(~admit.any(1)[None, :, None], 0.0)
            o[qs] = torch.matmul(p, v).permute(1, 0, 2).reshape(-1, h * d)
            if train:
                g = heads_of(w["do"][qs], h, d)
                dp = torch.matmul(g, v.transpose(1, 2).contiguous())
                ds = p * (dp - (p * dp).sum(2, keepdim=True))
                grads["q"][qs] += torch.matmul(ds, k).permute(1, 0, 2).reshape(-1, h * d) / math.sqrt(d)
                dk = torch.matmul(ds.transpose(1, 2).contiguous(), q).view(h // share, share, -1, d).sum(1) / math.sqrt(d)
                dv = torch.matmul(p.transpose(1, 2).contiguous(), g).view(h // share, share, -1, d).sum(1)
                grads["k"][ks] += dk.permute(1, 0, 2).reshape(-1, grads["k"].shape[1])
                grads["v"][ks] += dv.permute(1, 0, 2).reshape(-1, grads["v"].shape[1])
                # distances of one bucket form whole diagonals
                for b in range(dtab.shape[1]):
                    dtab[:, b] += (ds * (bucket == b)).sum((1, 2))
            at = end
        base, first = base + n, first + nq
    return (o, grads["q"], grads["k"], grads["v"], dtab) if train else o


def heads_of(x, h, d):
    return x.reshape(-1, h, d).permute(1, 0, 2)
