"""Timed cases of the operators of a transformer layer in a pipeline stage: norm, products by expert, attention.

Three operators, in training and, where they have one, in single-token form:

* ``norm``: the root-mean-square norm with the residual's addition, whose outputs are kept in 8 bits, and its gradient;
* ``product``: rows times the weights of their expert over ragged row ranges, and the gradient of the rows;
* ``attention``: causal attention with grouped heads over packed sequences of different lengths, and its gradient.

8-bit form of a row: groups of 64 neighbouring values share a power-of-two scale 2^e, the least with |x| <= 127 2^e in the
group (e within what the type holds); a value is kept as the whole number nearest to x / 2^e, ties to the even one.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
GROUP = 64
LOW = {"f32": -126, "bf16": -126, "f16": -24}    # least and largest exponent of a scale
HIGH = {"f32": 121, "bf16": 121, "f16": 9}
EPS = 1e-6


def _norm(name, n, d, way, dtype="bf16", residual=True, keep=False):
    """way: forward, or both forward and backward; keep: the normalised rows are kept in 8 bits too."""
    return _named(name, dict(op="norm", n=n, d=d, way=way, dtype=dtype, residual=residual, keep=keep))


def _product(name, n, k, experts, o, i, way, dtype="bf16", out="same", dropped=0.0):
    """n tokens by k experts each; way: forward is [rows, i] to [rows, o], backward the reverse with the same weights."""
    return _named(name, dict(op="product", n=n, k=k, experts=experts, o=o, i=i, way=way, dtype=dtype, out=out, dropped=dropped))


def _attention(name, n, seqs, heads, kv_heads, dim, way, dtype="bf16", joint=True):
    """joint: q, k and v are parts of one product's rows."""
    return _named(name, dict(op="attention", n=n, seqs=seqs, heads=heads, kv_heads=kv_heads, dim=dim, way=way, dtype=dtype, joint=joint))


def _named(name, c):
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token through a layer's norm: the serving form, the call's latency
        _norm("norm_n1_d4096", 1, 4096, "forward"),
        # a wide layer's norm over a long micro-batch, forward and backward, its sum kept in 8 bits between the two
        _norm("norm_n32768_d8192", 32768, 8192, "both"),
        # an odd number of tokens and an odd width, in half precision, both outputs kept
        _norm("norm_n777_d1365_f16", 777, 1365, "both", "f16", keep=True),
        # one token through 8 of 64 experts: the serving form, the weights' bytes
        _product("product_n1_k8_e64", 1, 8, 64, 4096, 2048, "forward"),
        # a long micro-batch through 8 of 64 experts: the gate and up projection
        _product("product_n8192_k8_e64", 8192, 8, 64, 4096, 2048, "forward"),
        # the rows' gradient of 2 of 16 experts with some choices dropped over capacity, odd sizes, half precision
        _product("product_grad_n4001_k2_e16_f16", 4001, 2, 16, 1365, 1001, "backward", "f16", dropped=0.05),
        # a large layer's projection, the gradient of its rows: one range
        _product("product_grad_n16384_8192x4096", 16384, 1, 1, 8192, 4096, "backward"),
        # a few short prompts: the call's latency
        _attention("attention_n256_s3", 256, 3, 16, 4, 128, "forward"),
        # a long prompt
        _attention("attention_n16384_s1", 16384, 1, 16, 4, 128, "forward"),
        # a training sequence, forward and backward
        _attention("attention_grad_n8192_s1", 8192, 1, 32, 8, 128, "both"),
        # a micro-batch packed from sequences of very different lengths, forward and backward
        _attention("attention_grad_n16384_s24", 16384, 24, 16, 8, 128, "both"),
        # an odd number of tokens, small heads, half precision, separate tensors
        _attention("attention_grad_n1001_s5_f16", 1001, 5, 6, 2, 64, "both", "f16", joint=False),
    ]


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _width(rng, lo, hi):
    """A width, aligned as most models' are, or any."""
    w = _spread(rng, lo, hi)
    return w if rng.random() < 0.3 else max(64, w // 64 * 64)


def draw(rng):
    op = rng.choice(["norm", "norm", "product", "product", "attention", "attention"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    way = rng.choice(["forward", "both"])
    if op == "norm":
        dtype = rng.choice([dtype, "f32"])
        d = _width(rng, 64, 16384)
        return _norm(None, _spread(rng, 1, max(1, (1 << 27) // d)), d, way, dtype, rng.random() < 0.7, dtype != "f32" and rng.random() < 0.5)
    if op == "product":
        experts = rng.choice([1, _spread(rng, 2, 64)])
        k = rng.randint(1, min(8, experts))
        o, i = _width(rng, 64, 8192), _width(rng, 64, 8192)
        if experts > 1:
            o, i = min(o, 4096), min(i, 4096)
        n = _spread(rng, 1, max(1, min(65536, (1 << 38) // (o * i)) // k))
        return _product(None, n, k, experts, o, i, "backward" if way == "both" else way, dtype, rng.choice(["same", "same", "f32"]),
                        rng.choice([0.0, 0.0, 0.05]) if experts > 1 else 0.0)
    kv_heads, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * group
    dim = rng.choice([64, 128, 128, 8 * rng.randint(4, 16)])
    n = _spread(rng, 1, min(16384, int(math.sqrt((1 << 31) / heads))))
    return _attention(None, n, rng.choice([1, _spread(rng, 1, 64)]), heads, kv_heads, dim, way, dtype, rng.random() < 0.5)


# ---- inputs ----

def _activations(g, n, d, dtype, spread=1.0):
    """Normal values with a few channels an order of magnitude above the others, as hidden states have."""
    x = torch.randn(n, d, generator=g, device="cuda")
    gain = torch.exp(0.4 * torch.randn(d, generator=g, device="cuda"))
    gain[torch.rand(d, generator=g, device="cuda") < 0.004] *= 20
    return (x.mul_(gain).mul_(spread)).to(TYPES[dtype])


def _gradients(g, n, d, dtype):
    return (torch.randn(n, d, generator=g, device="cuda") * 0.05).to(TYPES[dtype])


def _lengths(n, seqs):
    """Lengths of packed sequences: most are short, a few long, as documents are; some are empty."""
    if seqs == 1:
        return [n]
    r = random.Random(n * 1000 + seqs)
    share = [math.exp(1.2 * r.gauss(0, 1)) for _ in range(seqs)]
    cut = [0]
    for s in share:
        cut.append(cut[-1] + s)
    cut = [int(c / cut[-1] * n) for c in cut[:-1]] + [n]
    return [b - a for a, b in zip(cut, cut[1:])]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c, s = case, dict(case)
    t = TYPES[c["dtype"]]
    if c["op"] == "norm":
        n, d = c["n"], c["d"]
        s["x"] = _activations(g, n, d, c["dtype"])
        s["residual"] = _activations(g, n, d, c["dtype"], 2.0) if c["residual"] else None
        s["weight"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(t)
        if c["way"] == "both":
            s["dout"] = _gradients(g, n, d, c["dtype"])
            s["dsum"] = _gradients(g, n, d, c["dtype"]) if c["residual"] else None
    elif c["op"] == "product":
        n, k, e = c["n"], c["k"], c["experts"]
        rows = n * k
        s["x"] = _activations(g, rows, c["i"], c["dtype"]) if c["way"] == "forward" else _gradients(g, rows, c["o"], c["dtype"])
        s["weights"] = (torch.randn(e, c["o"], c["i"], generator=g, device="cuda") * c["i"] ** -0.5).to(t)
        # ragged ranges as a router leaves them: a few experts are busy, some get almost nothing
        logits = torch.randn(n, e, generator=g, device="cuda") + torch.randn(e, generator=g, device="cuda")
        choice = torch.topk(logits, k, dim=1)[1].reshape(-1)
        choice = choice[torch.rand(rows, generator=g, device="cuda") >= c["dropped"]]
        ends = torch.cumsum(torch.bincount(choice, minlength=e), 0)
        s["offsets"] = torch.cat([ends.new_zeros(1), ends]).to(torch.int32)
        s["longest"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())
    else:
        n, h, kv, d = c["n"], c["heads"], c["kv_heads"], c["dim"]
        both = torch.randn(n, (h + 2 * kv) * d, generator=g, device="cuda")
        both[:, :(h + kv) * d] *= 1.5        # scores spread over a few units, so that attention is neither flat nor one token
        both = both.to(t)
        parts = both.split([h * d, kv * d, kv * d], dim=1)
        s["q"], s["k"], s["v"] = ((p if c["joint"] else p.contiguous()).view(n, -1, d) for p in parts)
        ends = torch.tensor(_lengths(n, c["seqs"])).cumsum(0)
        s["offsets"] = torch.cat([ends.new_zeros(1), ends]).to(torch.int32).cuda()
        if c["way"] == "both":
            s["dout"] = _gradients(g, n, h * d, c["dtype"]).view(n, h, d)
    return s


# ---- the plain forms ----

def _power(e):
    """2^e as a 32-bit float, for whole e in [-126, 127]."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _kept(x, dtype):
    """Rows as their 8-bit form gives them back, in 32 bits."""
    n, d = x.shape
    g = -(-d // GROUP)
    v = torch.zeros(n, g * GROUP, dtype=torch.float32, device=x.device)
    v[:, :d] = x
    v = v.view(n, g, GROUP)
    a = v.abs().amax(2, keepdim=True)
    part, e = torch.frexp(a)                       # a = part 2^e, part in [0.5, 1)
    e = torch.clamp(e - 7 + (part > 127 / 128), LOW[dtype], HIGH[dtype])
    q = torch.clamp(torch.round(v * _power(-e)), -127, 127)
    v = torch.where(torch.isfinite(a), q * _power(e), torch.full_like(q, math.nan))
    return v.view(n, -1)[:, :d]


def _plain_norm(s):
    t = TYPES[s["dtype"]]
    h, w = s["x"].float(), s["weight"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    rstd = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    out = (h * rstd * w).to(t)
    r = {"out": out, "rstd": rstd.view(-1)}
    h = h.to(t)
    if s["residual"] is not None:
        r["sum"] = h
    if s["keep"]:
        r["kept"] = _kept(out, s["dtype"]).to(t)
    if s["way"] == "both":
        n = _kept(h, s["dtype"]) * rstd
        dout = s["dout"].float()
        g = dout * w
        dx = rstd * (g - n * (n * g).mean(1, keepdim=True))
        if s["dsum"] is not None:
            dx = dx + s["dsum"].float()
        r |= {"dx": dx.to(t), "dweight": (dout * n).sum(0)}
    return r


def _plain_product(s):
    x, w = s["x"].float(), s["weights"].float()
    out = torch.float32 if s["out"] == "f32" else TYPES[s["dtype"]]
    at = s["offsets"][:-1].long().unsqueeze(1) + torch.arange(max(1, s["longest"]), device=x.device)
    inside = at < s["offsets"][1:].unsqueeze(1)
    at = at.clamp(max=x.shape[0] - 1)
    y = torch.bmm(x[at], w.transpose(1, 2).contiguous() if s["way"] == "forward" else w)
    result = torch.zeros(x.shape[0], y.shape[2], dtype=out, device=x.device)
    result[at[inside]] = y[inside].to(out)         # rows of no range stay zero
    return result


def _plain_attention(s):
    n, h, kv, d, t = s["n"], s["heads"], s["kv_heads"], s["dim"], TYPES[s["dtype"]]
    group, scale = h // kv, d ** -0.5
    at = torch.arange(n, device=s["q"].device)
    of = torch.searchsorted(s["offsets"][1:].long(), at, right=True)     # the token's sequence
    seen = (of.unsqueeze(1) == of.unsqueeze(0)) & (at.unsqueeze(1) >= at.unsqueeze(0))
    # [kv heads, group * tokens, dim]: a key's head with all the queries that share it
    q = s["q"].float().view(n, kv, group, d).permute(1, 2, 0, 3).reshape(kv, group * n, d)
    k, v = (s[x].float().transpose(0, 1).contiguous() for x in "kv")
    scores = torch.bmm(q, k.transpose(1, 2).contiguous()).view(h, n, n).mul_(scale).masked_fill_(~seen, -math.inf)
    most = scores.amax(2, keepdim=True)
    p = scores.sub_(most).exp_()
    total = p.sum(2, keepdim=True)
    p = p.div_(total).view(kv, group * n, n)

    def rows(x):
        return x.view(kv, group, n, d).permute(2, 0, 1, 3).reshape(n, h, d)

    out = torch.bmm(p, v)
    r = {"out": rows(out).to(t), "lse": (most + torch.log(total)).view(h, n)}
    if s["way"] == "both":
        dout = s["dout"].float().view(n, kv, group, d).permute(1, 2, 0, 3).reshape(kv, group * n, d)
        r["dv"] = torch.bmm(p.transpose(1, 2), dout).transpose(0, 1).contiguous().to(t)
        ds = torch.bmm(dout, v.transpose(1, 2).contiguous()).sub_((dout * out).sum(2, keepdim=True)).mul_(p).mul_(scale)
        r["dq"] = rows(torch.bmm(ds, k)).to(t)
        r["dk"] = torch.bmm(ds.transpose(1, 2), q).transpose(0, 1).contiguous().to(t)
    return r


def _plain(s):
    return {"norm": _plain_norm, "product": _plain_product, "attention": _plain_attention}[s["op"]](s)


# ---- the framework's operators ----

def _own(s):
    from paper_2609_06086_amd import layers as L

    if s["op"] == "norm":
        both = s["way"] == "both"
        y = L.poseidon_norm_forward(s["x"], s["weight"], s["residual"], eps=EPS, keep_out=s["keep"], keep_sum=both)
        r = {"out": y.out, "rstd": y.rstd}
        if s["residual"] is not None:
            r["sum"] = y.sum
        if s["keep"]:
            r["kept"] = L.poseidon_restore(y.kept_out)
        if both:
            r["dx"], r["dweight"] = L.poseidon_norm_backward(s["dout"], y.kept_sum, y.rstd, s["weight"], s["dsum"])
        return r
    if s["op"] == "product":
        return L.poseidon_expert_product(s["x"], s["weights"], s["offsets"], transposed=s["way"] == "backward",
                                         dtype=torch.float32 if s["out"] == "f32" else None)
    out, lse = L.poseidon_attention_forward(s["q"], s["k"], s["v"], s["offsets"])
    r = {"out": out, "lse": lse}
    if s["way"] == "both":
        r["dq"], r["dk"], r["dv"] = L.poseidon_attention_backward(s["dout"], s["q"], s["k"], s["v"], out, lse, s["offsets"])
    return r


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    c = case
    z = SIZE[c["dtype"]]
    if c["op"] == "norm":
        n, d, kept = c["n"], c["d"], 1 + 1 / GROUP
        more = 2 * z if c["residual"] else 0                         # the residual read, the sum written
        size = n * d * (2 * z + more + (2 * kept + z if c["keep"] else 0))   # what is kept written, read and restored
        if c["way"] == "both":                                       # kept between, dout and dsum read, dx written
            size += n * d * (2 * kept + 2 * z + more / 2)
        return {"bytes": size + d * z, "flops": n * d * (16 if c["way"] == "both" else 5)}
    if c["op"] == "product":
        m = c["n"] * c["k"]
        out = 4 if c["out"] == "f32" else z
        wide, into = (c["i"], c["o"]) if c["way"] == "forward" else (c["o"], c["i"])
        return {"bytes": m * (wide * z + into * out) + min(m, c["experts"]) * c["o"] * c["i"] * z, "flops": 2 * m * c["o"] * c["i"]}
    n, h, kv, d = c["n"], c["heads"], c["kv_heads"], c["dim"]
    pairs = h * sum(x * (x + 1) // 2 for x in _lengths(n, c["seqs"]))
    size = n * d * z * (2 * h + 2 * kv) + 4 * n * h
    if c["way"] == "both":
        size += n * d * z * (4 * h + 4 * kv) + 4 * n * h - n * d * z * h     # out is at hand, dout read, three gradients written
    return {"bytes": size, "flops": pairs * d * (14 if c["way"] == "both" else 4)}


# ---- the definitions in 64 bits ----

def _power64(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _kept64(x, dtype):
    pieces = []
    for lo in range(0, x.shape[1], GROUP):
        v = x[:, lo:lo + GROUP].double()
        a = v.abs().max(1, keepdim=True).values
        e = torch.floor(torch.log2(a.clamp(min=2.0 ** -300) / 127))
        for _ in range(2):           # the logarithm may be one off: step up to the least e with a <= 127 2^e
            e = torch.where(a > 127 * _power64(e), e + 1, e)
        e = torch.where(a <= 127 * _power64(e - 1), e - 1, e)
        unit = _power64(e.clamp(LOW[dtype], HIGH[dtype]))
        back = torch.round(v / unit).clamp(-127, 127) * unit
        pieces.append(torch.where(torch.isfinite(a), back, torch.full_like(back, math.nan)))
    return torch.cat(pieces, 1)


def exact(case, seed):
    s = prepare(case, seed)
    t = TYPES[s["dtype"]]
    if s["op"] == "norm":
        h, w = s["x"].double(), s["weight"].double()
        if s["residual"] is not None:
            h += s["residual"].double()
        size = torch.sqrt(h.square().sum(1) / s["d"] + EPS)
        r = {"out": h / size.unsqueeze(1) * w, "rstd": 1 / size}
        if s["residual"] is not None:
            r["sum"] = h
        if s["keep"]:
            r["kept"] = _kept64(r["out"].to(t), s["dtype"])          # the 8-bit form of the output in its type
        if s["way"] == "both":
            n = _kept64(h.to(t), s["dtype"]) / size.unsqueeze(1)
            dout = s["dout"].double()
            r["dweight"] = torch.sum(n * dout, dim=0)
            along = torch.sum(n * dout * w, dim=1, keepdim=True) / s["d"]
            r["dx"] = (dout * w - along * n) / size.unsqueeze(1)
            if s["dsum"] is not None:
                r["dx"] += s["dsum"].double()
        return r
    if s["op"] == "product":
        cuts, x = s["offsets"].tolist(), s["x"]
        y = torch.zeros(x.shape[0], s["o"] if s["way"] == "forward" else s["i"], dtype=torch.float64, device=x.device)
        for e, (a, b) in enumerate(zip(cuts, cuts[1:])):
            if b > a:
                w = s["weights"][e].double()
                y[a:b] = torch.matmul(x[a:b].double(), w.t().contiguous() if s["way"] == "forward" else w)
        return y
    cuts, h, group, scale = s["offsets"].tolist(), s["heads"], s["heads"] // s["kv_heads"], 1 / math.sqrt(s["dim"])
    both = s["way"] == "both"
    r = {"out": torch.zeros_like(s["q"], dtype=torch.float64), "lse": torch.full((h, s["n"]), -math.inf, dtype=torch.float64, device="cuda")}
    if both:
        r |= {"d" + x: torch.zeros(s[x].shape, dtype=torch.float64, device="cuda") for x in "qkv"}
    for a, b in zip(cuts, cuts[1:]):
        if b == a:
            continue
        later = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1)
        for j in range(h):
            q, k, v = s["q"][a:b, j].double(), s["k"][a:b, j // group].double(), s["v"][a:b, j // group].double()
            score = (torch.matmul(q, k.t().contiguous()) * scale).masked_fill_(later, -math.inf)
            lse = torch.logsumexp(score, 1)
            p = torch.exp(score - lse.unsqueeze(1))
            out = torch.matmul(p, v)
            r["out"][a:b, j], r["lse"][j, a:b] = out, lse
            if both:
                dout = s["dout"][a:b, j].double()
                r["dv"][a:b, j // group] += torch.matmul(p.t().contiguous(), dout)
                ds = p * (torch.matmul(dout, v.t().contiguous()) - torch.sum(out * dout, 1, keepdim=True)) * scale
                r["dq"][a:b, j] = torch.matmul(ds, k)
                r["dk"][a:b, j // group] += torch.matmul(ds.t().contiguous(), q)
    return r
