"""Timed cases of the layer operators: what a pipeline stage computes and keeps between its forward and its backward.

Five operators, in training and, where they have one, in single-token form:

* ``stash``: rows of activations kept in 8 bits for the backward pass, and restored;
* ``gated``: the gated activation silu(gate) * up, which keeps its inputs in 8 bits, with its gradient from what it kept;
* ``wgrad``: a weight gradient from the 8-bit rows, of one matrix or of one matrix per expert over ragged row ranges;
* ``experts``: tokens sorted by expert, gathered, combined with their weights, and the gradient of both;
* ``embed``: embedding lookup with a scale, and its gradient summed by token.

8-bit form of a row: groups of 64 neighbouring values share a power-of-two scale 2^e, the least with |x| <= 127 2^e in the
group (e within what the type holds); a value is kept as the whole number nearest to x / 2^e, ties to the even one.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
GROUP = 64
LOW = {"f32": -126, "bf16": -126, "f16": -24}    # least and largest exponent of a scale: restored values stay
HIGH = {"f32": 121, "bf16": 121, "f16": 9}       # finite, and exact in the type they came from


def _stash(name, n, d, dtype="bf16", **more):
    return _named(name, dict(op="stash", n=n, d=d, dtype=dtype, **more))


def _gated(name, n, f, dtype="bf16", joint=True):
    """joint: gate and up are the two halves of one product's rows."""
    return _named(name, dict(op="gated", n=n, f=f, dtype=dtype, joint=joint))


def _wgrad(name, m, o, i, experts=0, dtype="bf16", out="f32"):
    return _named(name, dict(op="wgrad", m=m, o=o, i=i, experts=experts, dtype=dtype, out=out))


def _experts(name, n, k, experts, d, way, dtype="bf16", dropped=0.0, keep=False):
    return _named(name, dict(op="experts", n=n, k=k, experts=experts, d=d, way=way, dtype=dtype, dropped=dropped, keep=keep))


def _embed(name, n, vocab, d, dtype="bf16", out="f32"):
    return _named(name, dict(op="embed", n=n, vocab=vocab, d=d, dtype=dtype, out=out))


def _named(name, c):
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest micro-batch of a profile run: the call's latency
        _stash("stash_n256_d1024", 256, 1024),
        # what a wide layer keeps of a long micro-batch
        _stash("stash_n32768_d8192", 32768, 8192),
        # an odd number of tokens and an odd width, in half precision: nothing is aligned
        _gated("gated_n777_f1365_f16", 777, 1365, "f16", joint=False),
        # the feed-forward part of a wide layer, gate and up from one product
        _gated("gated_n16384_f12288", 16384, 12288),
        # a small projection: few output tiles, so the token axis has to be split
        _wgrad("wgrad_m4096_1024x1024", 4096, 1024, 1024),
        # a large layer's projection
        _wgrad("wgrad_m16384_8192x4096", 16384, 8192, 4096, out="bf16"),
        # the experts' projections: 64 ragged row ranges, some of them short
        _wgrad("wgrad_m65536_e64_2048x2048", 65536, 2048, 2048, experts=64),
        # one token through 8 of 64 experts: the serving form
        _experts("experts_n1_k8_e64", 1, 8, 64, 4096, "forward"),
        # a long micro-batch through 8 of 64 experts, whose inputs are kept in 8 bits too
        _experts("experts_n16384_k8_e64", 16384, 8, 64, 4096, "forward", keep=True),
        # the gradient of 2 of 8 experts with some choices dropped over capacity, an odd number of tokens
        _experts("experts_grad_n16001_k2_e8", 16001, 2, 8, 4096, "backward", dropped=0.05),
        # a small vocabulary and an odd number of tokens
        _embed("embed_n1001_v8000_d1024", 1001, 8000, 1024, "f32"),
        # a long micro-batch over a large vocabulary
        _embed("embed_n32768_v131072_d2048", 32768, 131072, 2048),
    ]


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _width(rng, lo, hi):
    """A width, aligned as most models' are, or any."""
    w = _spread(rng, lo, hi)
    return w if rng.random() < 0.3 else max(64, w // 64 * 64)


def draw(rng):
    op = rng.choice(["stash", "gated", "wgrad", "wgrad", "experts", "experts", "embed"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "stash":
        d = _width(rng, 64, 16384)
        return _stash(None, _spread(rng, 1, max(1, (1 << 28) // d)), d, dtype)
    if op == "gated":
        f = _width(rng, 64, 16384)
        return _gated(None, _spread(rng, 1, max(1, (1 << 27) // f)), f, dtype, joint=rng.random() < 0.5)
    if op == "wgrad":
        experts = rng.choice([0, 0, rng.randint(2, 64)])
        o, i = _width(rng, 64, 8192), _width(rng, 64, 8192)
        if experts:
            o, i = min(o, 2048), min(i, 2048)
        m = _spread(rng, 1, min(65536, (1 << 39) // (o * i)))
        return _wgrad(None, m, o, i, experts, rng.choice(["bf16", "bf16", "f16"]), rng.choice(["f32", "bf16"]))
    if op == "experts":
        experts = _spread(rng, 2, 256)
        k = rng.randint(1, min(8, experts))
        d = _width(rng, 64, 8192)
        n = _spread(rng, 1, min(32768, (1 << 28) // (k * d)))
        way = rng.choice(["forward", "backward"])
        return _experts(None, n, k, experts, d, way, dtype, rng.choice([0.0, 0.05, 0.5]), way == "forward" and rng.random() < 0.5)
    d = _width(rng, 64, 8192)
    vocab = _spread(rng, 100, min(131072, (1 << 27) // d))
    return _embed(None, _spread(rng, 1, min(65536, (1 << 26) // d)), vocab, d, dtype, rng.choice(["f32", "bf16"]))


# ---- inputs ----

def _activations(g, n, d, dtype, spread=1.0):
    """Normal values with a few channels an order of magnitude above the others, as hidden states have."""
    x = torch.randn(n, d, generator=g, device="cuda")
    gain = torch.exp(0.4 * torch.randn(d, generator=g, device="cuda"))
    gain[torch.rand(d, generator=g, device="cuda") < 0.004] *= 20
    return (x.mul_(gain).mul_(spread)).to(TYPES[dtype])


def _gradients(g, n, d, dtype):
    return (torch.randn(n, d, generator=g, device="cuda") * 0.05).to(TYPES[dtype])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c, s = case, dict(case)
    op = c["op"]
    if op == "stash":
        s["x"] = _activations(g, c["n"], c["d"], c["dtype"])
    elif op == "gated":
        n, f = c["n"], c["f"]
        if c["joint"]:
            both = _activations(g, n, 2 * f, c["dtype"])
            s["gate"], s["up"] = both[:, :f], both[:, f:]
        else:
            s["gate"], s["up"] = _activations(g, n, f, c["dtype"]), _activations(g, n, f, c["dtype"])
        s["dout"] = _gradients(g, n, f, c["dtype"])
    elif op == "wgrad":
        m = c["m"]
        s["dy"] = _gradients(g, m, c["o"], c["dtype"])
        s["codes"], s["scales"] = _codes(_activations(g, m, c["i"], c["dtype"]), c["dtype"])
        if c["experts"]:
            # ragged ranges as a router leaves them: a few experts are busy, some get almost nothing
            share = torch.exp(torch.randn(c["experts"], generator=g, device="cuda"))
            cut = torch.floor(torch.cumsum(share, 0) / share.sum() * m).to(torch.int32)
            cut[-1] = m
            s["offsets"] = torch.cat([cut.new_zeros(1), torch.cummax(cut, 0).values])
            s["longest"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())
    elif op == "experts":
        n, k, e = c["n"], c["k"], c["experts"]
        logits = torch.randn(n, e, generator=g, device="cuda") + torch.randn(e, generator=g, device="cuda")
        top, choice = torch.topk(logits, k, dim=1)
        gone = torch.rand(n, k, generator=g, device="cuda") < c["dropped"]
        s["choice"] = torch.where(gone, torch.full_like(choice, -1), choice).to(torch.int32)
        s["weights"] = torch.softmax(top, 1)
        if c["way"] == "forward":
            s["x"] = _activations(g, n, c["d"], c["dtype"])
            s["ys"] = _activations(g, n * k, c["d"], c["dtype"], 0.5)   # what the experts' products gave
        else:
            s["order"], s["position"], s["offsets"] = _sorted(s["choice"], e)   # the forward's plan
            s["dout"] = _gradients(g, n, c["d"], c["dtype"])
            s["ys"] = _activations(g, n * k, c["d"], c["dtype"], 0.5)
            s["dxs"] = _gradients(g, n * k, c["d"], c["dtype"])         # what the experts' backward gave
    else:
        n, v = c["n"], c["vocab"]
        s["table"] = (torch.randn(v, c["d"], generator=g, device="cuda") * 0.02).to(TYPES[c["dtype"]])
        # tokens by rank: the most frequent make up much of a text; a hundredth of the places is padding
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
        ids = torch.clamp(torch.exp(u * math.log(v + 1.0)) - 1, 0, v - 1).to(torch.int32)
        ids[torch.rand(n, generator=g, device="cuda") < 0.01] = -1
        s["ids"] = ids
        s["scale"] = math.sqrt(c["d"])
        s["dout"] = _gradients(g, n, c["d"], c["dtype"])
    return s


# ---- the plain forms ----

def _power(e):
    """2^e as a 32-bit float, for whole e in [-126, 127]."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _groups(x):
    """Rows in groups of 64, in 32 bits, the last group filled up with zeros."""
    n, d = x.shape
    g = -(-d // GROUP)
    v = torch.zeros(n, g * GROUP, dtype=torch.float32, device=x.device)
    v[:, :d] = x
    return v.view(n, g, GROUP)


def _quantised(x, dtype):
    """(whole numbers as floats [n, g, 64], exponents [n, g, 1], whether each group is finite)."""
    v = _groups(x)
    a = v.abs().amax(2, keepdim=True)
    part, e = torch.frexp(a)                       # a = part 2^e, part in [0.5, 1)
    e = torch.clamp(e - 7 + (part > 127 / 128), LOW[dtype], HIGH[dtype])
    return torch.clamp(torch.round(v * _power(-e)), -127, 127), e, torch.isfinite(a)


def _codes(x, dtype):
    q, e, fine = _quantised(x, dtype)
    n, g, _ = q.shape
    scales = torch.where(fine, e + 127, torch.full_like(e, 255)).view(n, g).to(torch.uint8)
    return torch.where(fine, q, torch.zeros_like(q)).view(n, g * GROUP).to(torch.int8), scales


def _kept(x, dtype):
    """Rows as their 8-bit form gives them back, in 32 bits."""
    q, e, fine = _quantised(x, dtype)
    v = torch.where(fine, q * _power(e), torch.full_like(q, math.nan))
    return v.view(x.shape[0], -1)[:, :x.shape[1]]


def _sorted(choice, experts):
    """Stable order of the flat choices by expert, each choice's place in it (-1: dropped) and the experts' offsets."""
    key = choice.reshape(-1)
    key = torch.where((key < 0) | (key >= experts), torch.full_like(key, experts), key)
    by, order = torch.sort(key, stable=True)
    position = torch.empty_like(order)
    position[order] = torch.arange(order.numel(), device=order.device)
    position = torch.where(key == experts, torch.full_like(position, -1), position).view(choice.shape)
    offsets = torch.searchsorted(by, torch.arange(experts + 1, device=by.device, dtype=by.dtype))
    return order.to(torch.int32), position.to(torch.int32), offsets.to(torch.int32)


def _combined(rows, position, weights):
    """sum_j weights[t, j] rows[position[t, j]] over the choices that were not dropped, in 32 bits."""
    picked = rows[position.clamp(min=0).long()].float()
    picked = torch.where((position >= 0).unsqueeze(2), picked, torch.zeros_like(picked))
    if weights is not None:
        picked = picked * weights.unsqueeze(2)
    return picked.sum(1)


def _plain(s):
    op, t = s["op"], TYPES[s["dtype"]]
    if op == "stash":
        return _kept(s["x"], s["dtype"]).to(t)
    if op == "gated":
        gate, up = s["gate"].float(), s["up"].float()
        out = gate / (1 + torch.exp(-gate)) * up
        gate, up, dout = _kept(s["gate"], s["dtype"]), _kept(s["up"], s["dtype"]), s["dout"].float()
        sig = 1 / (1 + torch.exp(-gate))
        return {"out": out.to(t), "dgate": (dout * up * sig * (1 + gate * (1 - sig))).to(t), "dup": (dout * gate * sig).to(t)}
    if op == "wgrad":
        q = s["codes"].float().view(s["m"], -1, GROUP)
        x = (q * _power(s["scales"].int() - 127).unsqueeze(2)).view(s["m"], -1)[:, :s["i"]]
        dy = s["dy"].float()
        if not s["experts"]:
            return (dy.t() @ x).to(TYPES[s["out"]])
        at = s["offsets"][:-1].long().unsqueeze(1) + torch.arange(s["longest"], device=dy.device)
        inside = (at < s["offsets"][1:].unsqueeze(1)).unsqueeze(2)
        at = at.clamp(max=s["m"] - 1)
        rows = torch.where(inside, dy[at], dy.new_zeros(()))
        return torch.bmm(rows.transpose(1, 2).contiguous(), x[at]).to(TYPES[s["out"]])
    if op == "experts":
        n, k, d = s["n"], s["k"], s["d"]
        if s["way"] == "forward":
            order, position, offsets = _sorted(s["choice"], s["experts"])
            there = (torch.arange(n * k, device=order.device) < offsets[-1]).unsqueeze(1)
            xs = torch.where(there, s["x"][order.long() // k], s["x"].new_zeros(()))
            r = {"order": order, "position": position, "offsets": offsets, "xs": xs,
                 "out": _combined(s["ys"], position, s["weights"]).to(t)}
            if s["keep"]:
                r["kept"] = _kept(xs, s["dtype"]).to(t)
            return r
        position, weights, dout = s["position"], s["weights"], s["dout"].float()
        there = position >= 0
        picked = s["ys"][position.clamp(min=0).long()].float()
        dw = torch.where(there, (picked * dout.unsqueeze(1)).sum(2), weights.new_zeros(()))
        flat = s["order"].long()
        dys = weights.reshape(-1)[flat].unsqueeze(1) * dout[flat // k]
        dys = torch.where((torch.arange(n * k, device=flat.device) < s["offsets"][-1]).unsqueeze(1), dys, dys.new_zeros(()))
        return {"dys": dys.to(t), "dweights": dw, "dx": _combined(s["dxs"], position, None).to(t)}
    ids = s["ids"].long()
    there = ((ids >= 0) & (ids < s["vocab"])).unsqueeze(1)
    ids = ids.clamp(0, s["vocab"] - 1)
    out = torch.where(there, s["table"][ids].float() * s["scale"], torch.zeros((), device=ids.device))
    dout = torch.where(there, s["dout"].float() * s["scale"], torch.zeros((), device=ids.device))
    dtable = torch.zeros(s["vocab"], s["d"], dtype=torch.float32, device=ids.device).index_add_(0, ids, dout)
    return {"out": out.to(t), "dtable": dtable.to(TYPES[s["out"]])}


# ---- the framework's operators ----

def _own(s):
    from paper_2609_06086_amd import layers as L

    op = s["op"]
    if op == "stash":
        return L.poseidon_restore(L.poseidon_stash(s["x"]))
    if op == "gated":
        out, gate, up = L.poseidon_gated_forward(s["gate"], s["up"])
        dgate, dup = L.poseidon_gated_backward(s["dout"], gate, up)
        return {"out": out, "dgate": dgate, "dup": dup}
    if op == "wgrad":
        stash = L.Stash(s["codes"], s["scales"], s["i"], TYPES[s["dtype"]])
        return L.poseidon_weight_gradient(s["dy"], stash, offsets=s.get("offsets"), dtype=TYPES[s["out"]])
    if op == "experts":
        if s["way"] == "forward":
            plan = L.poseidon_expert_sort(s["choice"], s["experts"])
            xs, kept = L.poseidon_expert_gather(s["x"], plan, keep=s["keep"])
            out = L.poseidon_expert_combine(s["ys"], plan, s["weights"])
            r = {"order": plan.order, "position": plan.position, "offsets": plan.offsets, "xs": xs, "out": out}
            if s["keep"]:
                r["kept"] = L.poseidon_restore(kept)
            return r
        plan = L.ExpertPlan(s["order"], s["position"], s["offsets"])
        dys, dweights = L.poseidon_expert_combine_backward(s["dout"], s["ys"], plan, s["weights"])
        return {"dys": dys, "dweights": dweights, "dx": L.poseidon_expert_combine(s["dxs"], plan)}
    out = L.poseidon_embed(s["ids"], s["table"], s["scale"])
    dtable = L.poseidon_embed_backward(s["ids"], s["dout"], s["vocab"], s["scale"], dtype=TYPES[s["out"]])
    return {"out": out, "dtable": dtable}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    c = case
    op, z = c["op"], SIZE[c["dtype"]]
    kept = 1 + 1 / GROUP
    if op == "stash":      # read, keep, read what was kept, write
        return {"bytes": c["n"] * c["d"] * (2 * z + 2 * kept), "flops": 4 * c["n"] * c["d"]}
    if op == "gated":      # forward: two read, one written, two kept; backward: two kept and one read, two written
        return {"bytes": c["n"] * c["f"] * (6 * z + 4 * kept), "flops": 24 * c["n"] * c["f"]}
    if op == "wgrad":
        e = max(1, c["experts"])
        return {"bytes": c["m"] * (c["o"] * z + c["i"] * kept) + e * c["o"] * c["i"] * SIZE[c["out"]],
                "flops": 2 * c["m"] * c["o"] * c["i"]}
    if op == "experts":
        n, m, d = c["n"], c["n"] * c["k"], c["d"]
        if c["way"] == "forward":    # x read, xs written; ys read, out written; what is kept written, read and restored
            more = m * d * (2 * kept + z) if c["keep"] else 0
            return {"bytes": (2 * n + 2 * m) * d * z + more + 16 * m, "flops": 2 * m * d}
        return {"bytes": (n + 2 * m) * d * z + (m + n) * d * z + 16 * m, "flops": 5 * m * d}
    n, v, d = c["n"], c["vocab"], c["d"]
    rows = min(n, v)
    return {"bytes": (rows + 2 * n) * d * z + v * d * SIZE[c["out"]] + 8 * n, "flops": 3 * n * d}


# ---- the definitions in 64 bits ----

def _kept64(x, dtype):
    n, d = x.shape
    pieces = []
    for lo in range(0, d, GROUP):
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


def _power64(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "stash":
        return _kept64(s["x"], s["dtype"])
    if op == "gated":
        gate = s["gate"].double()
        out = gate * torch.sigmoid(gate) * s["up"].double()
        gate, up, dout = _kept64(s["gate"], s["dtype"]), _kept64(s["up"], s["dtype"]), s["dout"].double()
        sig = torch.sigmoid(gate)
        slope = sig + gate * sig * torch.sigmoid(-gate)
        return {"out": out, "dgate": dout * up * slope, "dup": dout * gate * sig}
    if op == "wgrad":
        unit = _power64(s["scales"].long() - 127)
        x = s["codes"].double() * unit.repeat_interleave(GROUP, dim=1)
        x, dy = x[:, :s["i"]], s["dy"].double()
        if not s["experts"]:
            return torch.matmul(dy.t().contiguous(), x.contiguous())
        cuts = s["offsets"].tolist()
        return torch.stack([torch.matmul(dy[a:b].t().contiguous(), x[a:b].contiguous()) for a, b in zip(cuts, cuts[1:])])
    if op == "experts":
        n, k, d = s["n"], s["k"], s["d"]
        position = s["position"] if s["way"] == "backward" else _sorted(s["choice"], s["experts"])[1]
        place = position.reshape(-1).long()
        there = place >= 0
        token = torch.arange(n, device=place.device).repeat_interleave(k)

        def gathered(rows):          # rows by place from rows by choice
            v = torch.zeros(n * k, d, dtype=torch.float64, device=place.device)
            v[place[there]] = rows[there]
            return v

        def summed(rows, by):
            v = torch.zeros(n, d, dtype=torch.float64, device=place.device)
            for j in range(k):
                p = position[:, j].long()
                keep = (p >= 0).double() * (by[:, j].double() if by is not None else 1.0)
                v += rows[p.clamp(min=0)].double() * keep.unsqueeze(1)
            return v

        if s["way"] == "forward":
            xs = gathered(s["x"].double()[token])
            r = {"order": None, "position": None, "offsets": None, "xs": xs, "out": summed(s["ys"], s["weights"])}
            if s["keep"]:
                r["kept"] = _kept64(xs, s["dtype"])
            return r
        dout = s["dout"].double()
        dys = gathered(dout[token] * s["weights"].double().reshape(-1, 1))
        dw = torch.stack([(s["ys"][position[:, j].clamp(min=0).long()].double() * dout).sum(1) * (position[:, j] >= 0)
                          for j in range(k)], 1)
        return {"dys": dys, "dweights": dw, "dx": summed(s["dxs"], None)}
    ids = s["ids"].long()
    fine = (ids >= 0) & (ids < s["vocab"])
    out = torch.zeros(s["n"], s["d"], dtype=torch.float64, device=ids.device)
    out[fine] = s["table"][ids[fine]].double() * s["scale"]
    dtable = torch.zeros(s["vocab"], s["d"], dtype=torch.float64, device=ids.device)
    dtable.index_add_(0, ids[fine], s["dout"][fine].double() * s["scale"])
    return {"out": out, "dtable": dtable}
