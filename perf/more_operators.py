"""The operators of a training step on a routed batch, and the calls they are timed on.

After the rows of a batch are grouped by the model they went to, a program that
serves or trains those models runs their layers, scores tokens and moves the
weights:

* linear: y[r] = act(x[r] W[g(r)] + bias[g(r)]) + residual[r], a product with the
  weights of the row's group and what follows it, and the gradients of x, W and bias;
* probs: from rows of logits the log probability of a given token, the entropy of
  the distribution and the most likely tokens, and the gradient of the logits;
* adamw: one step of AdamW over many tensors, with states in 32 bits, or in 8
  (e4m3 with a scale for every 256 values, the root of the second moment in place of
  it) rounded by dither, so that small changes add up.

A row in no group gets the residual alone (zeros without one).  Weights are
[in][out], row-major.  Widths and batch sizes are those of the routing workloads and of
the operators beside these; vocabularies are generic.
"""
import math
from functools import lru_cache

import torch

own = False

#: how rows spread over the groups: the share of group i is proportional to (i + 1) ** -SKEW
SKEW = {"even": 0.0, "mild": 0.5, "steep": 1.0}

#: values that share a scale in 8-bit states, and where the tensors of a step begin in their flat buffers
BLOCK = 256


def _probs(name, op, dtype, n, m, top=0, scale=1.0, entropy=True, banned=0.0):
    return {"name": name, "op": op, "dtype": dtype, "n": n, "m": m, "top": top, "scale": scale, "entropy": entropy,
            "banned": banned}


def _linear(name, op, dtype, n, groups, k, out, act="none", residual=False, keep=False, skew="mild", none=0.0):
    return {"name": name, "op": op, "dtype": dtype, "n": n, "groups": groups, "k": k, "out": out, "act": act,
            "residual": residual, "keep": keep, "skew": skew, "none": none}


def _adamw(name, dtype, tensors, k, out, rank, bits=32, master=False, whole=False):
    return {"name": name, "op": "adamw", "dtype": dtype, "tensors": tensors, "k": k, "out": out, "rank": rank, "bits": bits,
            "master": master, "whole": whole}


def listed():
    return [
        # one request generating one token: its log probability and five alternatives
        _probs("probs_token", "probs", "bf16", 1, 32000, top=5),
        # the requests in flight, a large vocabulary, a temperature, some tokens not allowed
        _probs("probs_tokens", "probs", "bf16", 48, 128000, top=20, scale=1.25, banned=0.01),
        # scoring the tokens of a training batch
        _probs("probs_batch", "probs", "bf16", 8192, 32000),
        # the gradient of that batch's loss
        _probs("probs_grad", "probs_grad", "bf16", 8192, 32000, entropy=False),
        # with a bonus on the entropy, in fp32, rows that no vector divides
        _probs("probs_grad_f32", "probs_grad", "f32", 1003, 10007, scale=0.8, banned=0.02),
        # token generation: a few rows a model
        _linear("linear_tokens", "linear", "bf16", 40, 16, 1024, 2048, act="silu"),
        # prompts of a batch, what the gradient needs kept, some rows rejected
        _linear("linear_prompts", "linear", "bf16", 12288, 8, 2048, 4096, act="gelu", residual=True, keep=True, none=0.05),
        # a training step's gradients
        _linear("linear_grad", "linear_grad", "bf16", 12000, 8, 2048, 2048, act="gelu"),
        # the same in fp32, widths that no tile divides
        _linear("linear_grad_f32", "linear_grad", "f32", 1003, 5, 771, 390, act="silu", skew="steep"),
        # the adapters of 16 models, small tensors of odd sizes
        _adamw("adamw_adapters", "f32", 48, 1003, 771, 16),
        # whole weights, their fp32 masters and states
        _adamw("adamw_weights", "bf16", 16, 4096, 4096, 16, master=True, whole=True),
        # the same in little memory: bf16 weights alone, states in 8 bits
        _adamw("adamw_weights_8", "bf16", 16, 4096, 4096, 16, bits=8, whole=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["probs", "probs", "probs_grad", "linear", "linear", "linear_grad", "adamw", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op.startswith("probs"):
        m = _log(rng, 96, 160000)
        if rng.random() < 0.5:                                     # half of them whole vectors
            m = (m + 63) // 64 * 64
        c = _probs("", op, dtype, _log(rng, 1, 16384), m, top=rng.choice([0, rng.randint(1, 20)]) if op == "probs" else 0,
                   scale=rng.choice([1.0, round(rng.uniform(0.5, 2.0), 3)]), entropy=rng.random() < 0.7,
                   banned=rng.choice([0.0, rng.uniform(0.001, 0.1)]))
        size = "n"
    elif op.startswith("linear"):
        wide = 4096 if dtype == "bf16" else 1536
        k, out = (_log(rng, 256, wide) for _ in range(2))
        if rng.random() < 0.5:
            k, out = (k + 63) // 64 * 64, (out + 63) // 64 * 64
        n = _log(rng, 1, 64) if op == "linear" and rng.random() < 0.4 else _log(rng, 64, 16384 if dtype == "bf16" else 4096)
        c = _linear("", op, dtype, n, _log(rng, 1, 32), k, out, act=rng.choice(["none", "relu", "silu", "gelu"]),
                    residual=op == "linear" and rng.random() < 0.5, keep=op == "linear" and rng.random() < 0.5,
                    skew=rng.choice(sorted(SKEW)), none=rng.choice([0.0, 0.0, rng.uniform(0.01, 0.3)]))
        size = "n"
    else:
        c = _adamw("", dtype, _log(rng, 1, 160), _log(rng, 16, 4096), _log(rng, 16, 4096), rng.choice([4, 8, 16, 32, 64]),
                   bits=rng.choice([32, 8]), master=dtype == "bf16" and rng.random() < 0.5, whole=rng.random() < 0.4)
        size = "tensors"
    del c["name"]
    cap = max(_cost(x) for x in listed())
    while _cost(c) > cap:
        c[size] = max(1, int(c[size] * 0.7))
    return c


# ---------------------------------------------------------------- inputs
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _sizes(c):
    """Elements of the step's tensors: adapters A and B, a bias, and where weights are trained whole a matrix."""
    kinds = [c["k"] * c["rank"], c["rank"] * c["out"], c["out"]] + ([c["k"] * c["out"]] if c["whole"] else [])
    return [kinds[i % len(kinds)] for i in range(c["tensors"])]


def _shares(c):
    p = [(i + 1.0) ** -SKEW[c["skew"]] for i in range(c["groups"])]
    return [x / sum(p) for x in p]


def _prepare_probs(c, g, t):
    n, m = c["n"], c["m"]
    x = torch.randn((n, m), generator=g, device="cuda").mul_(2.5)
    token = torch.randint(0, m, (n,), generator=g, device="cuda")
    rows = torch.arange(n, device="cuda")
    x[rows, token] += 8 * torch.rand(n, generator=g, device="cuda")  # the text goes on as the model expects, more or less
    if c["banned"]:
        away = torch.rand((n, m), generator=g, device="cuda") < c["banned"]
        away[rows, token] = False
        x.masked_fill_(away, -math.inf)
    s = {"x": x.to(t), "token": token.to(torch.int32), "scale": c["scale"], "top": c["top"], "entropy": c["entropy"]}
    f32 = {"dtype": torch.float32, "device": "cuda"}
    if c["op"] == "probs":
        s["out"] = {"logp": torch.empty(n, **f32), "lse": torch.empty(n, **f32)}
        if c["entropy"]:
            s["out"]["entropy"] = torch.empty(n, **f32)
        if c["top"]:
            s["out"].update(top_logp=torch.empty((n, c["top"]), **f32),
                            top_token=torch.empty((n, c["top"]), dtype=torch.int32, device="cuda"))
        return s
    # what the forward pass left, and the gradients of its results; some places have no token to learn
    s["token"][torch.rand(n, generator=g, device="cuda") < 0.05] = -100
    z = s["x"].float() * c["scale"]
    s["lse"] = torch.logsumexp(z, 1)
    s["dlogp"] = torch.randn(n, generator=g, device="cuda") / n
    if c["entropy"]:
        p = torch.exp(z - s["lse"][:, None])
        s["ent"] = s["lse"] - torch.where(p > 0, p * z, 0.0).sum(1)
        s["dent"] = torch.full((n,), -0.01 / n, device="cuda")
    s["out"] = {"dlogits": torch.empty_like(s["x"])}
    return s


def _prepare_linear(c, g, t):
    n, G, k, out = c["n"], c["groups"], c["k"], c["out"]
    share = torch.tensor(_shares(c), device="cuda")
    gid = torch.randperm(G, generator=g, device="cuda")[torch.multinomial(share, n, replacement=True, generator=g)]
    gid = torch.where(torch.rand(n, generator=g, device="cuda") < c["none"], G, gid)
    keys, order = torch.sort(gid, stable=True)
    offsets = torch.searchsorted(keys, torch.arange(G + 1, device="cuda"))

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(t)

    s = {"act": c["act"], "n": n, "offsets": offsets.to(torch.int32), "order": order.to(torch.int32),
         "cap": int((offsets[1:] - offsets[:-1]).max()),              # the plain form's: rows of the largest group
         "x": normal(n, k), "w": normal(G, k, out, std=k ** -0.5)}
    s["x"][:, ::97] *= 8                                           # a few channels are much larger than the others
    if c["op"] == "linear":
        s["bias"] = normal(G, out, std=0.5)
        s["residual"] = normal(n, out) if c["residual"] else None
        s["out"] = {"y": torch.empty(n, out, dtype=t, device="cuda")}
        if c["keep"]:
            s["out"]["z"] = torch.empty(n, out, dtype=t, device="cuda")
        return s
    s["dy"], s["z"] = normal(n, out, std=1e-2), normal(n, out, std=1.5)
    s["out"] = {"dx": torch.empty_like(s["x"]), "dw": torch.empty_like(s["w"]),
                "dbias": torch.empty(G, out, dtype=t, device="cuda")}
    return s


def _prepare_adamw(c, g, t):
    sizes = _sizes(c)
    blocks = [(n + BLOCK - 1) // BLOCK for n in sizes]
    starts = [BLOCK * sum(blocks[:i]) for i in range(len(blocks))]
    total = BLOCK * sum(blocks)
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for a, n in zip(starts, sizes):
        inside[a:a + n] = True

    def normal(std):
        return torch.randn(total, generator=g, device="cuda") * std * inside

    def views(flat, per=1):
        return [flat[a // per:a // per + (n + per - 1) // per] for a, n in zip(starts, sizes)]

    master = normal(c["k"] ** -0.5)
    # tensors learn at different paces
    pace = torch.exp(2 * torch.randn(sum(blocks), generator=g, device="cuda")).repeat_interleave(BLOCK) * 1e-4
    flat = {"p": master.to(t), "g": (normal(1.0) * pace).to(t)}
    m = 0.3 * normal(1.0) * pace
    root = (0.2 + torch.rand(total, generator=g, device="cuda")) * pace * inside
    if c["bits"] == 8:
        for name, v in (("m", m), ("v", root)):
            scale = v.view(-1, BLOCK).abs().amax(1) / 448.0
            flat[name + "_scale"] = scale
            flat[name] = (v.view(-1, BLOCK) / scale[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(-1)
    else:
        flat.update(m=m, v=root * root)
    if c["master"]:
        flat["master"] = flat["p"].float() + normal(1e-5)
    out = {k: v for k, v in flat.items() if k != "g"}
    lists = {k: views(v, BLOCK if k.endswith("scale") else 1) for k, v in flat.items()}
    return {"flat": flat, "lists": lists, "out": out, "bits": c["bits"], "steps": 100, "lr": 2e-5, "betas": (0.9, 0.999),
            "eps": 1e-8, "weight_decay": 0.1, "seed": 1234567}


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(1000003 * seed + 17)
    make = {"p": _prepare_probs, "l": _prepare_linear, "a": _prepare_adamw}[case["op"][0]]
    return {"op": case["op"], **make(case, g, _TYPES[case["dtype"]])}


# ---------------------------------------------------------------- the plain forms
def _plain_probs(s):
    z = s["x"].float() * s["scale"]
    most = z.amax(1, keepdim=True)
    d = z - most
    e = torch.exp(d)
    total = e.sum(1)
    lse = most[:, 0] + torch.log(total)
    token = s["token"].long()
    out = {"logp": z.gather(1, token[:, None])[:, 0] - lse, "lse": lse}
    if s["entropy"]:
        out["entropy"] = torch.log(total) - torch.where(e > 0, e * d, 0.0).sum(1) / total
    if s["top"]:
        # the larger logit first, of equal ones the lower token
        at = torch.sort(s["x"].float(), dim=1, descending=True, stable=True)[1][:, :s["top"]]
        out.update(top_logp=z.gather(1, at) - lse[:, None], top_token=at.to(torch.int32))
    return out


def _plain_probs_grad(s):
    x, token = s["x"], s["token"].long()
    v = x.float() * s["scale"] - s["lse"][:, None]                     # log probabilities
    p = torch.exp(v)
    held = token >= 0
    dlogp = torch.where(held, s["dlogp"], 0.0)
    d = -dlogp[:, None] * p
    rows = torch.arange(len(token), device=x.device)
    d[rows, token.clamp(min=0)] += dlogp
    if "dent" in s:
        d -= s["dent"][:, None] * torch.where(p > 0, p * (v + s["ent"][:, None]), 0.0)
    return {"dlogits": (d * s["scale"]).to(x.dtype)}


def _padded(s):
    """[G][rows of the largest group]: the rows of every group, and which of the places hold one."""
    off = s["offsets"].long()
    at = off[:-1, None] + torch.arange(s["cap"], device=off.device)
    held = at < off[1:, None]
    return s["order"].long()[at.clamp(max=s["n"] - 1)], held


def _take(x, rows, held):
    return torch.where(held[..., None], x.float()[rows], 0.0)


def _put(v, rows, held, n):
    """The groups' results by row; a row in no group has zeros."""
    y = torch.zeros((n + 1, v.shape[-1]), device=v.device)
    y[torch.where(held, rows, n)] = v
    return y[:n]


def _act(name, z):
    if name == "relu":
        return z * (z > 0)
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z


def _slope(name, z):
    if name == "relu":
        return (z > 0).float()
    if name == "silu":
        h = 1 / (1 + torch.exp(-z))
        return h * (1 + z * (1 - h))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    return torch.ones_like(z)


def _plain_linear(s):
    t = s["x"].dtype
    rows, held = _padded(s)
    z = torch.bmm(_take(s["x"], rows, held), s["w"].float()) + s["bias"].float()[:, None]
    y = _put(_act(s["act"], z), rows, held, s["n"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(t)}
    if "z" in s["out"]:
        out["z"] = _put(z, rows, held, s["n"]).to(t)
    return out


def _plain_linear_grad(s):
    t = s["x"].dtype
    rows, held = _padded(s)
    dz = _take(s["dy"], rows, held) * _slope(s["act"], _take(s["z"], rows, held))
    dx = torch.bmm(dz, s["w"].float().transpose(1, 2).contiguous())
    dw = torch.bmm(_take(s["x"], rows, held).transpose(1, 2).contiguous(), dz)
    return {"dx": _put(dx, rows, held, s["n"]).to(t), "dw": dw.to(t), "dbias": dz.sum(1).to(t)}


_U32 = 0xFFFFFFFF


def _noise(s, count, device):
    """A random number of 32 bits for every value of the step, and another one: whole functions of the seed, the
    step and the value's place."""
    key = ((s["seed"] * 0x9E3779B97F4A7C15 + s["steps"]) * 0xBB67AE8584CAA73B >> 32) & _U32
    h = (torch.arange(count, device=device) + key & _U32) * 0x9E3779B9 & _U32
    h = (h ^ h >> 15) * 0xBB67AE85 & _U32
    h = h ^ h >> 16
    more = h * 0x510E527F & _U32
    return h, more ^ more >> 16


def _dithered_e4m3(x, noise):
    """x >= 0, at most 448, to e4m3: up or down, up with the probability of how near it is."""
    small = x < 2.0 ** -6
    bits = torch.where(small, x + 2.0 ** -6, x).view(torch.int32).long() + (noise << 4) >> 20
    return (bits - 960 - 8 * small).clamp(max=126)


def _dithered_bf16(x, noise):
    bits = x.view(torch.int32)
    up = bits + noise.int()
    up = torch.where(up & 0x7F800000 == 0x7F800000, bits, up) & -65536
    return up.view(torch.float32).bfloat16()


def _plain_adamw(s):
    f, (b1, b2) = s["flat"], s["betas"]
    s["steps"] += 1
    lr, step = s["lr"], s["steps"]
    rate, root_rate = lr / (1 - b1 ** step), (1 - b2 ** step) ** -0.5
    g = f["g"].float()
    if s["bits"] == 8:
        m = (f["m"].float().view(-1, BLOCK) * f["m_scale"][:, None]).view(-1)
        root = (f["v"].float().view(-1, BLOCK) * f["v_scale"][:, None]).view(-1)
        v = root * root
    else:
        m, v = f["m"], f["v"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    root = torch.sqrt(v)
    p = f["master"] if "master" in f else f["p"].float()
    p = p * (1 - lr * s["weight_decay"]) - m / (root * root_rate + s["eps"]) * rate
    low, high = (None, None) if s["bits"] == 32 and ("master" in f or f["p"].dtype == torch.float32) else _noise(s, len(g), g.device)
    if s["bits"] == 8:
        for name, x, noise in (("m", m, low & 0xFFFF), ("v", root, low >> 16)):
            most = x.view(-1, BLOCK).abs().amax(1)
            f[name + "_scale"].copy_(most / 448.0)
            y = (x.view(-1, BLOCK).abs() * torch.where(most > 0, 448.0 / most, 0.0)[:, None]).view(-1).clamp(max=448)
            code = _dithered_e4m3(y, noise)
            code = torch.where(x < 0, code + 128, code) if name == "m" else torch.where(y > 0, code.clamp(min=1), code)
            f[name].view(torch.uint8).copy_(code)
    else:
        f["m"].copy_(m)
        f["v"].copy_(v)
    if "master" in f:
        f["master"].copy_(p)
        f["p"].copy_(p)
    else:
        f["p"].copy_(p if f["p"].dtype == torch.float32 else _dithered_bf16(p, high >> 16))
    return s["out"]


# ---------------------------------------------------------------- the framework's operators
@lru_cache(maxsize=None)
def _ops(stream):
    from paper_2608_14575_amd import routed
    return routed.RoutedOps(stream=stream)


def _own_adamw(ops, s):
    if "opt" not in s:                                             # a program keeps it with the weights
        from paper_2608_14575_amd import routed
        f = s["lists"]
        s["opt"] = routed.AdamW(ops, f["p"], f["g"], state={k: v for k, v in f.items() if k not in "pg"}, steps=s["steps"],
                                lr=s["lr"], betas=s["betas"], eps=s["eps"], weight_decay=s["weight_decay"], seed=s["seed"])
    s["opt"].step()


def run(state):
    s, op = state, state["op"]
    if not own:
        return {"probs": _plain_probs, "probs_grad": _plain_probs_grad, "linear": _plain_linear,
                "linear_grad": _plain_linear_grad, "adamw": _plain_adamw}[op](s)
    ops, out = _ops(torch.cuda.current_stream().cuda_stream), s["out"]
    if op == "probs":
        ops.log_probs(s["x"], s["token"], scale=s["scale"], **out)
    elif op == "probs_grad":
        ops.log_probs_grad(s["x"], s["token"], s["lse"], s["dlogp"], entropy=s.get("ent"), dentropy=s.get("dent"),
                           scale=s["scale"], **out)
    elif op == "linear":
        ops.linear(s["x"], s["w"], s["offsets"], s["order"], bias=s["bias"], act=s["act"], residual=s["residual"], **out)
    elif op == "linear_grad":
        ops.linear_grad(s["dy"], s["x"], s["w"], s["offsets"], s["order"], act=s["act"], z=s["z"], **out)
    else:
        _own_adamw(ops, s)
    return out


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    size = 2 if c["dtype"] == "bf16" else 4
    if c["op"].startswith("probs"):
        n, m = c["n"], c["m"]
        if c["op"] == "probs":
            return {"bytes": n * m * size + 4 * n * (3 + c["entropy"]) + 8 * n * c["top"], "flops": 4 * n * m}
        return {"bytes": 2 * n * m * size + 4 * n * (3 + 2 * c["entropy"]), "flops": 4 * n * m}
    if c["op"] == "adamw":
        each = 3 * size + (8 if c["master"] else 0) + (16 if c["bits"] == 32 else 4 + 16 / BLOCK)
        return {"bytes": each * sum(_sizes(c)), "flops": 16 * sum(_sizes(c))}
    n, G, k, out = c["n"], c["groups"], c["k"], c["out"]
    held = n * (1 - c["none"])
    used = sum(1 - (1 - p * (1 - c["none"])) ** n for p in _shares(c))   # groups that have a row
    index = 4 * n + 4 * (G + 1)
    if c["op"] == "linear":
        rows = n * out * (1 + c["residual"] + c["keep"])
        return {"bytes": size * (held * k + used * (k + 1) * out + rows) + index, "flops": 2 * held * k * out}
    kept = c["act"] != "none"
    return {"bytes": size * (held * ((1 + kept) * out + k) + used * k * out + n * k + G * (k + 1) * out) + index,
            "flops": 4 * held * k * out}


def _cost(c):
    """Seconds at rates that a large pass and a large product reach."""
    w = work(c)
    return w["bytes"] / 4e12 + (w["flops"] / (1e15 if c["dtype"] == "bf16" else 1e14) if c["op"].startswith("linear") else 0)


# ---------------------------------------------------------------- the same in 64 bits
def _exact_probs(c, s):
    z = s["x"].double() * c["scale"]
    lse = torch.logsumexp(z, 1)
    logp = z - lse[:, None]
    token = s["token"].long()
    if c["op"] == "probs":
        out = {"logp": logp.gather(1, token[:, None])[:, 0], "lse": lse}
        p = logp.exp()
        if c["entropy"]:
            out["entropy"] = -torch.nansum(p * logp, 1)                # (a token that is not allowed: 0 * inf)
        if c["top"]:
            out.update(top_logp=torch.sort(logp, 1, descending=True)[0][:, :c["top"]], top_token=None)
        return out
    p = (z - s["lse"].double()[:, None]).exp()
    held = (token >= 0).double()[:, None]
    d = -p * s["dlogp"].double()[:, None] * held
    d.scatter_add_(1, token.clamp(min=0)[:, None], s["dlogp"].double()[:, None] * held)
    if c["entropy"]:
        h = torch.nan_to_num(p * (z - s["lse"].double()[:, None] + s["ent"].double()[:, None]), nan=0.0)
        d = d - s["dent"].double()[:, None] * h
    return {"dlogits": d * c["scale"]}


def _exact_linear(c, s):
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v) and v.is_floating_point()}
    off = s["offsets"].tolist()
    rows = [s["order"][a:b].long() for a, b in zip(off[:-1], off[1:])]
    forms = {"none": lambda z: z, "relu": torch.relu, "silu": lambda z: z * torch.sigmoid(z),
             "gelu": lambda z: z * torch.special.ndtr(z)}
    act = forms[c["act"]]
    if c["op"] == "linear":
        y = d["residual"].clone() if c["residual"] else torch.zeros((c["n"], c["out"]), dtype=torch.float64, device="cuda")
        kept = torch.zeros_like(y)
        for g, r in enumerate(rows):
            kept[r] = d["x"][r] @ d["w"][g] + d["bias"][g]
            y[r] += act(kept[r])
        return {"y": y, "z": kept} if c["keep"] else {"y": y}
    z = d["z"].requires_grad_()
    dz = torch.autograd.grad(act(z), z, d["dy"])[0]
    dx, dw = torch.zeros_like(d["x"]), torch.zeros_like(d["w"])
    dbias = torch.zeros((c["groups"], c["out"]), dtype=torch.float64, device="cuda")
    for g, r in enumerate(rows):
        dx[r], dw[g], dbias[g] = dz[r] @ d["w"][g].t(), d["x"][r].t() @ dz[r], dz[r].sum(0)
    return {"dx": dx, "dw": dw, "dbias": dbias}


def _exact_adamw(c, s):
    f = {k: v.double() for k, v in s["flat"].items()}
    out = {k: torch.zeros_like(v) for k, v in f.items() if k != "g"}
    (b1, b2), step = s["betas"], s["steps"] + 1
    m, v = f["m"], f["v"]
    if c["bits"] == 8:
        m, v = m * f["m_scale"].repeat_interleave(BLOCK), (v * f["v_scale"].repeat_interleave(BLOCK)).square()
    m, v = b1 * m + (1 - b1) * f["g"], b2 * v + (1 - b2) * f["g"].square()
    p = f["master" if c["master"] else "p"]
    p = p - s["lr"] * (s["weight_decay"] * p + (m / (1 - b1 ** step)) / ((v / (1 - b2 ** step)).sqrt() + s["eps"]))
    out["p"] = p
    if c["master"]:
        out["master"] = p
    if c["bits"] == 32:
        return {**out, "m": m, "v": v}
    return {**out, "m": None, "v": None, "m_scale": m.view(-1, BLOCK).abs().amax(1) / 448,
            "v_scale": v.sqrt().view(-1, BLOCK).amax(1) / 448}


def exact(case, seed):
    s = prepare(case, seed)
    return {"p": _exact_probs, "l": _exact_linear, "a": _exact_adamw}[case["op"][0]](case, s)
