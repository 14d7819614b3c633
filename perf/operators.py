"""The operators on a routed batch, and the calls they are timed on.

The router answers a batch with one pair per query.  What a serving or training
program does next on the card is to run every row with the weights of the model
it went to:

* group: the rows of each model, in row order (offsets and a row order), from
  the router's choices and the pair -> model table;
* matmul: y[r] = x[r] W[g(r)], a product with the weights of the row's group, of
  ragged sizes, and its gradients dx[r] = dy[r] W[g(r)]^T and
  dW[g] = sum over the group's rows of x[r]^T dy[r];
* adapter: y[r] = x[r] W + s[g] (x[r] A[g]) B[g], one shared projection and the
  low-rank adapter of the row's group, and the gradients of x, A and B.

A row in no group gets zeros from matmul and the shared projection alone from
adapter.  Weights are [in][out], row-major, as everywhere in the library.

Widths and batch sizes are those of the routing workloads (384 to 1536 wide
embeddings, 1 to a million queries, 4 to 32 models) and generic ones beside them.
"""
import math
from functools import lru_cache

import torch

own = False

#: how rows spread over the groups: the share of group i is proportional to (i + 1) ** -SKEW
SKEW = {"even": 0.0, "mild": 0.5, "steep": 1.0}


def _case(name, op, dtype, n, groups, k=0, out=0, rank=0, skew="mild", none=0.0, pairs=0):
    return {"name": name, "op": op, "dtype": dtype, "n": n, "groups": groups, "k": k, "out": out, "rank": rank,
            "skew": skew, "none": none, "pairs": pairs}


def listed():
    return [
        # one step of a serving loop: the choices of the requests in flight, 16 models on 2 kinds of GPU
        _case("group_step", "group", "i32", 64, 16, pairs=32),
        # the choices of a million queries among 256 pairs of 32 models
        _case("group_million", "group", "i32", 1048576, 32, pairs=256),
        # token generation: a few rows a model, every model's weights are read
        _case("matmul_tokens", "matmul", "bf16", 40, 16, 1024, 2048),
        # prompts of a batch, spread unevenly, some rejected
        _case("matmul_prompts", "matmul", "bf16", 16384, 16, 2048, 4096, none=0.05),
        # fp32 heads on small embeddings, an odd number of rows
        _case("matmul_f32", "matmul", "f32", 1003, 13, 576, 384),
        # a training step's gradients
        _case("matmul_grad", "matmul_grad", "bf16", 12000, 8, 2048, 2048),
        # the same in fp32, widths that no tile divides
        _case("matmul_grad_f32", "matmul_grad", "f32", 2051, 5, 771, 390, skew="steep"),
        # one request generating one token
        _case("adapter_token", "adapter", "bf16", 1, 32, 4096, 4096, 16),
        # the requests in flight generating one token each, some on the shared model itself
        _case("adapter_tokens", "adapter", "bf16", 48, 32, 4096, 4096, 16, none=0.1),
        # prompts of a batch
        _case("adapter_prompts", "adapter", "bf16", 12288, 12, 4096, 4096, 32, none=0.1),
        # fp32, ordinary size
        _case("adapter_f32", "adapter", "f32", 777, 6, 1024, 1536, 8),
        # fine-tuning of several adapters in one batch
        _case("adapter_grad", "adapter_grad", "bf16", 8192, 8, 2048, 2048, 16, none=0.05),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["group", "matmul", "matmul", "matmul_grad", "adapter", "adapter", "adapter_grad"])
    groups = _log(rng, 1, 32)
    c = _case("", op, "i32", 1, groups, skew=rng.choice(sorted(SKEW)), none=rng.choice([0.0, 0.0, rng.uniform(0.01, 0.3)]))
    del c["name"]
    if op == "group":
        c.update(n=_log(rng, 1, 1048576), pairs=groups * rng.randint(1, 8))
        return c
    c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
    wide = 4096 if c["dtype"] == "bf16" else 1536
    # widths: half of them whole vectors, the others as they come
    k, out = (_log(rng, 256, wide) for _ in range(2))
    if rng.random() < 0.5:
        k, out = (k + 63) // 64 * 64, (out + 63) // 64 * 64
    tokens = op in ("matmul", "adapter") and rng.random() < 0.4
    n = _log(rng, 1, 64) if tokens else _log(rng, 64, 16384 if c["dtype"] == "bf16" else 4096)
    c.update(k=k, out=out, n=n, rank=rng.choice([4, 8, 16, 24, 32, 64]) if op.startswith("adapter") else 0)
    cap = max(_cost(x) for x in listed())
    while _cost(c) > cap:
        c["n"] = max(1, int(c["n"] * 0.7))
    return c


# ---------------------------------------------------------------- inputs
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _shares(c):
    p = [(i + 1.0) ** -SKEW[c["skew"]] for i in range(c["groups"])]
    return [x / sum(p) for x in p]


def prepare(case, seed):
    c = case
    n, G, k, out, R = c["n"], c["groups"], c["k"], c["out"], c["rank"]
    g = torch.Generator("cuda").manual_seed(1000003 * seed + 11)
    share = torch.tensor(_shares(c), device="cuda")
    perm = torch.randperm(G, generator=g, device="cuda")
    gid = perm[torch.multinomial(share, n, replacement=True, generator=g)]
    away = torch.rand(n, generator=g, device="cuda") < c["none"]
    gid = torch.where(away, -1, gid)
    s = {"op": c["op"], "n": n, "groups": G}
    if c["op"] == "group":
        # the router's choices: one of the pairs that hold the row's model, -1 for a query that was turned away
        P = c["pairs"]
        model = torch.arange(P, device="cuda") % G                 # pair -> model
        pick = torch.randint(0, P // G, (n,), generator=g, device="cuda") * G + gid
        s.update(choice=torch.where(away, -1, pick).to(torch.int32), model=model.to(torch.int32),
                 out={"offsets": torch.empty(G + 1, dtype=torch.int32, device="cuda"),
                      "order": torch.empty(n, dtype=torch.int32, device="cuda")})
        return s
    s.update(_plain_group(torch.where(away, G, gid), G))
    s["cap"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())   # the plain form's: rows of the largest group
    t = _TYPES[c["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(t)

    s["x"] = normal(n, k)
    s["x"][:, ::97] *= 8                                           # a few channels are much larger than the others
    if c["op"].startswith("matmul"):
        s["w"] = normal(G, k, out, std=k ** -0.5)
    else:
        s["w"] = normal(k, out, std=k ** -0.5)
        s["a"], s["b"] = normal(G, k, R, std=k ** -0.5), normal(G, R, out, std=0.3 * R ** -0.5)
        s["scale"] = 0.5 + 1.5 * torch.rand(G, generator=g, device="cuda")
    if c["op"].endswith("_grad"):
        s["dy"] = normal(n, out, std=1e-2)
        like = {"dx": "x", "dw": "w"} if c["op"] == "matmul_grad" else {"dx": "x", "da": "a", "db": "b"}
        s["out"] = {d: torch.empty_like(s[v]) for d, v in like.items()}
    else:
        s["out"] = {"y": torch.empty(n, out, dtype=t, device="cuda")}
    return s


# ---------------------------------------------------------------- the plain forms
def _plain_group(key, G):
    """Stable order of the rows by group (key G: in none), and where each group begins."""
    keys, order = torch.sort(key, stable=True)
    offsets = torch.searchsorted(keys, torch.arange(G + 1, device=key.device))
    return {"offsets": offsets.to(torch.int32), "order": order.to(torch.int32)}


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


def _product(x, w, rows, held, n):
    return _put(torch.bmm(_take(x, rows, held), w.float()), rows, held, n)


def _plain(s):
    op, n = s["op"], s["n"]
    if op == "group":
        c, G = s["choice"].long(), s["groups"]
        return _plain_group(torch.where(c >= 0, s["model"].long()[c.clamp(min=0)], G), G)
    t = s["x"].dtype
    rows, held = _padded(s)
    if op == "matmul":
        return {"y": _product(s["x"], s["w"], rows, held, n).to(t)}
    if op == "matmul_grad":
        dx = _product(s["dy"], s["w"].float().transpose(1, 2).contiguous(), rows, held, n)
        dw = torch.bmm(_take(s["x"], rows, held).transpose(1, 2).contiguous(), _take(s["dy"], rows, held))
        return {"dx": dx.to(t), "dw": dw.to(t)}
    scale = s["scale"][:, None, None]
    a, b, w = s["a"].float(), s["b"].float(), s["w"].float()
    if op == "adapter":
        low = torch.bmm(_take(s["x"], rows, held), a) * scale
        return {"y": (s["x"].float() @ w + _put(torch.bmm(low, b), rows, held, n)).to(t)}
    x, dy = _take(s["x"], rows, held), _take(s["dy"], rows, held)
    low = torch.bmm(x, a) * scale
    up = torch.bmm(dy, b.transpose(1, 2).contiguous()) * scale
    dx = s["dy"].float() @ w.t() + _put(torch.bmm(up, a.transpose(1, 2).contiguous()), rows, held, n)
    da = torch.bmm(x.transpose(1, 2).contiguous(), up)
    db = torch.bmm(low.transpose(1, 2).contiguous(), dy)
    return {"dx": dx.to(t), "da": da.to(t), "db": db.to(t)}


# ---------------------------------------------------------------- the framework's operators
@lru_cache(maxsize=None)
def _ops(stream):
    from paper_2608_14575_amd import routed
    return routed.RoutedOps(stream=stream)


def run(state):
    s = state
    if not own:
        return _plain(s)
    ops, op, out = _ops(torch.cuda.current_stream().cuda_stream), s["op"], s["out"]
    if op == "group":
        ops.group(s["choice"], s["groups"], table=s["model"], **out)
    elif op == "matmul":
        ops.matmul(s["x"], s["w"], s["offsets"], s["order"], **out)
    elif op == "matmul_grad":
        ops.matmul_grad(s["dy"], s["x"], s["w"], s["offsets"], s["order"], **out)
    elif op == "adapter":
        ops.adapter(s["x"], s["w"], s["a"], s["b"], s["scale"], s["offsets"], s["order"], **out)
    else:
        ops.adapter_grad(s["dy"], s["x"], s["w"], s["a"], s["b"], s["scale"], s["offsets"], s["order"], **out)
    return out


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    n, G, k, out, R = c["n"], c["groups"], c["k"], c["out"], c["rank"]
    if c["op"] == "group":
        return {"bytes": 4 * n + 4 * c["pairs"] + 4 * (G + 1) + 4 * n, "flops": 0}
    size = 2 if c["dtype"] == "bf16" else 4
    held = n * (1 - c["none"])
    used = sum(1 - (1 - p * (1 - c["none"])) ** n for p in _shares(c))   # groups that have a row
    index = 4 * n + 4 * (G + 1)
    if c["op"] == "matmul":
        return {"bytes": size * (held * k + used * k * out + n * out) + index, "flops": 2 * held * k * out}
    if c["op"] == "matmul_grad":
        return {"bytes": size * (held * (out + k) + used * k * out + n * k + G * k * out) + index, "flops": 4 * held * k * out}
    low = 2 * held * R * (k + out)
    if c["op"] == "adapter":
        return {"bytes": size * (n * (k + out) + k * out + used * R * (k + out)) + 4 * G + index,
                "flops": 2 * n * k * out + low}
    return {"bytes": size * (n * (out + 2 * k) + k * out + (used + G) * R * (k + out)) + 4 * G + index,
            "flops": 2 * n * k * out + 2.5 * low}


def _cost(c):
    """Arithmetic of the plain form, in units of bf16 work: fp32 products run at a fraction of the rate."""
    return work(c)["flops"] * (8 if c["dtype"] == "f32" else 1)


# ---------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "group":
        return None
    t = torch.float64
    x, w = s["x"].to(t), s["w"].to(t)
    off = s["offsets"].tolist()
    rows = [s["order"][a:b].long() for a, b in zip(off[:-1], off[1:])]
    if c["op"] == "matmul":
        y = torch.zeros((c["n"], c["out"]), dtype=t, device="cuda")
        for g, r in enumerate(rows):
            y[r] = x[r] @ w[g]
        return {"y": y}
    if c["op"] == "matmul_grad":
        dy, dx, dw = s["dy"].to(t), torch.zeros_like(x), torch.zeros_like(w)
        for g, r in enumerate(rows):
            dx[r] = dy[r] @ w[g].t()
            dw[g] = x[r].t() @ dy[r]
        return {"dx": dx, "dw": dw}
    a, b, scale = s["a"].to(t), s["b"].to(t), s["scale"].to(t)
    if c["op"] == "adapter":
        y = x @ w
        for g, r in enumerate(rows):
            y[r] += scale[g] * ((x[r] @ a[g]) @ b[g])
        return {"y": y}
    dy, da, db = s["dy"].to(t), torch.zeros_like(a), torch.zeros_like(b)
    dx = dy @ w.t()
    for g, r in enumerate(rows):
        up = scale[g] * (dy[r] @ b[g].t())
        dx[r] += up @ a[g].t()
        da[g] = x[r].t() @ up
        db[g] = scale[g] * (x[r] @ a[g]).t() @ dy[r]
    return {"dx": dx, "da": da, "db": db}
