"""Operators of a model whose gradients the engine's caller passes in, as they are measured.

The engine takes one gradient per worker.  These operators are the layers by which a program makes them:

  products    matrix products grouped by ragged shards of rows (a worker's shard or an expert's tokens)
  norm        layer normalisation; the gradients of its weight and bias are summed by group of rows
  dropout     zeros from the counter-based generator, with or without a residual
  preference  the logistic loss of paired sequences' log ratios, from logits

With `own` false, `run` computes each in plain form from elementary torch operations in 32 bits (64 for sums over a sequence);
with `own` true it calls `paper_2211_00188_amd.layers`.  Group sizes follow from the case, values from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-5


# ---------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------
def _products(name, type, groups, rows, n, k, shared=False, train=True, ragged=True):
    return dict(name=name, kind="products", type=type, groups=groups, rows=rows, n=n, k=k, shared=shared, train=train, ragged=ragged)


def _norm(name, type, groups, rows, d, train=True):
    return dict(name=name, kind="norm", type=type, groups=groups, rows=rows, d=d, train=train)


def _dropout(name, type, rows, d, p, residual):
    return dict(name=name, kind="dropout", type=type, rows=rows, d=d, p=p, residual=residual)


def _preference(name, type, pairs, tokens, v, smoothing=0.0):
    return dict(name=name, kind="preference", type=type, pairs=pairs, tokens=tokens, v=v, smoothing=smoothing)


def listed():
    return [
        # serving: a few tokens, each with the weights of the expert it was sent to (some experts get none)
        _products("products, single tokens", "bf16", 8, 8, 4096, 1024, train=False),
        # a layer of a federated model: a thousand workers with 32 samples each, one layer of 256 x 256 = 65536 weights for all
        # of them, and a gradient of that layer for each
        _products("products, federated", "fp32", 1000, 32000, 256, 256, shared=True, ragged=False),
        # a layer of a small model whose sizes are odd, shards of all lengths
        _products("products, odd", "fp32", 10, 2030, 503, 1001),
        # training the experts' first product over a large batch
        _products("products, experts", "bf16", 16, 16384, 4096, 2048),
        # serving: one token's state
        _norm("norm, one row", "bf16", 1, 1, 4096, train=False),
        # an odd width, shards of all lengths
        _norm("norm, odd", "fp32", 10, 5003, 1001),
        # a large batch of sixteen workers
        _norm("norm, large batch", "bf16", 16, 65536, 2048),
        # a short vector of odd length
        _dropout("dropout, odd", "fp32", 203, 5003, 0.25, False),
        # the end of a residual block over a large batch
        _dropout("dropout, residual", "bf16", 65536, 2048, 0.1, True),
        # two short pairs over a small vocabulary
        _preference("preference, short", "fp32", 2, 61, 1000),
        # an odd vocabulary, label smoothing
        _preference("preference, odd", "fp16", 20, 1500, 49999, 0.1),
        # a batch of pairs over a usual vocabulary
        _preference("preference, batch", "bf16", 16, 8192, 32000),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi, step=64):
    """A width: usually a multiple of `step`, one in three times any number."""
    w = _log(rng, lo, hi)
    return w if rng.random() < 1 / 3 else max(step, w // step * step)


def draw(rng):
    kind = rng.choice(["products", "products", "norm", "dropout", "preference"])
    type = rng.choice(["bf16", "bf16", "fp16", "fp32", "fp32"])
    if kind == "products":
        if rng.random() < 0.3:                       # serving
            c = _products("", type, rng.randint(1, 32), rng.randint(1, 64), _width(rng, 256, 4096), _width(rng, 256, 4096), train=False)
            c["shared"] = rng.random() < 0.3
        else:
            n, k, groups = _width(rng, 64, 4096), _width(rng, 64, 4096), _log(rng, 1, 1000)
            groups = max(1, min(groups, 67000000 // (n * k)))            # (a gradient for each)
            most = min(274877906944 // (2 * n * k) // (4 if type == "fp32" else 1), 800000000 // (2 * SIZE[type] * (n + k)))
            c = _products("", type, groups, _log(rng, 16, max(32, min(65536, most))), n, k)
            c["shared"], c["ragged"] = rng.random() < 0.5, rng.random() < 0.7
    elif kind == "norm":
        d = _width(rng, 64, 8192)
        rows = _log(rng, 1, 134217728 // d // (2 if type == "fp32" else 1))
        c = _norm("", type, max(1, min(_log(rng, 1, 200), rows)), rows, d, rng.random() < 0.7)
    elif kind == "dropout":
        d = _width(rng, 64, 8192)
        c = _dropout("", type, _log(rng, 1, 134217728 // d // (2 if type == "fp32" else 1)), d, rng.choice([0.05, 0.1, 0.2, 0.5]),
                     rng.random() < 0.5)
    else:
        v = _width(rng, 200, 128000)
        tokens = _log(rng, 8, max(16, min(32768, 262144000 // v // (2 if type == "fp32" else 1))))
        c = _preference("", type, max(1, min(_log(rng, 1, 64), tokens // 4)), tokens, v, rng.choice([0.0, 0.0, 0.1]))
    del c["name"]
    return c


def _parts(rows, groups, ragged=True):
    """Sizes that add up to `rows`: even ones, or of very different lengths with empty ones among them."""
    if not ragged:
        return [rows * (g + 1) // groups - rows * g // groups for g in range(groups)]
    rng = random.Random(rows * 1000003 + groups)
    share = [0.0 if groups > 4 and rng.random() < 0.1 else math.exp(rng.uniform(-1.5, 1.5)) for _ in range(groups)]
    if sum(share) == 0.0:
        share[0] = 1.0
    total, done, out = sum(share), 0.0, []
    for s in share:
        a = round(rows * done / total)
        done += s
        out.append(round(rows * done / total) - a)
    return out


def _sizes(case):
    if case["kind"] == "preference":
        return _parts(case["tokens"], 2 * case["pairs"])
    return _parts(case["rows"], case["groups"], case.get("ragged", True))


# ---------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1000003 * seed + 17)
    type = TYPES[case["type"]]

    def normal(*shape, scale=1.0, to=type):
        return torch.randn(*shape, generator=gen, device="cuda").mul_(scale).to(to)

    st = dict(case=case)
    if case["kind"] != "dropout":
        st["sizes"] = _sizes(case)
        st["offsets"] = torch.tensor(np.concatenate([[0], np.cumsum(st["sizes"])]), dtype=torch.int64, device="cuda")
    if case["kind"] == "products":
        g, r, n, k = case["groups"], case["rows"], case["n"], case["k"]
        st["x"] = normal(r, k)
        w = normal(1 if case["shared"] else g, n, k, scale=k ** -0.5)
        st["w"] = w.expand(g, n, k)
        if case["train"]:
            st["dy"] = normal(r, n, scale=1e-2)
    elif case["kind"] == "norm":
        r, d = case["rows"], case["d"]
        # activations: columns of different size, a few of them large, rows off centre
        col = torch.exp(torch.randn(d, generator=gen, device="cuda") * 0.5)
        st["x"] = (torch.randn(r, d, generator=gen, device="cuda") * col + torch.randn(r, 1, generator=gen, device="cuda") * 0.5).to(type)
        st["weight"], st["bias"] = 1.0 + normal(d, scale=0.1, to=torch.float32), normal(d, scale=0.1, to=torch.float32)
        if case["train"]:
            st["dy"] = normal(r, d, scale=1e-2)
    elif case["kind"] == "dropout":
        st["x"] = normal(case["rows"], case["d"])
        st["residual"] = normal(case["rows"], case["d"]) if case["residual"] else None
        st["seed"], st["step"], st["layer"] = 0x9E3779B97F4A7C15 ^ seed, 7 + seed, 3
    else:
        t, v, p = case["tokens"], case["v"], case["pairs"]
        logits = torch.randn(t, v, generator=gen, device="cuda").mul_(2.0)
        targets = torch.randint(0, v, (t,), generator=gen, device="cuda")
        logits[torch.arange(t, device="cuda"), targets] += 6.0
        st["logits"] = logits.to(type)
        # prompts and padding carry no target
        st["targets"] = torch.where(torch.rand(t, generator=gen, device="cuda") < 0.25, -100, targets)
        # log-probabilities of the targets under the model that training began with
        t0 = torch.gather(torch.log_softmax(logits, 1), 1, targets[:, None])[:, 0]
        st["ref"] = t0 + 0.3 * torch.randn(t, generator=gen, device="cuda")
        st["dloss"] = torch.full((p,), 1.0 / p, device="cuda")                  # the mean over a worker's pairs
        st["beta"] = 0.1
    return st


# ---------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(st):
    from paper_2211_00188_amd import layers as L
    case = st["case"]
    train = case.get("train", True)
    if case["kind"] == "products":
        y = L.group_matmul(st["x"], st["w"], st["offsets"])
        if not train:
            return y
        return y, L.group_matmul_dx(st["dy"], st["w"], st["offsets"]), L.group_matmul_dw(st["dy"], st["x"], st["offsets"])
    if case["kind"] == "norm":
        y, mean, rstd = L.layer_norm(st["x"], st["weight"], st["bias"], EPS)
        if not train:
            return y
        dx, dw, db = L.layer_norm_backward(st["dy"], st["x"], st["weight"], mean, rstd, st["offsets"])
        return y, mean, rstd, dx, dw, db
    if case["kind"] == "dropout":
        return L.dropout(st["x"], case["p"], st["seed"], step=st["step"], layer=st["layer"], residual=st["residual"])
    loss, margin, logp, lse = L.preference_loss(st["logits"], st["targets"], st["offsets"], st["ref"], st["beta"], case["smoothing"])
    return loss, margin, logp, lse, L.preference_loss_backward(st["dloss"], st["logits"], st["targets"], st["offsets"], margin, lse,
                                                               st["beta"], case["smoothing"])


def _philox(c0, c1, c2, c3, seed):
    """Ten rounds of Philox4x32 on int64 tensors that hold 32-bit words."""
    low, k0, k1 = 0xFFFFFFFF, seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57        # (modulo 2^64)
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _run_plain(st):
    case = st["case"]
    train = case.get("train", True)
    if case["kind"] == "products":
        x, w, sizes = st["x"].float(), st["w"], st["sizes"]
        y = torch.empty(x.shape[0], w.shape[1], device=x.device)
        if train:
            dy = st["dy"].float()
            dx, dw = torch.empty_like(x), torch.zeros(w.shape, device=x.device)
        if case["shared"]:
            w0 = w[0].float()
            y = x @ w0.t()
            if train:
                dx = dy @ w0
        a = 0
        for g, m in enumerate(sizes):
            b = a + m
            if m and not case["shared"]:
                wg = w[g].float()
                y[a:b] = x[a:b] @ wg.t()
                if train:
                    dx[a:b] = dy[a:b] @ wg
            if m and train:
                dw[g] = dy[a:b].t() @ x[a:b]
            a = b
        to = st["x"].dtype
        return (y.to(to), dx.to(to), dw) if train else y.to(to)
    if case["kind"] == "norm":
        x = st["x"].float()
        mean = x.mean(1, keepdim=True)
        c = x - mean
        rstd = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
        xh = c * rstd
        y = (xh * st["weight"] + st["bias"]).to(st["x"].dtype)
        if not train:
            return y
        dy = st["dy"].float()
        dxh = dy * st["weight"]
        dx = rstd * (dxh - dxh.mean(1, keepdim=True) - xh * (dxh * xh).mean(1, keepdim=True))
        prod, a, dw, db = dy * xh, 0, [], []
        for m in st["sizes"]:
            dw.append(prod[a:a + m].sum(0))
            db.append(dy[a:a + m].sum(0))
            a += m
        return y, mean[:, 0], rstd[:, 0], dx.to(st["x"].dtype), torch.stack(dw), torch.stack(db)
    if case["kind"] == "dropout":
        x = st["x"]
        e = x.numel()
        block = torch.arange((e + 7) // 8, device=x.device)
        zero = torch.zeros_like(block)
        words = torch.stack(_philox(block & 0xFFFFFFFF, block >> 32, zero + st["step"], zero + st["layer"] + 1, st["seed"]), 1)
        draws = torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)[:e].view(x.shape)
        cut = int(math.floor(case["p"] * 65536 + 0.5))
        scale = torch.tensor(65536.0 / (65536 - cut), dtype=torch.float32, device=x.device)
        out = torch.where(draws >= cut, x.float() * scale, 0.0)
        if st["residual"] is not None:
            out = out + st["residual"].float()
        return out.to(x.dtype)
    logits, target, sizes = st["logits"].float(), st["targets"], st["sizes"]
    t = logits.shape[0]
    top = logits.max(1, keepdim=True).values
    ex = torch.exp(logits - top)
    total = ex.sum(1, keepdim=True)
    rows, valid = torch.arange(t, device=logits.device), target >= 0
    at = target.clamp(min=0)
    logsum = torch.log(total[:, 0].double())
    logp = torch.where(valid, (logits[rows, at] - top[:, 0]).double() - logsum, 0.0)
    ratio = torch.where(valid, logp - st["ref"].double(), 0.0)
    seq = torch.repeat_interleave(torch.arange(len(sizes), device=logits.device), torch.tensor(sizes, device=logits.device))
    sums = torch.zeros(len(sizes), dtype=torch.float64, device=logits.device).index_add_(0, seq, ratio)
    margin = sums[0::2] - sums[1::2]
    z = st["beta"] * margin
    s = case["smoothing"]
    soft = torch.log1p(torch.exp(-z.abs()))
    loss = (1 - s) * (soft + (-z).clamp(min=0)) + s * (soft + z.clamp(min=0))
    dz = s / (1 + torch.exp(-z)) - (1 - s) / (1 + torch.exp(z))
    dlogp = (st["dloss"] * dz * st["beta"])[:, None] * torch.tensor([1.0, -1.0], dtype=torch.float64, device=logits.device)
    scale = torch.where(valid, dlogp.reshape(-1)[seq].float(), 0.0)
    grad = -(ex / total)
    grad[rows, at] += 1.0
    lse = torch.where(valid, top[:, 0].double() + logsum, 0.0)
    return loss.float(), margin.float(), logp.float(), lse.float(), (grad * scale[:, None]).to(st["logits"].dtype)


# ---------------------------------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    train = case.get("train", True)
    if case["kind"] == "products":
        x, w = st["x"].double(), st["w"]
        dy = st["dy"].double() if train else None
        ys, dxs, dws = [], [], []
        first = st["offsets"].tolist()
        for g in range(case["groups"]):
            part = slice(first[g], first[g + 1])
            wg = w[g].double()
            ys.append(torch.mm(wg, x[part].t()).t())
            if train:
                dxs.append(torch.mm(wg.t(), dy[part].t()).t())
                dws.append(torch.mm(x[part].t(), dy[part]).t())
        return (torch.cat(ys), torch.cat(dxs), torch.stack(dws)) if train else torch.cat(ys)
    if case["kind"] == "norm":
        x, w, b = st["x"].double(), st["weight"].double(), st["bias"].double()
        d = case["d"]
        mean = x.sum(1) / d
        var = ((x - mean[:, None]) ** 2).sum(1) / d
        rstd = (var + EPS) ** -0.5
        xh = (x - mean[:, None]) * rstd[:, None]
        y = xh * w + b
        if not train:
            return y
        dy = st["dy"].double()
        a = dy * w
        # dx_i = r (a_i - sum_j a_j (1 + xh_i xh_j) / d)
        dx = rstd[:, None] * (a - (a.sum(1)[:, None] + xh * (a * xh).sum(1)[:, None]) / d)
        group = torch.repeat_interleave(torch.arange(case["groups"], device=x.device), torch.tensor(st["sizes"], device=x.device))
        pick = (group[None, :] == torch.arange(case["groups"], device=x.device)[:, None]).double()
        return y, mean, rstd, dx, torch.mm(pick, dy * xh), torch.mm(pick, dy)
    if case["kind"] == "dropout":
        count = case["rows"] * case["d"]
        blocks = (count + 7) // 8
        # (32-bit words in 64-bit numbers)
        c = [np.arange(blocks, dtype=np.uint64), np.zeros(blocks, np.uint64), np.full(blocks, st["step"], np.uint64),
             np.full(blocks, st["layer"] + 1, np.uint64)]
        c[1], c[0] = c[0] >> np.uint64(32), c[0] & np.uint64(0xFFFFFFFF)
        key = [st["seed"] % 2 ** 32, st["seed"] // 2 ** 32]
        for r in range(10):
            ka, kb = (np.uint64((key[0] + r * 0x9E3779B9) % 2 ** 32), np.uint64((key[1] + r * 0xBB67AE85) % 2 ** 32))
            a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
            c = [(b >> np.uint64(32)) ^ c[1] ^ ka, b & np.uint64(0xFFFFFFFF), (a >> np.uint64(32)) ^ c[3] ^ kb, a & np.uint64(0xFFFFFFFF)]
        halves = np.empty((blocks, 8), np.uint16)
        for i in range(4):
            halves[:, 2 * i], halves[:, 2 * i + 1] = c[i] & np.uint64(0xFFFF), c[i] >> np.uint64(16)
        cut = math.floor(case["p"] * 65536 + 0.5)
        keep = torch.from_numpy(halves.reshape(-1)[:count].astype(np.int32) >= cut).cuda().view(st["x"].shape)
        out = st["x"].double() * keep * (65536 / (65536 - cut))
        return out if st["residual"] is None else out + st["residual"].double()
    first = st["offsets"].tolist()
    s, beta = case["smoothing"], st["beta"]
    logp, lse, sums, probs = [], [], [], []
    for i in range(2 * case["pairs"]):
        part = slice(first[i], first[i + 1])
        x, at = st["logits"][part].double(), st["targets"][part]
        lp = torch.log_softmax(x, 1)
        has = (at >= 0).nonzero()[:, 0]
        token = torch.zeros_like(x[:, 0])
        lse.append(torch.zeros_like(token))
        lse[-1][has] = torch.logsumexp(x[has], 1)
        token[has] = lp[has, at[has]]
        logp.append(token)
        sums.append((token[has] - st["ref"][part][has].double()).sum())
        grad = torch.zeros_like(lp)
        grad[has] = -torch.exp(lp[has])
        grad[has, at[has]] += 1.0
        probs.append(grad)
    loss, margin = [], []
    for p in range(case["pairs"]):
        margin.append(sums[2 * p] - sums[2 * p + 1])
        m, zero = margin[p] * beta, torch.zeros_like(margin[p])
        loss.append((1 - s) * torch.logaddexp(-m, zero) + s * torch.logaddexp(m, zero))
        slope = beta * ((1 - s) * torch.sigmoid(-m) - s * torch.sigmoid(m)) * st["dloss"][p].double()      # - d loss / d margin
        probs[2 * p] *= -slope
        probs[2 * p + 1] *= slope
    return torch.stack(loss), torch.stack(margin), torch.cat(logp), torch.cat(lse), torch.cat(probs)


# ---------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------
def work(case):
    e = SIZE[case["type"]]
    if case["kind"] == "products":
        g, r, n, k = case["groups"], case["rows"], case["n"], case["k"]
        used = 1 if case["shared"] else sum(m > 0 for m in _sizes(case))
        size = e * (r * k + used * n * k + r * n) + 8 * (g + 1)
        if case["train"]:
            size += e * (r * n + r * k) + 4 * g * n * k
        return dict(bytes=size, flops=2 * r * n * k * (3 if case["train"] else 1))
    if case["kind"] == "norm":
        r, d = case["rows"], case["d"]
        size = 2 * e * r * d + 8 * d
        if case["train"]:
            size += 2 * e * r * d + 8 * r + 8 * case["groups"] * d
        return dict(bytes=size, flops=r * d * (24 if case["train"] else 8))
    if case["kind"] == "dropout":
        count = case["rows"] * case["d"]
        return dict(bytes=e * count * (3 if case["residual"] else 2), flops=count * (3 if case["residual"] else 2))
    t, v = case["tokens"], case["v"]
    # (the quarter of the tokens that carry no target is not read)
    return dict(bytes=(e * t * v * 7) // 4 + 20 * t + 28 * case["pairs"], flops=t * v * 8)
