"""The proposing operators' calls: what is timed, on which inputs, and what the results are.

A learned search over frequency policies draws each pack's level from a row of logits (adjust: penalties,
bias, temperature, mask, and a choice), evaluates the drawn candidates, and moves the logits towards the best of
them (distillation).  The same two operators serve wide rows: a choice among a batch's candidates, a
vocabulary's logits, a larger model's top logits as teacher.

Fields of a case: `op` ("adjust", or the distillation's "forward", "backward" or "step"), `rows` (rows of the
call), `distinct` (rows of the logits: row r reads row r % distinct), `V` (entries of a row), `dtype` of the
logits.  adjust: `noise` (rows of noise added for the choice, 0: none), `mask` (rows of mask words, 0: none),
`bias` (its rows), `L` (history columns, 0: no penalties), `ids` (type of the history), `out` (type of the
adjusted logits, "": not written), `choice` (type of the chosen index, "": none).  distillation: `K` (teacher
entries of a row), `ids` (their type), `elites` (ids are K candidates' level bytes read column by column and
the teacher's logits are shared by all rows), `mask`, `tau` (temperature), `padded` (rows at the end without a
teacher).
"""
from __future__ import annotations

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "u8": torch.uint8, "i32": torch.int32,
          "i64": torch.int64}
SIZES = {"f32": 4, "bf16": 2, "f16": 2, "u8": 1, "i32": 4, "i64": 8}

# ------------------------------------------------------------------------------ the cases


def _adjust(name, rows, V, dtype, distinct=0, noise=0, mask=0, bias=0, L=0, ids="i32", out="", choice=""):
    c = {"op": "adjust", "rows": rows, "distinct": distinct or rows, "V": V, "dtype": dtype, "noise": noise, "mask": mask,
         "bias": bias, "L": L, "ids": ids, "out": out, "choice": choice}
    return {"name": name, **c} if name else c


def _distill(name, op, rows, V, dtype, K, ids="i32", elites=False, mask=0, tau=1.0, padded=0):
    c = {"op": op, "rows": rows, "distinct": rows, "V": V, "dtype": dtype, "K": K, "ids": ids, "elites": elites, "mask": mask,
         "tau": tau, "padded": padded}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one policy of a 64-pack serving graph drawn from its packs' logits (latency)
        _adjust("choose-64p", 64, 8, "f32", noise=64, mask=64, choice="u8"),
        # 4,096 candidates of a 512-pack training graph drawn at once from the packs' logits, levels masked by pack
        _adjust("propose-512p", 512 * 4096, 16, "f32", distinct=512, noise=512 * 4096, mask=512, choice="u8"),
        # a draw among one million evaluated candidates under each of two latency targets' feasibility masks
        _adjust("among-1m", 2, 1 << 20, "f32", distinct=1, noise=2, mask=2, choice="i64"),
        # one token: penalties over its history, a bias and a grammar mask, adjusted logits and the greedy choice
        _adjust("token-32768", 1, 32768, "bf16", mask=1, bias=1, L=500, out="bf16", choice="i32"),
        # a decoding batch with a large vocabulary
        _adjust("decode-131072", 256, 131072, "bf16", mask=256, bias=1, L=1024, out="bf16", choice="i32"),
        # a decoding batch of an odd vocabulary, long ragged histories, one mask for all, results in 32 bits
        _adjust("ragged-100003", 333, 100003, "f16", mask=1, L=4096, ids="i64", out="f32", choice="i64"),
        # a small graph's logits learn from its 32 best candidates (latency)
        _distill("elites-64p", "step", 64, 8, "f32", 32, ids="u8", elites=True),
        # a per-kernel graph's logits learn from its 64 best candidates
        _distill("elites-65536k", "step", 65536, 16, "f32", 64, ids="u8", elites=True, mask=65536),
        # a larger model's top 64 logits, large vocabulary: the two passes of a training step on their own
        _distill("forward-131072", "forward", 2048, 131072, "bf16", 64, tau=2.0),
        _distill("backward-131072", "backward", 2048, 131072, "bf16", 64, tau=2.0),
        # a training step's loss and gradient in one call
        _distill("step-32768", "step", 8192, 32768, "bf16", 32, ids="i64"),
        # an odd vocabulary in 32 bits, masked entries, a padded batch
        _distill("step-50021", "step", 517, 50021, "f32", 100, mask=1, tau=1.5, padded=23),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more call of the listed ranges: rows of 2 to 64 levels by the thousand or million, rows of up to
    a million entries down to a single row, histories of 1 to 8,192 ids, teachers of 1 to 128 entries."""
    entries = 1 << 27
    if rng.random() < 0.5:
        dtype = rng.choice(["f32", "bf16", "f16"])
        if rng.random() < 0.4:                                  # levels of packs, for some candidates
            V, P = rng.choice([2, 4, 7, 8, 11, 16, 24, 64]), _log_int(rng, 8, 4096)
            B = _log_int(rng, 1, max(2, min(4096, (1 << 25) // (V * P))))
            return _adjust(None, P * B, V, dtype, distinct=P, noise=P * B, mask=rng.choice([0, 1, P]), choice="u8")
        V = _log_int(rng, 65, 1 << 20)
        rows = _log_int(rng, 1, max(2, min(4096, (1 << 25) // V)))
        L = rng.choice([0, _log_int(rng, 1, 8192)])
        out = rng.choice(["", "f32", dtype])
        return _adjust(None, rows, V, dtype, noise=rng.choice([0, rows]), mask=rng.choice([0, 1, rows]),
                       bias=rng.choice([0, 1, rows]), L=L, ids=rng.choice(["i32", "i64"]), out=out,
                       choice=rng.choice(["i32", "i64"]))
    op = rng.choice(["forward", "backward", "step"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    tau = rng.choice([1.0, 0.7, 2.0])
    if rng.random() < 0.4:
        V, rows = rng.choice([2, 4, 7, 8, 11, 16, 24, 64]), _log_int(rng, 8, 65536)
        return _distill(None, op, rows, V, dtype, rng.choice([1, 8, 33, 64, 100]), ids="u8", elites=True,
                        mask=rng.choice([0, 1, rows]), tau=tau)
    V = _log_int(rng, 65, 1 << 18)
    rows = _log_int(rng, 1, max(2, min(8192, entries // V)))
    return _distill(None, op, rows, V, dtype, rng.choice([1, 7, 20, 64, 128]), ids=rng.choice(["i32", "i64"]),
                    mask=rng.choice([0, 1, rows]), tau=tau, padded=rows // 20)


# ------------------------------------------------------------------------------ inputs


def _words(gen, n, V, keep):
    """Mask words of n rows: bit v % 32 of word v / 32 is 1 where entry v is allowed (a share `keep` of them)."""
    W = (V + 31) // 32
    allowed = torch.rand((n, W * 32), generator=gen, device="cuda") < keep
    allowed[:, V:] = False
    bits = allowed.view(n, W, 32).to(torch.int64) << torch.arange(32, device="cuda")
    return bits.sum(-1).to(torch.int32)


def _uniform(gen, shape, lo, hi):
    return torch.rand(shape, generator=gen, device="cuda") * (hi - lo) + lo


def _inputs(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    R, V = c["rows"], c["V"]
    s = {"c": c, "mask": None}
    s["logits"] = torch.randn((c["distinct"], V), generator=gen, device="cuda").mul_(2.5).to(DTYPES[c["dtype"]])
    if c["mask"]:
        s["mask"] = _words(gen, c["mask"], V, 0.7)
        if c["mask"] > 2:
            s["mask"][1] = 0                # a row whose mask leaves nothing
    if c["op"] == "adjust":
        s["noise"] = s["bias"] = s["history"] = s["lengths"] = None
        s["rates"] = {}
        if c["noise"]:                      # Gumbel noise: the greatest sum is a draw from the row's softmax
            u = torch.rand((c["noise"], V), generator=gen, device="cuda").clamp_(min=1e-7, max=1 - 1e-7)
            s["noise"] = u.log_().neg_().log_().neg_()
        if c["bias"]:
            s["bias"] = torch.randn((c["bias"], V), generator=gen, device="cuda").mul_(0.5)
        if c["L"]:
            # a text repeats itself: ids crowd towards the low end of the vocabulary
            u = torch.rand((R, c["L"]), generator=gen, device="cuda").pow_(3.0)
            s["history"] = (u * V).to(torch.int64).clamp_(max=V - 1).to(DTYPES[c["ids"]])
            s["lengths"] = torch.randint(0, c["L"] + 1, (R,), generator=gen, device="cuda", dtype=torch.int32)
            s["lengths"][0] = c["L"]
            s["rates"] = {"repetition": _uniform(gen, R, 1.0, 1.3), "frequency": _uniform(gen, R, 0.0, 0.5),
                          "presence": _uniform(gen, R, 0.0, 0.6)}
        s["rates"]["inv_temperature"] = _uniform(gen, R if V > 64 else 1, 0.6, 1.6)
        return s
    N, K = R, c["K"]
    if c["elites"]:
        # the levels of the K best candidates, as the evaluator reads them, and their energies over a temperature
        levels = torch.randint(0, V, (K, N), generator=gen, device="cuda", dtype=torch.uint8)
        s["ids"] = levels.t()
        s["teacher"] = torch.rand((1, K), generator=gen, device="cuda").mul_(-3.0)
    else:
        s["ids"] = torch.randint(0, V, (N, K), generator=gen, device="cuda").to(DTYPES[c["ids"]])
        s["teacher"] = torch.randn((N, K), generator=gen, device="cuda").mul_(1.5).add_(6.0).sort(-1, descending=True)[0]
    if c["padded"]:
        s["ids"][N - c["padded"]:] = -1
    mean = (16384.0 if c["dtype"] == "f16" else 1.0) / N        # 16-bit floats of 5 exponent bits: a scaled loss
    s["scale"] = torch.full((1,), mean, device="cuda") if c["op"] == "step" else _uniform(gen, N, 0.0, 2.0 * mean)
    return s


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    R, V = c["rows"], c["V"]
    if c["op"] == "adjust":
        s["out"] = torch.empty((R, V), dtype=DTYPES[c["out"]], device="cuda") if c["out"] else None
        s["choice"] = torch.empty(R, dtype=DTYPES[c["choice"]], device="cuda") if c["choice"] else None
        return s
    s["loss"] = torch.empty(R, dtype=torch.float32, device="cuda")
    s["stats"] = torch.empty((R, 2), dtype=torch.float32, device="cuda")
    if c["op"] == "backward":               # kept from the forward pass
        for r, n, x, _ in _blocks(s, torch.float64):
            s["stats"][r:r + n] = torch.cat(_statistics(x, c["tau"]), 1)
    if c["op"] != "forward":
        s["grad"] = torch.empty((R, V), dtype=DTYPES[c["dtype"]], device="cuda")
    return s


# ------------------------------------------------------------------------------ plain forms


def _allowed(words, V):
    bits = (words.unsqueeze(-1) >> torch.arange(32, device=words.device, dtype=torch.int32)) & 1
    return bits.reshape(words.shape[0], -1)[:, :V].bool()


def _rows(t, R):
    """Row r of the call reads row r % n of an operand of n rows."""
    return t if t.shape[0] in (1, R) else t.repeat((R // t.shape[0],) + (1,) * (t.dim() - 1))


def _pick(y, dtype):
    """The lowest index of each row's greatest value; -1 (255 in a byte) where nothing is above -inf."""
    V = y.shape[1]
    best = y.amax(-1, keepdim=True)
    at = torch.where(y == best, torch.arange(V, device=y.device, dtype=torch.int32), V).amin(-1)
    return torch.where(best[:, 0] > float("-inf"), at, torch.full_like(at, -1)).to(dtype)


def _plain_adjust(s):
    c = s["c"]
    R, V = c["rows"], c["V"]
    x = s["logits"].float()
    rates = {k: _rows(t.unsqueeze(-1), R) for k, t in s["rates"].items()}
    if c["L"]:
        live = torch.arange(c["L"], device=x.device) < s["lengths"].unsqueeze(-1)
        n = torch.zeros((R, V), dtype=torch.int32, device=x.device)
        n.scatter_add_(1, s["history"].long(), live.int())
        x = torch.where(n > 0, torch.where(x > 0, x / rates["repetition"], x * rates["repetition"]), x)
        x = x - n.float() * rates["frequency"]
        x = torch.where(n > 0, x - rates["presence"], x)
    if c["bias"]:
        x = x + _rows(s["bias"], R)
    x = x * rates["inv_temperature"]
    if c["mask"]:
        allowed = _allowed(s["mask"], V)
        if allowed.shape[0] > x.shape[0]:
            x = _rows(x, allowed.shape[0])
        x = torch.where(_rows(allowed, x.shape[0]), x, float("-inf"))
    out = {"logits": x.to(DTYPES[c["out"]])} if c["out"] else {}
    if c["choice"]:
        if c["noise"] and c["distinct"] in (1, R):
            x = x + s["noise"]
        elif c["noise"]:
            x = (x.unsqueeze(0) + s["noise"].view(-1, c["distinct"], V)).view(R, V)
        out["choice"] = _pick(x, DTYPES[c["choice"]])
    return out


def _teacher(ids, teacher, allowed, V, wide):
    """The teacher's probabilities, zero where an entry does not count, and the ids kept in range."""
    ids = ids.long()
    at = ids.clamp(0, V - 1)
    t = teacher.to(wide).expand(ids.shape)
    valid = (ids >= 0) & (ids < V) & (t > float("-inf"))
    if allowed is not None:
        valid &= allowed.expand(ids.shape[0], V).gather(1, at)
    t = torch.where(valid, t, float("-inf"))
    has = valid.any(-1, keepdim=True)
    e = torch.exp(t - torch.where(has, t.amax(-1, keepdim=True), 0.0))
    return at, e / torch.where(has, e.sum(-1, keepdim=True), 1.0), has


def _statistics(x, tau):
    """Each row's greatest entry and the sum of exponentials below it (-inf and 0 where every entry is masked)."""
    m = x.amax(-1, keepdim=True)
    return m, torch.exp((x - torch.where(m > float("-inf"), m, 0.0)) / tau).sum(-1, keepdim=True)


def _plain_distill(s):
    c = s["c"]
    V, tau = c["V"], c["tau"]
    x = s["logits"].float()
    allowed = _allowed(s["mask"], V) if c["mask"] else None
    if allowed is not None:
        x = torch.where(allowed, x, float("-inf"))
    at, p, has = _teacher(s["ids"], s["teacher"] / tau, allowed, V, torch.float32)
    if c["op"] == "backward":
        m, total = s["stats"][:, :1], s["stats"][:, 1:]
    else:
        m, total = _statistics(x, tau)
    out = {}
    if c["op"] != "backward":
        away = torch.where(p > 0, torch.log(total) - (x.gather(1, at) - m) / tau, 0.0)
        out["loss"] = tau * tau * (p * away).sum(-1)
    if c["op"] == "forward":
        out["stats"] = torch.cat([m, total], 1)
    else:
        q = torch.exp((x - m) / tau) / total
        g = (tau * s["scale"]).unsqueeze(-1) * q.scatter_add_(1, at, -p)
        g = torch.where(has, g, 0.0)
        out["grad"] = (g if allowed is None else torch.where(allowed, g, 0.0)).to(s["logits"].dtype)
    return out


# ------------------------------------------------------------------------------ one pass


def run(state):
    s = state
    c = s["c"]
    if not own:
        return _plain_adjust(s) if c["op"] == "adjust" else _plain_distill(s)
    from paper_2607_12324_amd import emo
    if c["op"] == "adjust":
        emo.adjust_logits(s["logits"], rows=c["rows"], history=s["history"], lengths=s["lengths"], bias=s["bias"],
                          mask=s["mask"], noise=s["noise"], out=s["out"], choice=s["choice"], **s["rates"])
        out = {"logits": s["out"]} if c["out"] else {}
        return {**out, "choice": s["choice"]} if c["choice"] else out
    if c["op"] == "forward":
        emo.distill_forward(s["logits"], s["ids"], s["teacher"], c["tau"], mask=s["mask"], loss=s["loss"], stats=s["stats"])
        return {"loss": s["loss"], "stats": s["stats"]}
    if c["op"] == "backward":
        emo.distill_backward(s["logits"], s["stats"], s["ids"], s["teacher"], c["tau"], scale=s["scale"], mask=s["mask"],
                             grad=s["grad"])
        return {"grad": s["grad"]}
    emo.distill_step(s["logits"], s["ids"], s["teacher"], c["tau"], scale=s["scale"], mask=s["mask"], loss=s["loss"],
                     grad=s["grad"])
    return {"loss": s["loss"], "grad": s["grad"]}


def work(case):
    """Each input read once, each output written once; an entry costs a multiplication, a comparison and what its operands
    add, and in a softmax a subtraction, a multiplication, an exponential and a sum."""
    c = case
    R, V = c["rows"], c["V"]
    entries = R * V
    words = (V + 31) // 32 * 4 * c["mask"]
    if c["op"] == "adjust":
        read = c["distinct"] * V * SIZES[c["dtype"]] + words + 4 * V * (c["noise"] + c["bias"]) + R * c["L"] // 2 * SIZES[c["ids"]]
        wrote = (entries * SIZES[c["out"]] if c["out"] else 0) + (R * SIZES[c["choice"]] if c["choice"] else 0)
        return {"bytes": read + wrote, "flops": entries * (2 + bool(c["noise"]) + bool(c["bias"]) + 4 * bool(c["L"]))}
    read = entries * SIZES[c["dtype"]] + words + R * c["K"] * SIZES[c["ids"]] + (1 if c["elites"] else R) * c["K"] * 4
    wrote = (12 * R if c["op"] == "forward" else entries * SIZES[c["dtype"]] + 4 * R)
    return {"bytes": read + wrote, "flops": entries * {"forward": 5, "backward": 5, "step": 7}[c["op"]]}


# ------------------------------------------------------------------------------ exact results


def _blocks(s, wide):
    """Blocks of rows of the distillation's inputs: first row, count, masked logits, allowed entries."""
    c = s["c"]
    V = c["V"]
    step = max(1, (1 << 25) // V)
    for r in range(0, c["rows"], step):
        n = min(step, c["rows"] - r)
        x = s["logits"][r:r + n].to(wide)
        allowed = None
        if c["mask"]:
            allowed = _allowed(s["mask"] if c["mask"] == 1 else s["mask"][r:r + n], V)
            x = torch.where(allowed, x, float("-inf"))
        yield r, n, x, allowed


def _exact_adjust(s):
    """Entry by entry in fp64, a block of rows at a time; the choice is a whole number and has no such value."""
    c = s["c"]
    R, V = c["rows"], c["V"]
    if not c["out"]:
        return None
    y = torch.empty((R, V), dtype=torch.float64, device="cuda")
    for r in range(R):
        x = s["logits"][r % c["distinct"]].double()
        rate = {k: float(t[r % t.shape[0]]) for k, t in s["rates"].items()}
        if c["L"]:
            n = torch.bincount(s["history"][r, :int(s["lengths"][r])].long(), minlength=V).double()
            seen = n > 0
            x = torch.where(seen & (x > 0), x / rate["repetition"], torch.where(seen, x * rate["repetition"], x))
            x = x - n * rate["frequency"] - seen.double() * rate["presence"]
        if c["bias"]:
            x = x + s["bias"][r % c["bias"]].double()
        x = x * rate["inv_temperature"]
        if c["mask"]:
            x[~_allowed(s["mask"][r % c["mask"]][None], V)[0]] = float("-inf")
        y[r] = x
    return {"logits": y, "choice": None} if c["choice"] else {"logits": y}


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["op"] == "adjust":
        return _exact_adjust(s)
    R, V, K, tau = c["rows"], c["V"], c["K"], c["tau"]
    loss = torch.zeros(R, dtype=torch.float64, device="cuda")
    stats = torch.empty((R, 2), dtype=torch.float64, device="cuda")
    grad = torch.empty((R, V), dtype=torch.float64, device="cuda") if c["op"] != "forward" else None
    if c["op"] == "backward":
        # the statistics are inputs here, as kept: fp32 roundings of the exact ones
        kept = prepare(case, seed)["stats"].double()
    for r, n, x, allowed in _blocks(s, torch.float64):
        ids = s["ids"][r:r + n].long()
        t = (s["teacher"] if s["teacher"].shape[0] == 1 else s["teacher"][r:r + n]).double().expand(n, K) / tau
        # the teacher's weight of each entry: its exponentials summed where its ids point, over their sum
        ok = ids >= 0
        if allowed is not None:
            ok = ok & allowed.expand(n, V).gather(1, ids.clamp(min=0))
        w = torch.exp(t - t.amax(-1, keepdim=True)) * ok
        weight = torch.zeros((n, V), dtype=torch.float64, device="cuda").scatter_add_(1, ids.clamp(min=0), w)
        mass = weight.sum(-1, keepdim=True)
        taught = mass > 0
        weight = weight / torch.where(taught, mass, 1.0)
        if c["op"] == "backward":
            m, total = kept[r:r + n, :1], kept[r:r + n, 1:]
            logq = (x - m) / tau - total.log()
        else:
            lse = torch.logsumexp(x / tau, -1, keepdim=True)
            stats[r:r + n, :1] = x.amax(-1, keepdim=True)
            empty = stats[r:r + n, :1] == float("-inf")
            stats[r:r + n, 1:] = torch.where(empty, 0.0, torch.exp(lse - stats[r:r + n, :1] / tau))
            logq = x / tau - lse
        loss[r:r + n] = -tau * tau * torch.where(weight > 0, weight * logq, 0.0).sum(-1)
        if grad is not None:
            rate = s["scale"].double()[r:r + n] if s["scale"].shape[0] > 1 else s["scale"].double()
            g = tau * rate.unsqueeze(-1) * (logq.exp() - weight)
            g = torch.where(taught, g, 0.0)
            grad[r:r + n] = g if allowed is None else torch.where(allowed, g, 0.0)
    if c["op"] == "forward":
        return {"loss": loss, "stats": stats}
    return {"grad": grad} if c["op"] == "backward" else {"loss": loss, "grad": grad}
