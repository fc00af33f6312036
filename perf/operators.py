"""Performance cases of the head's training operators: code length with its gradient, distillation from a teacher's
top logits with its gradient, and the selection of those top logits.

A case names the operator (``op``), the rows, channels and symbols of the head, the type of its operands and whether
the gradients are wanted:

  code_length  bits_r = (lse_r - z_r[symbol_r]) / ln 2 of the linear head z = h w + b, and lse_r; rows whose symbol
               is -1 are left out (all zero); with gradients those of sum_r weight_r bits_r for h, w and b
  distill      bits_r = sum_j q_rj log2(q_rj / p_r[index_rj]), q the softmax of the teacher's kept logits at the
               temperature, p the student's at the same; entries whose index is -1 are not there
  top          the k largest logits of each row, their indices (ties to the lowest) and the row's normaliser

``run`` computes the plain form in float32, or with ``own`` calls the framework; ``exact`` recomputes the results in
float64 from the definitions, a few rows at a time.
"""
import math

import torch

own = False
DEV = "cuda" if torch.cuda.is_available() else "cpu"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
LN2 = math.log(2.0)
MOST_PRODUCTS = 8192 * 2048 * 65536   # rows x channels x symbols of the largest listed case
MOST_LOGITS = 8192 * 65536


def _case(name, op, rows, symbols, *, channels=0, dtype="fp32", k=0, temperature=1.0, grad=False):
    c = dict(op=op, rows=rows, channels=channels, symbols=symbols, dtype=dtype, k=k, temperature=temperature, grad=grad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one coarse scale of the 16-beam 10-bit scan, 16 channels: launches and host calls count
        _case("bits 87 rows c16", "code_length", 87, 256, channels=16),
        # all model voxels of the 64-beam 14-bit scan, one training step of the 32-channel head
        _case("bits grad 14-bit c32", "code_length", 233737, 256, channels=32, grad=True),
        # the 12-bit scan under the widest predictor
        _case("bits grad 12-bit c128", "code_length", 58711, 256, channels=128, grad=True),
        # one symbol scored by a head over a large alphabet: the weights are read once
        _case("bits one row 65536", "code_length", 1, 65536, channels=2048, dtype="bf16"),
        # a training batch over a large alphabet
        _case("bits grad 8192 rows 65536", "code_length", 8192, 65536, channels=2048, dtype="bf16", grad=True),
        # a ragged batch: nothing is a multiple of a tile
        _case("bits grad 1021 rows 50021", "code_length", 1021, 50021, channels=1000, dtype="fp16", grad=True),
        # the 32-channel head fitted to the wide predictor's most likely codes
        _case("distill grad 12-bit c32", "distill", 58711, 256, channels=32, k=16, temperature=2.0, grad=True),
        # a batch over a large alphabet, the teacher's 64 best
        _case("distill grad 4096 rows", "distill", 4096, 32768, channels=1024, dtype="bf16", k=64, grad=True),
        # validation of a student in 32 bits, ragged
        _case("distill 517 rows 10007", "distill", 517, 10007, channels=384, k=20, temperature=1.5),
        # the teacher's side of the 14-bit scan
        _case("top 16 14-bit", "top", 233737, 256, k=16),
        # and over a large alphabet
        _case("top 64 4096 rows", "top", 4096, 32768, dtype="bf16", k=64),
        # one row, an odd alphabet
        _case("top 8 one row", "top", 1, 131071, k=8),
    ]


def draw(rng):
    """One more case of the same ranges: the framework's heads (16..128 channels, 16 or 256 symbols) over whole
    frames, and heads over alphabets up to 65536 symbols with 64..2048 channels."""

    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["code_length", "code_length", "distill", "distill", "top"])
    small = rng.random() < 0.5
    symbols = rng.choice([16, 256, 256]) if small else log_int(1000, 65536)
    if op == "top":
        rows = max(1, min(log_int(1, 233737 if small else 8192), MOST_LOGITS // symbols))
        return _case(None, op, rows, symbols, dtype=rng.choice(["fp32", "bf16", "fp16"]), k=rng.randint(1, min(64, symbols)))
    if small:
        channels, rows, dtype = rng.choice([16, 32, 32, 64, 128]), log_int(1, 233737), "fp32"
    else:
        channels, dtype = log_int(64, 2048), rng.choice(["bf16", "bf16", "fp16", "fp32"])
        rows = max(1, min(log_int(1, 8192), MOST_LOGITS // symbols, MOST_PRODUCTS // (symbols * channels)))
        if dtype == "fp32":
            rows = min(rows, 2048)
    k, temperature = 0, 1.0
    if op == "distill":
        k, temperature = rng.randint(1, min(64, symbols - 1)), rng.choice([1.0, 1.0, 1.5, 2.0, 4.0])
    return _case(None, op, rows, symbols, channels=channels, dtype=dtype, k=k, temperature=temperature,
                 grad=rng.random() < 0.6)


# ---- inputs ----

def prepare(case, seed):
    """Features after a ReLU and a Kaiming-normal head; half of the rows carry their symbol's weights, so that the
    head predicts them; one row in sixteen is left out, as the padding of a batch is."""
    g = torch.Generator(device=DEV).manual_seed(1000003 * int(seed) + 17)
    N, V, dt = case["rows"], case["symbols"], TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    if case["op"] == "top":
        return {"case": case, "logits": (normal(N, V) * 3).to(dt)}
    C = case["channels"]
    w = (normal(C, V) * math.sqrt(2.0 / C)).to(dt)
    symbol = torch.randint(0, V, (N,), generator=g, device=DEV)
    known = torch.rand(N, generator=g, device=DEV) < 0.5
    h = normal(N, C).relu() + known[:, None] * (0.5 * (math.log(V) + 2)) * w.float().t()[symbol]
    out = torch.rand(N, generator=g, device=DEV) < 1 / 16
    s = {"case": case, "h": h.to(dt), "w": w, "b": (normal(V) * 0.1).to(dt)}
    if case["grad"]:
        scale = 1024.0 if case["dtype"] == "fp16" else 1.0   # the loss scale that 16 bits of range ask for
        s["weight"] = (0.5 + torch.rand(N, generator=g, device=DEV)) * (scale / N)
    if case["op"] == "code_length":
        s["symbol"] = torch.where(out, -1, symbol).int()
        return s
    K = case["k"]
    step = torch.randint(1, max(2, (V - 1) // K + 1), (N,), generator=g, device=DEV)
    rank = torch.arange(K, device=DEV)
    index = (symbol[:, None] + step[:, None] * rank) % V
    kept = torch.where(out, torch.randint(0, K, (N,), generator=g, device=DEV), K)   # some rows keep fewer, or none
    s["index"] = torch.where(rank < kept[:, None], index, -1).int().contiguous()
    s["logit"] = (3 * normal(N, K)).sort(1, descending=True)[0].contiguous()
    return s


# ---- the operators in plain float32, and the framework's calls ----

def _ordered(x):
    """Integers in the order of the floats x."""
    bits = x.view(torch.int32)
    return torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()


def _plain_top(s):
    x, k = s["logits"].float(), s["case"]["k"]
    V = x.shape[1]
    key = _ordered(x) * (1 << 24) + (V - 1 - torch.arange(V, device=x.device))
    best = key.topk(k, 1)[0]
    index = V - 1 - (best & ((1 << 24) - 1))
    m = x.amax(1)
    return {"index": index.int(), "value": x.gather(1, index), "lse": m + (x - m[:, None]).exp().sum(1).log()}


def _plain_head(s):
    case = s["case"]
    T = case["temperature"]
    h, w, b = s["h"].float(), s["w"].float(), s["b"].float()
    z = (h @ w + b) / T
    m = z.amax(1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(1, keepdim=True)
    logp = z - m - total.log()
    if case["op"] == "code_length":
        there = (s["symbol"] >= 0)[:, None]
        index, q = s["symbol"].long().clamp(min=0)[:, None], there.float()
    else:
        there = s["index"] >= 0
        index = s["index"].long().clamp(min=0)
        t = torch.where(there, s["logit"] / T, -math.inf)
        t = (t - t.amax(1, keepdim=True).clamp(min=-3e38)).exp()
        q = t / t.sum(1, keepdim=True).clamp(min=1e-38)
    logq = torch.where(q > 0, q, 1.0).log()
    bits = torch.where(q > 0, q * (logq - logp.gather(1, index)), 0.0).sum(1) / LN2
    row = there.any(1)
    lse = torch.where(row, (m + total.log())[:, 0], 0.0)
    if not case["grad"]:
        return {"bits": bits, "lse": lse}
    dz = torch.where(row[:, None], e / total, 0.0).scatter_add(1, index, -q)
    dz = dz * (s["weight"] / (T * LN2))[:, None]
    x = torch.where(row[:, None], h, 0.0)
    dt = s["h"].dtype
    return {"bits": bits, "lse": lse, "dh": (dz @ w.t()).to(dt), "dw": (x.t() @ dz).to(dt), "db": dz.sum(0).to(dt)}


def run(s):
    case = s["case"]
    if not own:
        return _plain_top(s) if case["op"] == "top" else _plain_head(s)
    import paper_2503_12382_amd as reno
    if case["op"] == "top":
        r = reno.top_logits(s["logits"], case["k"])
        return {"index": r.index, "value": r.value, "lse": r.lse}
    if case["op"] == "code_length":
        r = reno.head_code_length(s["h"], s["w"], s["b"], s["symbol"], row_weight=s.get("weight"), grad=case["grad"])
    else:
        r = reno.head_distill(s["h"], s["w"], s["b"], s["index"], s["logit"], temperature=case["temperature"],
                              row_weight=s.get("weight"), grad=case["grad"])
    if not case["grad"]:
        return {"bits": r.bits, "lse": r.lse}
    return {"bits": r.bits, "lse": r.lse, "dh": r.dh, "dw": r.dw, "db": r.db}


def work(case):
    N, C, V, K = case["rows"], case["channels"], case["symbols"], case["k"]
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "top":
        return {"bytes": size * N * V + 8 * N * K + 4 * N, "flops": 0}
    operands = size * (N * C + C * V + V)
    rows = 8 * N + (4 * N if case["op"] == "code_length" else 8 * N * K)
    if case["grad"]:
        return {"bytes": 2 * operands + rows + 4 * N, "flops": 6.0 * N * C * V}
    return {"bytes": operands + rows, "flops": 2.0 * N * C * V}


# ---- the definitions in float64 ----

def exact(case, seed):
    s = prepare(case, seed)
    V = case["symbols"]
    if case["op"] == "top":
        k, parts = case["k"], []
        for x in s["logits"].split(max(1, (1 << 26) // V)):
            value, index = x.double().sort(dim=1, descending=True, stable=True)
            parts.append((index[:, :k].int(), value[:, :k], x.double().logsumexp(1)))
        index, value, lse = (torch.cat(p) for p in zip(*parts))
        return {"index": index, "value": value, "lse": lse}
    T, w, b = case["temperature"], s["w"].double(), s["b"].double()
    bits, lse, dh = [], [], []
    dw, db = torch.zeros_like(w), torch.zeros_like(b)
    step = max(1, (1 << 26) // V)
    for r0 in range(0, case["rows"], step):
        rows = slice(r0, min(case["rows"], r0 + step))
        h = s["h"][rows].double()
        z = torch.addmm(b, h, w) / T
        logp = torch.log_softmax(z, 1)
        target = torch.zeros_like(logp)
        if case["op"] == "code_length":
            here = torch.nonzero(s["symbol"][rows] >= 0).flatten()
            target[here, s["symbol"][rows][here].long()] = 1.0
        else:
            index = s["index"][rows].long()
            logit = (s["logit"][rows].double() / T).masked_fill(index < 0, -math.inf)
            q = torch.softmax(logit, 1).nan_to_num(0.0)   # a row without any entry has no distribution
            target.scatter_add_(1, index.clamp(min=0), q)
        bits.append((torch.xlogy(target, target) - torch.xlogy(target, logp.exp())).sum(1) / LN2)
        full = target.sum(1, keepdim=True) > 0
        lse.append(torch.logsumexp(z, 1) * full[:, 0])
        if case["grad"]:
            d = (logp.exp() - target) * full * (s["weight"][rows].double() / (T * LN2))[:, None]
            dh.append(d @ w.T)
            dw += (h * full).T @ d
            db += d.sum(0)
    out = {"bits": torch.cat(bits), "lse": torch.cat(lse)}
    return dict(out, dh=torch.cat(dh), dw=dw, db=db) if case["grad"] else out
