"""Timed cases of the stand-alone operators for answers in 8 bits and for answers that are drawn: rows of a feature map (or of any matrix) quantised
to 8-bit integers with a scale of each row's own, as a parked batch is kept; the same rows read back, in any order; a projection in 8-bit integers with a
scale for each row and each channel; and the draw of a class (token) from logits under a temperature, the k largest, the nucleus and the share of the best.

A case is one pass, described by a dict of plain values.  ``run`` computes it in elementary torch operations, or, where ``own`` is true, through the library's
entry points.  ``exact`` is the definition in 64 bits.
"""
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _park(name, rows, c, dtype="bf16"):
    return {"name": name, "op": "park", "rows": rows, "c": c, "dtype": dtype}


def _read(name, rows, c, pool, dtype="bf16"):
    return {"name": name, "op": "read", "rows": rows, "c": c, "pool": pool, "dtype": dtype}


def _linear(name, rows, c, n, dtype="bf16", given=False, bias=True):
    return {"name": name, "op": "linear", "rows": rows, "c": c, "n": n, "dtype": dtype, "given": given, "bias": bias}


def _sample(name, rows, n, dtype, filters, probs=False):
    return {"name": name, "op": "sample", "rows": rows, "n": n, "dtype": dtype, "filters": filters, "probs": probs}


def listed():
    return [
        # one preempted request's last feature map, put away and read back: nothing but latency
        _park("park 49x2048", 49, 2048),
        # a full batch behind the second stage of the ResNet-50-shaped network: 64 maps of 28 x 28 pixels
        _park("park 50176x512", 50176, 512),
        # the fp32 model on odd maps (13 samples of 33 x 29), an odd number of channels
        _park("park 12441x99 f32", 12441, 99, "f32"),
        # one request's map read back in front of its next stage
        _read("read 196x1024", 196, 1024, 196),
        # 64 requests' maps of 14 x 14 pixels from a pool of twice as many, in the order in which they are resumed
        _read("read 12544x1024 of 25088", 12544, 1024, 25088),
        # one request's pooled channels through a head of 1000 classes
        _linear("linear 1x2048x1000", 1, 2048, 1000),
        # a serving batch, one row a request
        _linear("linear 64x4096x4096", 64, 4096, 4096),
        # whole sequences packed behind one another: the largest product
        _linear("linear 4096x4096x4096", 4096, 4096, 4096),
        # the fp32 model, a ragged batch that was quantised before, odd sizes
        _linear("linear 37x2043x1001 f32", 37, 2043, 1001, "f32", given=True),
        # the exit head's logits of one request
        _sample("sample 1x1000 f32", 1, 1000, "f32", "kp"),
        # 64 sequences over a large vocabulary, every request with settings of its own
        _sample("sample 64x128001 bf16 mixed", 64, 128001, "bf16", "mixed"),
        # five positions of 64 sequences, with the probabilities that a verification goes by
        _sample("sample 320x128001 bf16 p probs", 320, 128001, "bf16", "p", probs=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    r = rng.random()
    if r < 0.3:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        c = _log_int(rng, 2, 256) * 8 if rng.random() < 0.6 else _log_int(rng, 16, 2048)
        rows = min(_log_int(rng, 1, 50176), 50176 * 512 // ((1 if dtype == "bf16" else 2) * c))
        case = _park("", rows, c, dtype) if r < 0.18 else _read("", rows, c, rows * rng.randint(1, 2), dtype)
    elif r < 0.65:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        c = _log_int(rng, 2, 256) * 16 if rng.random() < 0.6 else _log_int(rng, 32, 4096)
        case = _linear("", _log_int(rng, 1, 4096), c, _log_int(rng, 10, 4096), dtype, rng.random() < 0.4, rng.random() < 0.5)
    else:
        n = _log_int(rng, 10, 128001)
        dtype = rng.choice(["bf16", "f32"])
        case = _sample("", min(_log_int(rng, 1, 320), max(1, 160 * 128001 // n)), n, dtype, rng.choice(["none", "k", "p", "m", "kp", "mixed", "mixed"]), rng.random() < 0.4)
    case.pop("name")
    return case


# ----------------------------------------------------------------------------- states

def _pitch(c):
    return (c + 15) // 16 * 16     # bytes of a quantised row


def _padded(q):
    out = torch.zeros((q.shape[0], _pitch(q.shape[1])), dtype=torch.int8, device=q.device)
    out[:, :q.shape[1]] = q
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    def integers(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=gen, device="cuda")

    st = dict(case)
    rows = case["rows"]
    if case["op"] in ("park", "read"):
        td, c = _TYPES[case["dtype"]], case["c"]
        count = rows if case["op"] == "park" else case["pool"]
        # a map behind its ReLU: channels of their own scale and offset
        x = (normal(count, c) * (0.5 + normal(c).abs()) + 0.5 * normal(c)).clamp(min=0).to(td)
        st.update(out=torch.empty((rows, c), dtype=td, device="cuda"))
        if case["op"] == "park":
            st.update(x=x, q=torch.empty((rows, _pitch(c)), dtype=torch.int8, device="cuda"), scale=torch.empty(rows, dtype=torch.float32, device="cuda"))
        else:
            q, scale = _quantised(x)
            st.update(q=_padded(q), scale=scale, index=torch.randperm(count, generator=gen, device="cuda")[:rows].int())
    elif case["op"] == "linear":
        td, c, n = _TYPES[case["dtype"]], case["c"], case["n"]
        x = normal(rows, c)
        x[:, integers(0, c, max(1, c // 256))] *= 8     # a few channels are far larger than the others
        w, w_scale = _quantised(normal(n, c) * c ** -0.5)
        st.update(w=_padded(w), w_scale=w_scale, bias_of=0.1 * normal(n) if case["bias"] else None, x_scale=None, room=None, out=torch.empty((rows, n), dtype=td, device="cuda"))
        if case["given"]:
            q, st["x_scale"] = _quantised(x.to(td))
            st["x"] = _padded(q)
        else:
            st.update(x=x.to(td), room=torch.empty(rows * (_pitch(c) + 4) + 512, dtype=torch.uint8, device="cuda"))
    else:
        n, f = case["n"], case["filters"]
        heat, k = 0.6 + 0.8 * uniform(rows), torch.clamp(integers(1, 101, rows), max=n)
        p, m = 0.8 + 0.19 * uniform(rows), 0.02 + 0.1 * uniform(rows)
        if f == "mixed":                                # a setting that a request does not make is the one that changes nothing
            heat = torch.where(uniform(rows) < 0.1, torch.zeros_like(heat), heat)       # 0: the best
            k = torch.where(uniform(rows) < 0.5, k, torch.zeros_like(k))
            p = torch.where(uniform(rows) < 0.5, p, torch.ones_like(p))
            m = torch.where(uniform(rows) < 0.3, m, torch.zeros_like(m))
        st.update(x=(normal(rows, n) * 3).to(_TYPES[case["dtype"]]), heat=heat, k=k.int() if f in ("k", "kp", "mixed") else None, p=p if f in ("p", "kp", "mixed") else None,
                  m=m if f in ("m", "mixed") else None, u=uniform(rows), tokens=torch.empty(rows, dtype=torch.int32, device="cuda"),
                  out=torch.empty((rows, n), dtype=torch.float32, device="cuda") if case["probs"] else None)
    return st


# ----------------------------------------------------------------------------- plain forms

def _quantised(x):
    """Rows as integers and scales.  The quotient in 64 bits, where it lies next to the middle of two integers only if it is the middle."""
    scale = x.float().abs().amax(1) / 127
    return torch.round(x.double() / torch.where(scale == 0, torch.ones_like(scale), scale).double()[:, None]).to(torch.int8), scale


def _plain_park(st):
    q, scale = _quantised(st["x"])
    return {"values": (q.float() * scale[:, None]).to(st["x"].dtype), "scale": scale}


def _plain_read(st):
    at = st["index"].long()
    return (st["q"][at, :st["c"]].float() * st["scale"][at][:, None]).to(st["out"].dtype)


def _plain_linear(st):
    if st["given"]:
        q, scale = st["x"][:, :st["c"]], st["x_scale"]
    else:
        q, scale = _quantised(st["x"])
    y = (q.float() @ st["w"][:, :st["c"]].float().t()) * st["w_scale"] * scale[:, None]
    if st["bias_of"] is not None:
        y = y + st["bias_of"]
    return y.to(st["out"].dtype)


def _plain_sample(st):
    x, n = st["x"].double(), st["n"]
    order = torch.sort(x, dim=1, descending=True, stable=True)[1]
    z = torch.gather(x, 1, order)
    heat = st["heat"].double()[:, None]
    cold = ~(heat > 0)
    w = torch.exp((z - z[:, :1]) / torch.where(cold, torch.ones_like(heat), heat))
    place = torch.arange(n, device=x.device)
    keep = torch.ones_like(w, dtype=torch.bool)
    if st["k"] is not None:
        k = st["k"].long()[:, None]
        keep = keep & ((place < k) | (k <= 0))
    if st["p"] is not None:
        v = torch.where(keep, w, torch.zeros_like(w))
        before = torch.cumsum(v, 1) - v
        keep = keep & ((before < st["p"].double()[:, None] * v.sum(1, keepdim=True)) | (st["p"][:, None] >= 1))
    if st["m"] is not None:
        keep = keep & (w >= st["m"].double()[:, None])
    keep = torch.where(cold, place < 1, keep | (place < 1))
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, torch.zeros_like(w)))      # in the order of the classes
    cum = torch.cumsum(w, 1)
    token = (cum <= st["u"].double()[:, None] * cum[:, -1:]).sum(1).int()
    return {"tokens": token, "probs": (w / cum[:, -1:]).float()} if st["probs"] else {"tokens": token}


# ----------------------------------------------------------------------------- one pass

def run(st):
    op = st["op"]
    if not own:
        return {"park": _plain_park, "read": _plain_read, "linear": _plain_linear, "sample": _plain_sample}[op](st)
    from paper_2209_13443_b200 import binding as eb

    if op == "park":
        eb.quantize_rows(st["dtype"], st["x"], st["rows"], st["c"], st["q"], st["scale"])
        eb.dequantize_rows(st["dtype"], st["q"], st["scale"], st["rows"], st["c"], st["out"], st["rows"])
        return {"values": st["out"], "scale": st["scale"]}
    if op == "read":
        eb.dequantize_rows(st["dtype"], st["q"], st["scale"], st["pool"], st["c"], st["out"], st["rows"], index=st["index"])
        return st["out"]
    if op == "linear":
        eb.int8_linear(st["dtype"], st["x"], st["rows"], st["c"], st["w"], st["w_scale"], st["n"], st["out"], workspace=st["room"], x_scale=st["x_scale"], bias=st["bias_of"])
        return st["out"]
    eb.sample(st["dtype"], st["x"], st["rows"], st["n"], st["u"], st["tokens"], temperature=st["heat"], top_k=st["k"], top_p=st["p"], min_p=st["m"], probs=st["out"])
    return {"tokens": st["tokens"], "probs": st["out"]} if st["probs"] else {"tokens": st["tokens"]}


# ----------------------------------------------------------------------------- the definitions in 64 bits

def _exact_integers(x):
    """(integers, scales) of rows: the integer nearest to x / scale, the even one of two, with scale the float nearest to the largest magnitude / 127."""
    scale = (x.double().abs().max(1)[0] / 127.0).float().double()
    ratio = x.double() / scale.clamp(min=1e-300)[:, None]
    low = torch.floor(ratio)
    rest = ratio - low
    up = (rest > 0.5) | ((rest == 0.5) & (torch.remainder(low, 2) == 1))
    return low + up.double(), scale


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "park":
        q, scale = _exact_integers(st["x"])
        return {"values": q * scale[:, None], "scale": scale}
    if case["op"] == "read":
        y = torch.empty((case["rows"], case["c"]), dtype=torch.float64, device="cuda")
        at = st["index"].long()
        for i in range(0, case["rows"], 4096):
            part = at[i:i + 4096]
            y[i:i + 4096] = st["q"].index_select(0, part)[:, :case["c"]].double() * st["scale"].index_select(0, part).double().unsqueeze(1)
        return y
    if case["op"] == "linear":
        if case["given"]:
            q, scale = st["x"][:, :case["c"]].double(), st["x_scale"].double()
        else:
            q, scale = _exact_integers(st["x"])
        w = st["w_scale"].double()[:, None] * st["w"][:, :case["c"]].double()
        return (scale[:, None] * q) @ w.t() + (st["bias_of"].double() if case["bias"] else 0.0)
    tokens, probs, n = [], [], case["n"]
    for i in range(case["rows"]):        # a row at a time, as the procedure is told
        x, t = st["x"][i].double(), float(st["heat"][i])
        best = int((x == x.max()).nonzero()[0, 0])
        if not t > 0:
            kept = torch.tensor([best], device="cuda")
        else:
            z, kept = torch.sort(x, descending=True, stable=True)
            if st["k"] is not None and 0 < int(st["k"][i]) < n:
                z, kept = z[:int(st["k"][i])], kept[:int(st["k"][i])]
            if st["p"] is not None and float(st["p"][i]) < 1:
                share = torch.softmax(z / t, 0)
                before = torch.cat([torch.zeros(1, dtype=torch.float64, device="cuda"), share.cumsum(0)[:-1]])
                count = max(1, int((before < float(st["p"][i])).sum()))
                z, kept = z[:count], kept[:count]
            if st["m"] is not None and float(st["m"][i]) > 0:
                count = max(1, int((torch.exp((z - z[0]) / t) >= float(st["m"][i])).sum()))
                kept = kept[:count]
        q = torch.zeros(n, dtype=torch.float64, device="cuda")
        q[kept] = torch.softmax(x[kept] / t, 0) if t > 0 else 1.0
        cum = q.cumsum(0)
        tokens.append(int(torch.searchsorted(cum, float(st["u"][i]) * cum[-1], right=True)))
        probs.append(q)
    tokens = torch.tensor(tokens, dtype=torch.int32)
    return {"tokens": tokens, "probs": torch.stack(probs)} if case["probs"] else {"tokens": tokens}


# ----------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Inputs read once, outputs written once; what is parked is written and read again."""
    es = 2 if case["dtype"] == "bf16" else 4
    rows = case["rows"]
    if case["op"] == "park":
        return {"bytes": rows * (case["c"] * (2 * es + 2) + 8), "flops": 4.0 * rows * case["c"]}
    if case["op"] == "read":
        return {"bytes": rows * (case["c"] * (es + 1) + 8), "flops": 1.0 * rows * case["c"]}
    if case["op"] == "linear":
        c, n = case["c"], case["n"]
        return {"bytes": rows * (c * (1 if case["given"] else es) + n * es) + n * (c + 8), "flops": 2.0 * rows * n * c}
    return {"bytes": rows * case["n"] * (es + (4 if case["probs"] else 0)) + 24 * rows, "flops": 3.0 * rows * case["n"]}
