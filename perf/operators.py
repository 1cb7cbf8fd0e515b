"""Timed cases of the stand-alone operators around an exit head: group norm with an activation on a feature map, a projection
shared by many requests with a low-rank adapter of each request's own, class probabilities, and the verification of the
classes (tokens) that an early exit drafted against the probabilities of a later one.

A case is one call, described by a dict of plain values.  ``run`` computes it in elementary torch operations, or, where
``own`` is true, through the library's entry points.  ``exact`` is the definition in 64 bits.
"""
import torch

own = False

_ACTS = {"none": 0, "relu": 1, "relu6": 2, "silu": 3}
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _norm(name, batch, h, w, c, groups, act, dtype="bf16", residual=False):
    return {"name": name, "op": "norm", "batch": batch, "h": h, "w": w, "c": c, "groups": groups, "act": act, "dtype": dtype, "residual": residual}


def _linear(name, rows, c, n, rank, adapters, order, dtype="bf16", bias=True):
    return {"name": name, "op": "linear", "rows": rows, "c": c, "n": n, "rank": rank, "adapters": adapters, "order": order, "dtype": dtype, "bias": bias}


def _softmax(name, rows, n, dtype, masked=0.0, temperature=False):
    return {"name": name, "op": "softmax", "rows": rows, "n": n, "dtype": dtype, "masked": masked, "temperature": temperature}


def _verify(name, batch, k, n, dense=True, ragged=False):
    return {"name": name, "op": "verify", "batch": batch, "k": k, "n": n, "dense": dense, "ragged": ragged}


def listed():
    return [
        # one request's last feature map of the ResNet-50-shaped network: nothing but latency
        _norm("norm b1 7x7x2048", 1, 7, 7, 2048, 32, "relu"),
        # the end of a bottleneck block at the benchmark's batch: the shortcut is added before the activation
        _norm("norm b64 56x56x256 residual", 64, 56, 56, 256, 32, "relu", residual=True),
        # an expanded map of the MobileNetV2-shaped network: 12 channels a group, which no 16-byte vector divides
        _norm("norm b32 112x112x96 g8", 32, 112, 112, 96, 8, "silu"),
        # the fp32 model on odd maps, a ragged batch, three channels a group
        _norm("norm b13 33x29x96 f32", 13, 33, 29, 96, 32, "silu", dtype="f32"),
        # one request through a personal head on 2048 pooled channels and 1000 classes
        _linear("linear 1x2048x1000 r8", 1, 2048, 1000, 8, 16, "mixed"),
        # a full serving batch, one row a request, every request with an adapter of its own
        _linear("linear 64x4096x4096 r16 mixed", 64, 4096, 4096, 16, 32, "mixed"),
        # whole sequences packed behind one another, each with its adapter: the largest product
        _linear("linear 4096x4096x4096 r64 runs", 4096, 4096, 4096, 64, 9, "runs"),
        # the fp32 model's head at a ragged batch and an odd rank
        _linear("linear 37x2048x1000 r5 f32", 37, 2048, 1000, 5, 7, "mixed", dtype="f32"),
        # the exit head's logits at the benchmark's batch
        _softmax("softmax 64x1000 f32", 64, 1000, "f32"),
        # five positions of 64 sequences over a large vocabulary, some entries masked, a temperature for each row
        _softmax("softmax 320x128001 bf16", 320, 128001, "bf16", masked=0.2, temperature=True),
        # one request, one answer of an early exit against the final one over 1000 classes
        _verify("verify b1 k1 n1000", 1, 1, 1000),
        # 64 sequences with up to five drafted tokens each over a large vocabulary
        _verify("verify b64 k5 n128001 ragged", 64, 5, 128001, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    r = rng.random()
    if r < 0.33:
        cpg, groups = rng.choice([1, 2, 3, 4, 6, 8, 12, 16, 32, 64, rng.randint(1, 40)]), rng.choice([1, 4, 8, 16, 32, 32, rng.randint(1, 40)])
        c = min(2048, cpg * groups) // groups * groups
        dtype, residual = rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.3
        h, w = _log_int(rng, 4, 112), _log_int(rng, 4, 112)
        most = 64 * 56 * 56 * 256 * 6 // ((2 if dtype == "bf16" else 4) * (3 if residual else 2))    # elements of the largest listed case's bytes
        batch = min(_log_int(rng, 1, 64), max(1, most // (h * w * c)))
        case = _norm("", batch, h, w, c, groups, rng.choice(list(_ACTS)), dtype, residual)
    elif r < 0.66:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rows = _log_int(rng, 1, 4096 if dtype == "bf16" else 256)
        case = _linear("", rows, _log_int(rng, 32, 512) * 8 if rng.random() < 0.7 else _log_int(rng, 64, 4096), _log_int(rng, 10, 4096),
                       rng.choice([4, 8, 16, 32, 64, rng.randint(1, 64)]), _log_int(rng, 1, 32), rng.choice(["mixed", "runs"]), dtype, rng.random() < 0.5)
    elif r < 0.83:
        n = _log_int(rng, 10, 128001)
        case = _softmax("", min(_log_int(rng, 1, 2048), 320 * 128001 // n), n, rng.choice(["bf16", "f32"]) if n < 64000 else "bf16",
                        rng.choice([0.0, 0.2, 0.9]), rng.random() < 0.5)
    else:
        n, k = _log_int(rng, 10, 128001), rng.randint(1, 8)
        case = _verify("", max(1, min(_log_int(rng, 1, 256), 64 * 6 * 128001 // (n * (k + 1)))), k, n, rng.random() < 0.7, rng.random() < 0.5)
    case.pop("name")
    return case


# ----------------------------------------------------------------------------- states

def _distributions(gen, shape, spread):
    """Two related sets of rows of probabilities, as an early and a later exit give them: (later, early)."""
    base = torch.randn(shape, generator=gen, device="cuda") * 2.5
    early = torch.softmax(base[:, :-1] + spread * torch.randn(base[:, :-1].shape, generator=gen, device="cuda"), -1)
    return torch.softmax(base, -1), early


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def integers(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=gen, device="cuda")

    st = dict(case)
    if case["op"] == "norm":
        td, c, shape = _TYPES[case["dtype"]], case["c"], (case["batch"], case["h"], case["w"], case["c"])
        # what a convolution leaves: channels of their own scale and offset
        st.update(x=(normal(*shape) * (0.5 + normal(c).abs()) + 1.5 * normal(c)).to(td), gamma=1 + 0.2 * normal(c), beta=0.1 * normal(c), eps=1e-5,
                  shortcut=normal(*shape).to(td) if case["residual"] else None, out=torch.empty(shape, dtype=td, device="cuda"))
    elif case["op"] == "linear":
        td, t, c, n, r, m = _TYPES[case["dtype"]], case["rows"], case["c"], case["n"], case["rank"], case["adapters"]
        if case["order"] == "mixed":
            which = integers(0, m + 1, t) - 1       # -1: a row without an adapter
        else:
            which = torch.sort(integers(0, m, t))[0]    # rows of a sequence stand together ...
            which = torch.cat([integers(-1, m, m), integers(0, m, 1)])[which]    # ... and adapters come in any order, or not at all
        st.update(x=normal(t, c).to(td), weight=(normal(n, c) * c ** -0.5).to(td), bias_of=0.1 * normal(n) if case["bias"] else None,
                  a=(normal(m, r, c) * c ** -0.5).to(td), b=(normal(m, n, r) * (0.5 * r ** -0.5)).to(td), scale=0.5 + 1.5 * torch.rand(m, generator=gen, device="cuda"),
                  which=which.int(), out=torch.empty((t, n), dtype=td, device="cuda"),
                  scratch=torch.empty(32 * t * r + 256, dtype=torch.uint8, device="cuda"))     # up to eight partial sums of the narrow product
    elif case["op"] == "softmax":
        t, n = case["rows"], case["n"]
        x = normal(t, n) * 3
        if case["masked"]:
            x.masked_fill_(torch.rand((t, n), generator=gen, device="cuda") < case["masked"], float("-inf"))
        st.update(x=x.to(_TYPES[case["dtype"]]), out=torch.empty((t, n), dtype=torch.float32, device="cuda"),
                  heat=0.5 + torch.rand(t, generator=gen, device="cuda") if case["temperature"] else None)
    else:
        b, k, n = case["batch"], case["k"], case["n"]
        p, q = _distributions(gen, (b, k + 1, n), 0.7)
        drafts = torch.multinomial(q.view(b * k, n), 1, generator=gen).view(b, k)
        st.update(p=p, q=q if case["dense"] else None, drafts=drafts.int(), u=torch.rand((b, k), generator=gen, device="cuda"),
                  r=torch.rand(b, generator=gen, device="cuda"), count=integers(0, k + 1, b).int() if case["ragged"] else None,
                  tokens=torch.empty((b, k + 1), dtype=torch.int32, device="cuda"), accepted=torch.empty(b, dtype=torch.int32, device="cuda"))
    return st


# ----------------------------------------------------------------------------- plain forms

def _act(y, act):
    if act == "relu":
        return torch.clamp(y, min=0)
    if act == "relu6":
        return torch.clamp(y, 0, 6)
    return y / (1 + torch.exp(-y)) if act == "silu" else y


def _plain_norm(st):
    x = st["x"].float()
    b, h, w, c = x.shape
    g = x.view(b, h * w, st["groups"], c // st["groups"])
    d = g - g.mean((1, 3), keepdim=True)
    y = d * torch.rsqrt((d * d).mean((1, 3), keepdim=True) + st["eps"])
    y = y.view(b, h, w, c) * st["gamma"] + st["beta"]
    if st["shortcut"] is not None:
        y = y + st["shortcut"].float()
    return _act(y, st["act"]).to(st["x"].dtype)


def _plain_linear(st):
    x, which = st["x"].float(), st["which"].long()
    t, m, r = st["rows"], st["adapters"], st["rank"]
    y = x @ st["weight"].float().t()
    if st["bias_of"] is not None:
        y = y + st["bias_of"]
    h = (x @ st["a"].float().view(m * r, -1).t()).view(t, m, r)
    mine = which[:, None] == torch.arange(m, device=x.device)      # a row of -1 has none
    h = torch.where(mine[:, :, None], h * st["scale"][None, :, None], torch.zeros((), device=x.device))
    y = y + h.view(t, m * r) @ st["b"].float().permute(0, 2, 1).reshape(m * r, -1)
    return y.to(st["x"].dtype)


def _plain_softmax(st):
    z = st["x"].float()
    if st["heat"] is not None:
        z = z / st["heat"][:, None]
    top = z.max(1, keepdim=True)[0]
    e = torch.exp(z - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    s = e.sum(1, keepdim=True)
    return e / torch.where(s == 0, torch.ones_like(s), s)      # a row with nothing left is all zero


def _plain_verify(st):
    p, q, drafts, u, r = st["p"], st["q"], st["drafts"].long(), st["u"], st["r"]
    b, k, n = drafts.shape[0], drafts.shape[1], p.shape[2]
    rows, at = torch.arange(b, device=p.device), torch.arange(k, device=p.device)
    count = torch.full((b,), k, device=p.device) if st["count"] is None else st["count"].long()
    pd = p[rows[:, None], at, drafts].double()
    qd = torch.ones_like(pd) if q is None else q[rows[:, None], at, drafts].double()
    ok = (u.double() * qd < pd) & (at < count[:, None])
    got = torch.cumprod(ok.long(), 1).sum(1)                         # drafts accepted before the first rejection
    w = p[rows, got].double()
    last = torch.clamp(got, max=k - 1)
    rejected = (got < count)[:, None]
    if q is None:
        less = torch.where(torch.arange(n, device=p.device) == drafts[rows, last][:, None], torch.zeros_like(w), w)
    else:
        less = torch.clamp(w - q[rows, last].double(), min=0)
    less = torch.where(rejected, less, w)
    w = torch.where(less.sum(1, keepdim=True) > 0, less, w)          # nothing left over: the target itself
    cum = torch.cumsum(w, 1)
    token = (cum <= r.double()[:, None] * cum[:, -1:]).sum(1)
    place = torch.arange(k + 1, device=p.device)
    padded = torch.cat([drafts, drafts[:, :1]], 1)
    tokens = torch.where(place < got[:, None], padded, torch.where(place == got[:, None], token[:, None], torch.full_like(padded, -1)))
    return {"tokens": tokens.int(), "accepted": got.int()}


# ----------------------------------------------------------------------------- one pass

def run(st):
    op = st["op"]
    if not own:
        return {"norm": _plain_norm, "linear": _plain_linear, "softmax": _plain_softmax, "verify": _plain_verify}[op](st)
    from paper_2209_13443_b200 import binding as eb

    if op == "norm":
        eb.group_norm(st["dtype"], st["x"], st["batch"], st["h"] * st["w"], st["c"], st["groups"], st["gamma"], st["beta"], st["eps"], _ACTS[st["act"]],
                      st["out"], residual=st["shortcut"])
        return st["out"]
    if op == "linear":
        eb.adapted_linear(st["dtype"], st["x"], st["rows"], st["c"], st["weight"], st["n"], st["a"], st["b"], st["rank"], st["adapters"], st["which"],
                          st["out"], st["scratch"], bias=st["bias_of"], scale=st["scale"])
        return st["out"]
    if op == "softmax":
        eb.softmax(st["dtype"], st["x"], st["rows"], st["n"], st["out"], temperature=st["heat"])
        return st["out"]
    eb.verify_drafts(st["p"], st["q"], st["drafts"], st["u"], st["r"], st["batch"], st["k"], st["n"], st["tokens"], st["accepted"], n_draft=st["count"])
    return {"tokens": st["tokens"], "accepted": st["accepted"]}


# ----------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        b, h, w, c, g = case["batch"], case["h"], case["w"], case["c"], case["groups"]
        y = torch.empty((b, h, w, c), dtype=torch.float64, device="cuda")
        for i in range(b):       # a sample at a time: mean and variance as moments of its groups
            x = st["x"][i].double().reshape(h * w, g, c // g).transpose(0, 1).reshape(g, -1)
            var, mean = torch.var_mean(x, 1, correction=0)
            z = ((x - mean[:, None]) / torch.sqrt(var + st["eps"])[:, None]).view(g, h * w, c // g).transpose(0, 1).reshape(h, w, c)
            y[i] = z * st["gamma"].double() + st["beta"].double() + (st["shortcut"][i].double() if case["residual"] else 0.0)
        return {"none": y, "relu": y.clamp(min=0), "relu6": y.clamp(0, 6), "silu": y * torch.sigmoid(y)}[case["act"]]
    if case["op"] == "linear":
        x = st["x"].double()
        y = x @ st["weight"].double().t() + (st["bias_of"].double() if case["bias"] else 0.0)
        for i in range(case["adapters"]):
            rows = (st["which"] == i).nonzero()[:, 0]
            y[rows] += float(st["scale"][i]) * ((x[rows] @ st["a"][i].double().t()) @ st["b"][i].double().t())
        return y
    if case["op"] == "softmax":
        y = torch.empty((case["rows"], case["n"]), dtype=torch.float64, device="cuda")
        for i in range(case["rows"]):
            z = st["x"][i].double() / (st["heat"][i].double() if case["temperature"] else 1.0)
            y[i] = torch.nan_to_num(torch.softmax(z, 0), nan=0.0)
        return y
    b, k, n = case["batch"], case["k"], case["n"]
    drafts, count = st["drafts"].tolist(), [k] * b if st["count"] is None else st["count"].tolist()
    u, r, tokens, accepted = st["u"].double().tolist(), st["r"].double().tolist(), [], []
    for i in range(b):           # the procedure as it is told, one sequence after the other
        said = []
        for j in range(count[i]):
            t = drafts[i][j]
            if u[i][j] * (1.0 if st["q"] is None else float(st["q"][i, j, t])) < float(st["p"][i, j, t]):
                said.append(t)
            else:
                break
        j = len(said)
        w = st["p"][i, j].double().cpu().numpy().copy()
        if j < count[i]:
            left = w.copy()
            if st["q"] is None:
                left[drafts[i][j]] = 0.0
            else:
                left = (left - st["q"][i, j].double().cpu().numpy()).clip(min=0.0)
            w = left if left.sum() > 0 else w
        cum = w.cumsum()
        accepted.append(j)
        tokens.append(said + [int(cum.searchsorted(r[i] * cum[-1], side="right"))] + [-1] * (k - j))
    return {"tokens": torch.tensor(tokens, dtype=torch.int32), "accepted": torch.tensor(accepted, dtype=torch.int32)}


# ----------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Inputs read once, outputs written once; of the probabilities the rows that a token is drawn from."""
    es = 2 if case.get("dtype") == "bf16" else 4
    if case["op"] == "norm":
        e = case["batch"] * case["h"] * case["w"] * case["c"]
        return {"bytes": (3 if case["residual"] else 2) * e * es + 8 * case["c"], "flops": 8.0 * e}
    if case["op"] == "linear":
        t, c, n, r = case["rows"], case["c"], case["n"], case["rank"]
        used = min(case["adapters"], t)
        return {"bytes": es * (t * (c + n) + n * c + used * r * (c + n)) + 4 * (n + t), "flops": 2.0 * t * (n * c + r * (c + n))}
    if case["op"] == "softmax":
        e = case["rows"] * case["n"]
        return {"bytes": (es + 4) * e, "flops": 4.0 * e}
    b, k, n = case["batch"], case["k"], case["n"]
    return {"bytes": 4 * b * ((2 if case["dense"] else 1) * n + 5 * k + 3), "flops": 3.0 * b * n}
