"""Operators that a model has around its expert layers when it answers and when it is fine-tuned: what is timed, and what it has to give.

A case is one pass through one of

  "score"      the vocabulary head: log probabilities of given tokens, the entropy of each token's distribution, and its K likeliest
               alternatives with their log probabilities
  "policy"     log probabilities and entropies, and the gradients of hidden states and head for given gradients of both
  "grad_norm"  the norm of all gradients of a model together
  "grad_clip"  the same, and the gradients scaled to a largest norm
  "qk"         norms of every head's queries and keys, and the rotation by position
  "qk_train"   the same, and the gradients of queries, keys and the norms' weights

  score, policy: T tokens, d hidden size, V vocabulary, temperature, `masked` the share of tokens without a target (prompts, padding).
  grad_*: a model of `layers` expert layers (d, f, E) with vocabulary V; `norm` is what its gradients' norm comes to, 1.0 the largest.
  qk*: T tokens, Hq and Hk heads of D columns of which R are rotated, as neighbours (`pairs`) or as halves; `packed`: queries and keys
  are columns of one matrix with the values; positions up to `far`.

``own`` false: the operators in elementary torch operations, in 32 bits (in 64: angles, sums over all gradients, and the logits that say
which alternative is likelier); true: the library's own calls.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
MAX_NORM = 1.0
SPARE = 16
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# the largest listed training step (T V d), model and attention input bound what draw() may give
MAX_TVD = 8192 * 50304 * 2048
MAX_ELEMENTS = 620_000_000
MAX_QK = 8192 * 40 * 128


def _head(name, kind, T, d, V, K=0, temperature=1.0, masked=0.0):
    return {"name": name, "kind": kind, "T": T, "d": d, "V": V, "K": K, "temperature": temperature, "masked": masked}


def _grads(name, kind, layers, d, f, E, V, norm):
    return {"name": name, "kind": kind, "layers": layers, "d": d, "f": f, "E": E, "V": V, "norm": norm}


def _qk(name, kind, T, Hq, Hk, D, R, pairs=False, packed=True, far=4096):
    return {"name": name, "kind": kind, "T": T, "Hq": Hq, "Hk": Hk, "D": D, "R": R, "pairs": pairs, "packed": packed, "far": far}


def listed():
    return [
        # one decoding step of a single sequence that reports the token's log probability beside 20 alternatives: the head's weights are read once
        _head("score_1", "score", 1, 2048, 50304, K=20),
        # one decoding step of a batch of sequences, five alternatives each, odd vocabulary, at the temperature of the sampling
        _head("score_131", "score", 131, 4096, 32003, K=5, temperature=0.7),
        # what a teacher says of the answers behind prompts: 20 alternatives for every token of them
        _head("score_4099", "score", 4099, 2048, 50304, K=20, masked=0.25),
        # the tiny model that tests train: launches are what counts
        _head("policy_tiny", "policy", 256, 128, 1031),
        # a step of reinforcement learning on ragged answers, a good part of the tokens belongs to prompts, odd vocabulary
        _head("policy_masked_3001", "policy", 3001, 1024, 50257, masked=0.4),
        # the largest step: four sequences of 2048 tokens, at the temperature that they were sampled with
        _head("policy_8192", "policy", 8192, 2048, 50304, temperature=0.9),
        # the norm that a training log shows for the example's model: the smallest call, all latency
        _grads("grad_norm_tiny", "grad_norm", 1, 256, 128, 8, 515, 0.6),
        # a model of many small layers: more than a hundred tensors of very different sizes, odd vocabulary
        _grads("grad_clip_24_layers", "grad_clip", 24, 704, 256, 8, 32003, 3.7),
        # one layer of the headline's model with embedding and head: a few large tensors
        _grads("grad_clip_olmoe", "grad_clip", 1, 2048, 1024, 64, 50304, 12.0),
        # one decoding step of a batch of sequences, far into their context
        _qk("qk_decode_48", "qk", 48, 16, 16, 128, 128, far=1 << 20),
        # several prompts, grouped heads of an odd width of which half is rotated, neighbours as pairs
        _qk("qk_prompt_4001", "qk", 4001, 24, 8, 96, 48, pairs=True),
        # the training step of four sequences of 2048 tokens with grouped heads
        _qk("qk_train_8192", "qk_train", 8192, 32, 8, 128, 128, far=2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["score", "score", "score", "policy", "policy", "grad_norm", "grad_clip", "grad_clip", "qk", "qk_train"])
    while True:
        if kind in ("score", "policy"):
            c = {"kind": kind, "T": _log_int(rng, 1, 16384), "d": 64 * _log_int(rng, 1, 64), "V": _log_int(rng, 200, 200000), "K": 0,
                 "temperature": rng.choice([1.0, 1.0, 0.7, 1.3]), "masked": rng.choice([0.0, 0.0, 0.3, 0.8])}
            if kind == "score":
                c["K"] = rng.choice([0, _log_int(rng, 1, 64), _log_int(rng, 1, 64), 20])
            if c["T"] * c["V"] * c["d"] <= MAX_TVD and c["T"] * c["V"] <= 8192 * 131072:
                return c
        elif kind.startswith("grad"):
            c = {"kind": kind, "layers": _log_int(rng, 1, 48), "d": 8 * _log_int(rng, 4, 512), "f": 8 * _log_int(rng, 4, 256),
                 "E": _log_int(rng, 2, 128), "V": _log_int(rng, 200, 100000), "norm": round(math.exp(rng.uniform(math.log(0.3), math.log(60.0))), 3)}
            if sum(math.prod(shape) for shape, _ in _tensors(c)) <= MAX_ELEMENTS:
                return c
        else:
            D = rng.choice([64, 80, 96, 128, 128, 192, 256])
            c = {"kind": kind, "T": _log_int(rng, 1, 16384), "Hk": _log_int(rng, 1, 16), "D": D, "R": rng.choice([D, D, D // 32 * 16]),
                 "pairs": rng.random() < 0.4, "packed": rng.random() < 0.6, "far": rng.choice([4096, 131072, 1 << 20])}
            c["Hq"] = c["Hk"] * rng.choice([1, 1, 2, 3, 4, 8])
            if c["T"] * (c["Hq"] + c["Hk"]) * D <= MAX_QK:
                return c


def _tensors(c):
    """(shape, type) of a model's gradients: matrices in bfloat16, the norms' and routers' in 32 bits."""
    bf, f32 = torch.bfloat16, torch.float32
    d, f, E = c["d"], c["f"], c["E"]
    layer = [((d,), f32), ((E, d), f32), ((E, f, d), bf), ((E, f, d), bf), ((E, d, f), bf)]
    return [((c["V"], d), bf)] + layer * c["layers"] + [((d,), f32), ((c["V"], d), bf)]


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device=DEV, dtype=torch.float32)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(c, kept={})
    if c["kind"].startswith("grad"):
        todo = _tensors(c)
        n = sum(math.prod(shape) for shape, _ in todo)
        s["grads"] = []
        for shape, dtype in todo:
            # layers' gradients differ in size; what they come to together is about c["norm"]
            size = c["norm"] / math.sqrt(n) * float(torch.exp(0.5 * torch.randn(1, generator=gen, device=DEV)))
            g = torch.empty(shape, dtype=dtype, device=DEV)
            for part in g.view(-1).split(1 << 26):
                part.copy_(torch.randn(part.numel(), generator=gen, device=DEV).mul_(size))
            s["grads"].append(g)
        return s
    T = c["T"]
    if c["kind"].startswith("qk"):
        Hq, Hk, D, R = c["Hq"], c["Hk"], c["D"], c["R"]
        # heads differ in size, columns too
        make = lambda H: (_normal(gen, T, H, D) * torch.exp(0.5 * _normal(gen, H, D))).bfloat16()  # noqa: E731
        if c["packed"]:
            packed = torch.cat([make(Hq), make(Hk), make(Hk)], 1)
            s["q"], s["k"] = packed[:, :Hq], packed[:, Hq:Hq + Hk]
        else:
            s["q"], s["k"] = make(Hq), make(Hk)
        s["wq"], s["wk"] = 0.8 + 0.4 * _uniform(gen, D), 0.8 + 0.4 * _uniform(gen, D)
        # sequences begin anywhere; a token's position is the one before it plus one
        start = int(torch.randint(0, c["far"], (1,), generator=gen, device=DEV))
        s["pos"] = ((start + torch.arange(T, device=DEV)) % c["far"]).int()
        s["freq"] = (10000.0 ** (-torch.arange(0, R, 2, device=DEV, dtype=torch.float64) / max(R, 1))).float()
        if c["kind"] == "qk_train":
            s["dqo"], s["dko"] = _normal(gen, T, Hq, D).bfloat16(), _normal(gen, T, Hk, D).bfloat16()
        return s
    d, V = c["d"], c["V"]
    s["W"] = torch.empty(V, d, dtype=torch.bfloat16, device=DEV)
    for v in range(0, V, 16384):
        s["W"][v:v + 16384] = _normal(gen, min(16384, V - v), d).mul_(0.02)
    target = torch.randint(0, V, (T,), generator=gen, device=DEV, dtype=torch.int64)
    # a trained model is sure of some of its tokens and not of others: logits of 0 to 12 above the others'
    known = _uniform(gen, T, 1) * (12.0 / (0.02 * 0.02 * d))
    s["x"] = (_normal(gen, T, d) + known * s["W"][target].float()).bfloat16()
    # one in five tokens was sampled though others were likelier
    target = torch.where(_uniform(gen, T) < 0.2, torch.randint(0, V, (T,), generator=gen, device=DEV, dtype=torch.int64), target)
    live = _uniform(gen, T) >= c["masked"]
    live[0] = True
    s["target"] = torch.where(live, target, -100).int()
    if c["kind"] == "policy":
        # minus the advantage, and minus what entropy counts, over the number of tokens
        s["dlogp"] = _normal(gen, T) / T
        s["dentropy"] = -0.02 * (0.5 + _uniform(gen, T)) / T
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------------


def _flat(s):
    """Where the scaled gradients go: a program's flat buffers, one for each type, and the tensors in them."""
    k = s["kept"]
    if "flat" not in k:
        k["flat"] = {n: torch.empty(sum(g.numel() for g in s["grads"] if g.dtype == t), dtype=t, device=DEV) for n, t in TYPES.items()}
        at, k["parts"] = dict.fromkeys(TYPES, 0), []
        for g in s["grads"]:
            n = "bf16" if g.dtype == torch.bfloat16 else "f32"
            k["parts"].append(k["flat"][n][at[n]:at[n] + g.numel()].view(g.shape))
            at[n] += g.numel()
    return k["flat"], k["parts"]


def _plain_grads(s):
    total = torch.zeros((), dtype=torch.float64, device=DEV)
    for g in s["grads"]:
        x = g.float()
        total = total + (x * x).sum(dtype=torch.float64)
    norm = total.sqrt()
    out = {"norm": norm.float().view(1)}
    if s["kind"] == "grad_clip":
        scale = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0).float()
        flat, parts = _flat(s)
        for g, part in zip(s["grads"], parts):
            part.copy_(g.float() * scale)
        out.update(flat)
    return out


def _rotate(v, cos, sin, pairs, back=False):
    """The first columns of v, as many as there are angles twice, by these angles."""
    n = cos.shape[-1]
    if back:
        sin = -sin
    a, b = (v[..., 0:2 * n:2], v[..., 1:2 * n:2]) if pairs else (v[..., :n], v[..., n:2 * n])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([a, b], -1).flatten(-2) if pairs else torch.cat([a, b], -1)
    return torch.cat([turned, v[..., 2 * n:]], -1)


def _plain_qk(s):
    angle = s["pos"].double()[:, None, None] * s["freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    out = {}
    for n in "qk":
        x, w = s[n].float(), s["w" + n]
        rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        out[n] = _rotate(x * rstd * w, cos, sin, s["pairs"]).bfloat16()
        if s["kind"] == "qk_train":
            dy = _rotate(s["d" + n + "o"].float(), cos, sin, s["pairs"], back=True)
            g = dy * w
            out["d" + n] = (rstd * (g - x * ((g * x).mean(-1, keepdim=True) * rstd * rstd))).bfloat16()
            out["dw" + n] = (dy * x * rstd).sum((0, 1))
    return out


def _plain_head(s):
    # Entropies and losses near zero are differences of nearly equal numbers as they are usually written.  Here what they are made of is
    # positive: with o_j the distance of a logit from the largest, R the sum of exp(-o) over the others and Q that of o exp(-o),
    # the largest has log probability -log(1 + R), and the entropy is log(1 + R) + Q / (1 + R).
    T, V, K, tau = s["T"], s["V"], s["K"], s["temperature"]
    there = (s["target"] >= 0) & (s["target"] < V)
    y = torch.where(there, s["target"], 0).long()[:, None]
    x, W = s["x"].float(), s["W"].float()
    z = x @ W.t()
    top, best = z.max(1, keepdim=True)
    o = (top - z) / tau
    e = (-o).exp()
    e.scatter_(1, best, 0.0)
    R, Q = e.sum(1, keepdim=True), (e * o).sum(1, keepdim=True)
    log_top = -torch.log1p(R)
    entropy = -log_top + Q / (1.0 + R)
    logp = log_top - torch.where(y == best, 0.0, o.gather(1, y))
    keep = lambda v: torch.where(there, v[:, 0], 0.0)  # noqa: E731
    out = {"logp": keep(logp), "entropy": keep(entropy)}
    if K:
        # which of two logits is larger has to be told in 64 bits; of equal ones the lower column comes first
        near = z.topk(min(V, K + SPARE), 1).indices.sort(1).values
        z64, order = _gathered(s, near).sort(dim=1, descending=True, stable=True)
        ids = near.gather(1, order)[:, :K]
        behind = ((z64[:, :1] - z64[:, :K]) / tau).float()
        out["ids"] = torch.where(there[:, None], ids, -1).int()
        out["top"] = torch.where(there[:, None], log_top - behind, 0.0)
    if s["kind"] == "policy":
        a, b = torch.where(there, s["dlogp"], 0.0)[:, None] / tau, torch.where(there, s["dentropy"], 0.0)[:, None] / tau
        log_p = log_top - o
        dz = -log_p.exp() * (a + b * (log_p + entropy))
        dz.scatter_(1, y, -torch.expm1(logp) * a - b * logp.exp() * (logp + entropy))
        out["dx"], out["dW"] = (dz @ W).bfloat16(), (dz.t() @ x).bfloat16()
    return out


def _gathered(s, near):
    """Logits at some columns of each token, in 64 bits."""
    parts = []
    for rows in torch.arange(s["T"], device=DEV).split(max(1, (1 << 27) // (near.shape[1] * s["d"]))):
        parts.append((s["W"][near[rows]].double() * s["x"][rows].double()[:, None, :]).sum(2))
    return torch.cat(parts)


# ---- the library's calls -----------------------------------------------------------------------------------------------------


def _new(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device=DEV)


def _space(nbytes):
    return _new(max(nbytes, 256), dtype=torch.uint8)


def _own_grads(s, B):
    k = s["kept"]
    if "ws" not in k:
        k.update(norm=_new(1), ws=_space(B.moe_grad_norm_workspace_bytes(len(s["grads"]))))
    if s["kind"] == "grad_norm":
        B.moe_grad_norm(s["grads"], k["norm"], k["ws"])
        return {"norm": k["norm"]}
    flat, parts = _flat(s)
    B.moe_grad_clip(s["grads"], MAX_NORM, k["norm"], parts, k["ws"])
    return {"norm": k["norm"], **flat}


def _own_qk(s, B):
    k = s["kept"]
    bf, T, Hq, Hk, D = torch.bfloat16, s["T"], s["Hq"], s["Hk"], s["D"]
    if not k:
        k.update(q=_new(T, Hq, D, dtype=bf), k=_new(T, Hk, D, dtype=bf))
        if s["kind"] == "qk_train":
            k.update(dq=_new(T, Hq, D, dtype=bf), dk=_new(T, Hk, D, dtype=bf), dwq=_new(D), dwk=_new(D),
                     ws=_space(B.moe_qk_norm_rope_bwd_workspace_bytes(T, Hq, Hk, D)))
    given = (s["q"], s["k"], s["wq"], s["wk"], s["pos"], s["freq"], s["pairs"], EPS)
    B.moe_qk_norm_rope(*given, k["q"], k["k"])
    if s["kind"] == "qk_train":
        B.moe_qk_norm_rope_bwd(s["dqo"], s["dko"], *given, k["dq"], k["dk"], k["dwq"], k["dwk"], k["ws"])
    return {n: k[n] for n in ("q", "dq", "dwq", "k", "dk", "dwk") if n in k}


def _own_head(s, B):
    k = s["kept"]
    T, d, V, K, policy = s["T"], s["d"], s["V"], s["K"], s["kind"] == "policy"
    if not k:
        k.update(logp=_new(T), entropy=_new(T), lse=_new(T), ids=None, top=None)
        nbytes = B.moe_head_score_fwd_workspace_bytes(T, d, V, K)
        if K:
            k.update(ids=_new(T, K, dtype=torch.int32), top=_new(T, K))
        if policy:
            k.update(dx=_new(T, d, dtype=torch.bfloat16), dW=_new(V, d, dtype=torch.bfloat16))
            nbytes = max(nbytes, B.moe_head_score_bwd_workspace_bytes(T, d, V, 0))
        k["ws"] = _space(nbytes)
    given = (s["x"], s["W"], s["target"], s["temperature"])
    B.moe_head_score_fwd(*given, k["logp"], k["entropy"], k["lse"], k["ids"], k["top"], k["ws"])
    out = {"logp": k["logp"], "entropy": k["entropy"]}
    if K:
        out.update(ids=k["ids"], top=k["top"])
    if policy:
        B.moe_head_score_bwd(*given, k["logp"], k["entropy"], k["lse"], s["dlogp"], s["dentropy"], 0, k["dx"], k["dW"], k["ws"])
        out.update(dx=k["dx"], dW=k["dW"])
    return out


def run(s):
    if own:
        from paper_2604_00785_amd import binding as B

        return _own_grads(s, B) if s["kind"].startswith("grad") else _own_qk(s, B) if s["kind"].startswith("qk") else _own_head(s, B)
    return _plain_grads(s) if s["kind"].startswith("grad") else _plain_qk(s) if s["kind"].startswith("qk") else _plain_head(s)


# ---- what a pass cannot do without, and its results in 64 bits -----------------------------------------------------------------


def work(case):
    c = case
    if c["kind"].startswith("grad"):
        sizes = [(math.prod(shape), 2 if dtype == torch.bfloat16 else 4) for shape, dtype in _tensors(c)]
        n, nbytes, clip = sum(k for k, _ in sizes), sum(k * b for k, b in sizes), c["kind"] == "grad_clip"
        return {"bytes": 4.0 + nbytes * (2.0 if clip else 1.0), "flops": n * (3.0 if clip else 2.0)}
    T = c["T"]
    if c["kind"].startswith("qk"):
        n, train = T * (c["Hq"] + c["Hk"]) * c["D"], c["kind"] == "qk_train"
        # read and written; backward: the outputs' gradients, the inputs' and the weights'
        return {"bytes": 4.0 * n + 4.0 * T + 8.0 * c["D"] + 2.0 * c["R"] + (4.0 * n + 8.0 * c["D"] if train else 0.0), "flops": n * (18.0 if train else 7.0)}
    V, d, K, live = c["V"], c["d"], c["K"], T * (1.0 - c["masked"])
    nbytes = 2.0 * V * d + 2.0 * live * d + 12.0 * T + 8.0 * T * K
    flops = 2.0 * live * V * d
    if c["kind"] == "policy":
        nbytes += 2.0 * V * d + 2.0 * T * d + 8.0 * T
        flops *= 3.0                                                     # logits once, and the two products of the backward pass
    return {"bytes": nbytes, "flops": flops}


def exact(case, seed):
    s = prepare(case, seed)
    kind, f64 = case["kind"], torch.float64
    if kind.startswith("grad"):
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.view(-1), dtype=f64) for g in s["grads"]]))
        out = {"norm": norm.view(1)}
        if kind == "grad_clip":
            scale = min(1.0, MAX_NORM / (float(norm) + 1e-6))
            for n, t in TYPES.items():
                out[n] = torch.cat([g.view(-1) for g in s["grads"] if g.dtype == t]).to(f64).mul_(scale)
        return out
    if kind.startswith("qk"):
        R, D = case["R"], case["D"]
        # the rotation as a matrix of a token, by which the rows are multiplied
        i = torch.arange(R // 2, device=DEV)
        one, two = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + R // 2)
        out = {}
        for n in "qk":
            x, w = s[n].to(f64), s["w" + n].to(f64)
            unit = x / (torch.linalg.vector_norm(x, dim=2, keepdim=True).square().div(D).add(EPS)).sqrt()
            y, back = torch.empty_like(x), torch.empty_like(x)
            dy = s["d" + n + "o"].to(f64) if kind == "qk_train" else None
            for rows in torch.arange(case["T"], device=DEV).split(2048):
                turn = torch.eye(D, dtype=f64, device=DEV).repeat(len(rows), 1, 1)
                angle = s["pos"][rows].to(f64).outer(s["freq"].to(f64))
                turn[:, one, one], turn[:, two, two] = torch.cos(angle), torch.cos(angle)
                turn[:, one, two], turn[:, two, one] = torch.sin(angle), -torch.sin(angle)
                y[rows] = (unit[rows] * w) @ turn
                if dy is not None:
                    back[rows] = dy[rows] @ turn.transpose(1, 2).contiguous()
            out[n] = y
            if dy is not None:
                g = back * w
                root = (torch.linalg.vector_norm(x, dim=2, keepdim=True).square().div(D).add(EPS)).sqrt()
                out["d" + n] = (g - unit * (g * unit).mean(2, keepdim=True)) / root
                out["dw" + n] = (back * unit).flatten(0, 1).sum(0)
        return out
    T, V, K, tau = case["T"], case["V"], case["K"], case["temperature"]
    W = s["W"].to(f64)
    zeros = lambda *shape: torch.zeros(*shape, dtype=f64, device=DEV)  # noqa: E731
    out = {"logp": zeros(T), "entropy": zeros(T)}
    if K:
        out["ids"], out["top"] = torch.full((T, K), -1, dtype=torch.int32, device=DEV), zeros(T, K)
    if kind == "policy":
        out["dx"], out["dW"] = zeros(T, case["d"]), zeros(V, case["d"])
    # rows that have a target, some at a time (the others have nothing in any output)
    for rows in torch.nonzero(s["target"] >= 0)[:, 0].split(2048):
        x, y = s["x"][rows].to(f64), s["target"][rows].long()
        z = x @ W.t()
        log_p = torch.log_softmax(z / tau, 1)
        p = log_p.exp()
        entropy = -(p * log_p).sum(1)
        out["logp"][rows] = log_p.gather(1, y[:, None])[:, 0]
        out["entropy"][rows] = entropy
        if K:
            ids = z.topk(K, 1).indices
            out["ids"][rows], out["top"][rows] = ids.int(), log_p.gather(1, ids)
        if kind == "policy":
            a, b = s["dlogp"][rows].to(f64)[:, None], s["dentropy"][rows].to(f64)[:, None]
            dz = -a * p - b * p * (log_p + entropy[:, None])
            dz[torch.arange(len(rows), device=DEV), y] += a[:, 0]
            out["dx"][rows] = (dz / tau) @ W
            out["dW"] += (dz / tau).t() @ x
    return out
