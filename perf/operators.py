"""Operators that stand between and behind the expert layers of a model: what is timed, and what it has to give.

A case is one pass through one of

  "norm"       residual addition and root-mean-square norm, result in bfloat16
  "norm8"      the same with the result as e4m3 codes and one scale per `group` columns
  "norm_train" forward (bfloat16) and backward
  "score"      cross entropy of the vocabulary head for given tokens, forward only: log probabilities of a text
  "train"      cross entropy of the vocabulary head, forward and backward
  "kd_score"   cross entropy and distillation loss against a teacher's top logits, forward only
  "kd_train"   both losses, forward and backward

  T tokens, d hidden size, V vocabulary, K entries of the teacher per token, temperature, `masked` the share of tokens without a target
  (prompts, padding).  A token without a target also has no teacher entries; of the others some have fewer than K.

``own`` false: the operators in elementary torch operations, in 32 bits; true: the library's own calls.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
# the largest listed training step (T V d) and the widest norm (T d) bound what draw() may give
MAX_TVD = 4096 * 131072 * 2048
MAX_TD = 8192 * 2048
E4M3_MAX = 448.0


def _norm(name, kind, T, d, group=0):
    return {"name": name, "kind": kind, "T": T, "d": d, "group": group}


def _head(name, kind, T, d, V, masked=0.0, K=0, temperature=1.0):
    return {"name": name, "kind": kind, "T": T, "d": d, "V": V, "masked": masked, "K": K, "temperature": temperature}


def listed():
    return [
        # in front of a layer in one decoding step of a single sequence: the smallest call, all latency
        _norm("norm_decode_1", "norm", 1, 2048),
        # in front of a wide layer, several prompts, input of products in 8 bits
        _norm("norm_8bit_4001", "norm8", 4001, 4096, group=128),
        # the norm of a training step of four sequences of 2048 tokens
        _norm("norm_train_8192", "norm_train", 8192, 2048),
        # log probability of one token: the head's weights are read once
        _head("score_1", "score", 1, 2048, 50304),
        # log probabilities of a batch of short continuations, odd vocabulary
        _head("score_57", "score", 57, 4096, 32003),
        # the tiny model that tests train: launches are what counts
        _head("train_tiny", "train", 256, 128, 1031),
        # a step of supervised fine-tuning: ragged, a good part of the tokens belongs to prompts, odd vocabulary
        _head("train_masked_3001", "train", 3001, 1024, 50257, masked=0.4),
        # the pretraining step: four sequences of 2048 tokens
        _head("train_8192", "train", 8192, 2048, 50304),
        # evaluation of a student on some sequences
        _head("kd_score_129", "kd_score", 129, 2048, 32000, K=16, temperature=1.0),
        # distillation on ragged answers behind prompts
        _head("kd_train_masked_1501", "kd_train", 1501, 2048, 65537, masked=0.25, K=20, temperature=2.0),
        # distillation over a large vocabulary: the largest
        _head("kd_train_4096", "kd_train", 4096, 2048, 131072, K=64, temperature=1.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm8", "norm_train", "score", "train", "train", "kd_score", "kd_train", "kd_train"])
    if kind.startswith("norm"):
        group = rng.choice([0, 32, 64, 128]) if kind == "norm8" else 0
        while True:
            step = group or 8
            c = {"kind": kind, "T": _log_int(rng, 1, 16384), "d": step * _log_int(rng, max(1, 64 // step), 8192 // step), "group": group}
            if c["T"] * c["d"] <= MAX_TD:
                return c
    while True:
        c = {"kind": kind, "T": _log_int(rng, 1, 16384), "d": 64 * _log_int(rng, 1, 64), "V": _log_int(rng, 200, 200000),
             "masked": rng.choice([0.0, 0.0, 0.3, 0.8]), "K": 0, "temperature": 1.0}
        if kind.startswith("kd"):
            c.update(K=_log_int(rng, 1, 128), temperature=rng.choice([1.0, 0.7, 1.5, 4.0]))
        if c["T"] * c["V"] * c["d"] <= MAX_TVD and c["T"] * c["V"] <= 8192 * 131072:
            return c


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device=DEV, dtype=torch.float32)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    T, d = c["T"], c["d"]
    s = dict(c, kept={})
    if c["kind"].startswith("norm"):
        # a residual stream has a few columns that are far larger than the others
        column = torch.exp(0.8 * _normal(gen, d))
        s["x"] = _normal(gen, T, d).bfloat16()
        s["r"] = (2.0 * _normal(gen, T, d) * column).bfloat16()
        s["w"] = 0.8 + 0.4 * _uniform(gen, d)
        if c["kind"] == "norm_train":
            s["dy"] = _normal(gen, T, d).bfloat16()
            s["dsum"] = _normal(gen, T, d).bfloat16()
        return s
    V, K = c["V"], c["K"]
    s["W"] = torch.empty(V, d, dtype=torch.bfloat16, device=DEV)
    for v in range(0, V, 16384):
        s["W"][v:v + 16384] = _normal(gen, min(16384, V - v), d).mul_(0.02)
    target = torch.randint(0, V, (T,), generator=gen, device=DEV, dtype=torch.int64)
    # a trained model knows some of its targets well and others not at all: logits of 0 to 10 above the others'
    known = _uniform(gen, T, 1) * (10.0 / (0.02 * 0.02 * d))
    s["x"] = (_normal(gen, T, d) + known * s["W"][target].float()).bfloat16()
    live = _uniform(gen, T) >= c["masked"]
    live[0] = True
    s["target"] = torch.where(live, target, -100).int()
    # tokens count alike but for a weight
    s["dloss"] = (0.5 + _uniform(gen, T)) / T
    if K:
        # K different entries a token, the target among them, logits falling from the first to the last
        step = 1 + torch.randint(0, max(1, (V - 1) // K), (T, 1), generator=gen, device=DEV, dtype=torch.int64)
        step = torch.where(step * K < V, step, 1)
        place = torch.arange(K, device=DEV)[None, :]
        ids = (target[:, None] + place * step) % V
        logits = 4.0 - torch.cumsum(0.4 * _uniform(gen, T, K), 1) + 0.05 * _normal(gen, T, K)
        count = torch.where(_uniform(gen, T, 1) < 0.2, torch.ceil(K * _uniform(gen, T, 1)), K)
        there = (place < count) & live[:, None] & (place < V)
        s["ids"] = torch.where(there, ids, -1).int().contiguous()
        s["tl"] = torch.where(there, logits, 0.0).contiguous()
        s["dkd"] = c["temperature"] ** 2 * (0.5 + _uniform(gen, T)) / T
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------------


def _plain_norm(s):
    total = (s["x"].float() + s["r"].float()).bfloat16()
    v = total.float()
    rstd = torch.rsqrt((v * v).mean(1) + EPS)
    y = v * rstd[:, None] * s["w"]
    if s["kind"] == "norm8":
        T, d = y.shape
        g = s["group"] or d
        y = y.view(T, d // g, g)
        scale = y.abs().amax(2) / E4M3_MAX
        inverse = torch.where(scale > 0, 1.0 / scale, 0.0)
        codes = (y * inverse[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).view(T, d).to(torch.float8_e4m3fn)
        return {"sum": total, "codes": codes, "scale": scale}
    out = {"sum": total, "y": y.bfloat16()}
    if s["kind"] == "norm_train":
        dy = s["dy"].float()
        g = dy * s["w"]
        c = (g * v).mean(1) * rstd * rstd
        out["dx"] = (s["dsum"].float() + rstd[:, None] * (g - v * c[:, None])).bfloat16()
        out["dw"] = (dy * v * rstd[:, None]).sum(0)
    return out


def _log_sum_exp(z):
    top = z.amax(1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    return top + (z - top).exp().sum(1, keepdim=True).log()


def _plain_head(s):
    # Losses near zero are differences of nearly equal numbers as they are usually written.  Here what they are made of is positive:
    # with r the log of the sum over all columns but the target, loss = log(1 + exp(r - z_target)).
    T, V, K = s["T"], s["V"], s["K"]
    there = (s["target"] >= 0) & (s["target"] < V)
    at = torch.where(there, s["target"], 0).long()[:, None]
    x, W = s["x"].float(), s["W"].float()
    z = x @ W.t()
    away = _log_sum_exp(z.scatter(1, at, -math.inf)) - z.gather(1, at)
    loss = away.clamp_min(0.0) + (-away.abs()).exp().log1p()
    lse = loss + z.gather(1, at)
    out = {"loss": torch.where(there, loss[:, 0], 0.0), "lse": torch.where(there, lse[:, 0], 0.0)}
    train = s["kind"].endswith("train")
    if train:
        dz = (z - lse).exp()
        dz.scatter_(1, at, torch.expm1(-loss))
        dz *= torch.where(there, s["dloss"], 0.0)[:, None]
    if K:
        tau = s["temperature"]
        entry = (s["ids"] >= 0) & (s["ids"] < V) & (s["tl"] > -math.inf)
        taught = entry.any(1, keepdim=True)
        # (an entry that is not there points at a column behind the last)
        ids = torch.where(entry, s["ids"], V).long()
        tl = torch.where(entry, s["tl"] / tau, -math.inf)
        log_q = torch.where(entry, tl - _log_sum_exp(tl), 0.0)
        q = torch.where(entry, log_q.exp(), 0.0)
        zt = torch.cat([z / tau, torch.zeros_like(lse)], 1)
        # with a_j = z_j / tau - log q_j, their mean a under q, u_j = a_j - a and r over the columns that are no entry:
        # kd = log(1 + exp(r - a) + sum q (exp(u) - 1 - u))
        a = torch.where(entry, zt.gather(1, ids) - log_q, 0.0)
        mean = (q * a).sum(1, keepdim=True)
        u = torch.where(entry, a - mean, 0.0)
        r = _log_sum_exp(zt.scatter(1, ids, -math.inf)[:, :V])
        kd = torch.log1p((r - mean).exp() + (q * (torch.expm1(u) - u)).sum(1, keepdim=True))
        out["kd"] = torch.where(taught, kd, 0.0)[:, 0]
        if train:
            p = (zt - (kd + mean)).exp()
            p.scatter_add_(1, ids, -q)
            dz += p[:, :V] * torch.where(taught, s["dkd"][:, None] / tau, 0.0)
    if train:
        out["dx"] = (dz @ W).bfloat16()
        out["dW"] = (dz.t() @ x).bfloat16()
    return out


# ---- the library's calls -----------------------------------------------------------------------------------------------------


def _kept(s, B):
    """Buffers that a program lays out once for a shape."""
    k = s["kept"]
    if k:
        return k
    T, d = s["T"], s["d"]
    new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device=DEV)  # noqa: E731
    space = lambda n: new(max(n, 256), dtype=torch.uint8)  # noqa: E731
    if s["kind"].startswith("norm"):
        k.update(sum=new(T, d, dtype=torch.bfloat16), rstd=new(T))
        if s["kind"] == "norm8":
            k.update(codes=new(T, d, dtype=torch.float8_e4m3fn), scale=new(T, d // (s["group"] or d)))
        else:
            k.update(y=new(T, d, dtype=torch.bfloat16))
        if s["kind"] == "norm_train":
            k.update(dx=new(T, d, dtype=torch.bfloat16), dw=new(d), ws=space(B.moe_add_rms_norm_bwd_workspace_bytes(T, d)))
        return k
    V, K = s["V"], s["K"]
    k.update(loss=new(T), lse=new(T))
    nbytes = B.moe_head_fwd_workspace_bytes(T, d, V, K)
    if K:
        k.update(kd=new(T), lse_t=new(T))
    if s["kind"].endswith("train"):
        k.update(dx=new(T, d, dtype=torch.bfloat16), dW=new(V, d, dtype=torch.bfloat16))
        nbytes = max(nbytes, B.moe_head_bwd_workspace_bytes(T, d, V, K, 0))
    k.update(ws=space(nbytes))
    return k


def _own(s):
    from paper_2604_00785_amd import binding as B

    k = _kept(s, B)
    if s["kind"] == "norm8":
        B.moe_add_rms_norm_8bit(s["x"], s["r"], s["w"], EPS, s["group"], k["sum"], k["codes"], k["scale"], None)
        return {"sum": k["sum"], "codes": k["codes"], "scale": k["scale"]}
    if s["kind"] == "norm":
        B.moe_add_rms_norm(s["x"], s["r"], s["w"], EPS, k["sum"], k["y"], None)
        return {"sum": k["sum"], "y": k["y"]}
    if s["kind"] == "norm_train":
        B.moe_add_rms_norm(s["x"], s["r"], s["w"], EPS, k["sum"], k["y"], k["rstd"])
        B.moe_add_rms_norm_bwd(s["dy"], s["dsum"], k["sum"], s["w"], k["rstd"], k["dx"], k["dw"], k["ws"])
        return {"sum": k["sum"], "y": k["y"], "dx": k["dx"], "dw": k["dw"]}
    train = s["kind"].endswith("train")
    x, W, target, ws = s["x"], s["W"], s["target"], k["ws"]
    out = {"loss": k["loss"], "lse": k["lse"]}
    if s["K"]:
        teacher = (s["ids"], s["tl"], s["temperature"])
        B.moe_head_distill_fwd(x, W, target, *teacher, k["loss"], k["lse"], k["kd"], k["lse_t"], ws)
        out["kd"] = k["kd"]
        if train:
            B.moe_head_distill_bwd(x, W, target, *teacher, k["loss"], k["lse"], k["lse_t"], s["dloss"], s["dkd"], 0, k["dx"], k["dW"], ws)
    else:
        B.moe_head_ce_fwd(x, W, target, k["loss"], k["lse"], ws)
        if train:
            B.moe_head_ce_bwd(x, W, target, k["loss"], k["lse"], s["dloss"], 0, k["dx"], k["dW"], ws)
    if train:
        out.update(dx=k["dx"], dW=k["dW"])
    return out


def run(s):
    if own:
        return _own(s)
    return _plain_norm(s) if s["kind"].startswith("norm") else _plain_head(s)


# ---- what a pass cannot do without, and its results in 64 bits -----------------------------------------------------------------


def work(case):
    c = case
    T, d = c["T"], c["d"]
    if c["kind"].startswith("norm"):
        nbytes = 8.0 * T * d + 4.0 * d                                   # x, r; sum, y
        if c["kind"] == "norm8":
            nbytes += -1.0 * T * d + 4.0 * T * (d // (c["group"] or d))  # codes instead of y, scales
        if c["kind"] == "norm_train":
            nbytes += 6.0 * T * d + 4.0 * d                              # dy, dsum; dx
        return {"bytes": nbytes, "flops": 6.0 * T * d * (2 if c["kind"] == "norm_train" else 1)}
    V, K, live = c["V"], c["K"], c["T"] * (1.0 - c["masked"])
    nbytes = 2.0 * V * d + 2.0 * live * d + 12.0 * T + 12.0 * T * (K > 0) + 8.0 * live * K
    flops = 2.0 * live * V * d
    if c["kind"].endswith("train"):
        nbytes += 2.0 * V * d + 2.0 * T * d + 4.0 * T
        flops *= 3.0                                                     # logits once, and the two products of the backward pass
    return {"bytes": nbytes, "flops": flops}


def exact(case, seed):
    s = prepare(case, seed)
    kind, f64 = case["kind"], torch.float64
    if kind.startswith("norm"):
        total = s["x"].to(f64).add(s["r"].to(f64)).to(torch.bfloat16)
        v = total.to(f64)
        root = torch.linalg.vector_norm(v, dim=1, keepdim=True).square().div(case["d"]).add(EPS).sqrt()
        y = v / root * s["w"].to(f64)
        if kind == "norm8":
            parts = y.unflatten(1, (-1, case["group"] or case["d"]))
            scale = torch.linalg.vector_norm(parts, ord=math.inf, dim=2) / E4M3_MAX
            codes = (parts / scale.clamp_min(1e-300).unsqueeze(2)).flatten(1).float().to(torch.float8_e4m3fn)
            return {"sum": total.to(f64), "codes": codes.to(f64), "scale": scale}
        out = {"sum": total.to(f64), "y": y}
        if kind == "norm_train":
            unit = v / root
            g = s["dy"].to(f64) * s["w"].to(f64)
            out["dx"] = s["dsum"].to(f64) + (g - unit * (g * unit).mean(1, keepdim=True)) / root
            out["dw"] = torch.einsum("td,td->d", s["dy"].to(f64), unit)
        return out
    T, V, K, tau = case["T"], case["V"], case["K"], case["temperature"]
    train = kind.endswith("train")
    W = s["W"].to(f64)
    out = {n: torch.zeros(T, dtype=f64, device=DEV) for n in ["loss", "lse"] + (["kd"] if K else [])}
    if train:
        out["dx"] = torch.zeros(T, case["d"], dtype=f64, device=DEV)
        out["dW"] = torch.zeros(V, case["d"], dtype=f64, device=DEV)
    # rows that have a target, some at a time (the others have nothing in any output)
    for rows in torch.nonzero(s["target"] >= 0)[:, 0].split(2048):
        x = s["x"][rows].to(f64)
        z = x @ W.t()
        one = torch.zeros_like(z)
        one[torch.arange(len(rows), device=DEV), s["target"][rows].long()] = 1.0
        lse = torch.logsumexp(z, 1)
        out["lse"][rows] = lse
        out["loss"][rows] = lse - (z * one).sum(1)
        dz = (torch.softmax(z, 1) - one) * s["dloss"][rows].to(f64)[:, None]
        if K:
            ids, tl = s["ids"][rows].long(), s["tl"][rows].to(f64)
            # a column behind the last takes the entries that are not there
            full = torch.full((len(rows), V + 1), -math.inf, dtype=f64, device=DEV)
            full.scatter_(1, torch.where(ids >= 0, ids, V), torch.where(ids >= 0, tl / tau, -math.inf))
            some = (ids >= 0).any(1, keepdim=True)
            q = torch.softmax(full[:, :V], 1).nan_to_num_(0.0)
            log_p = torch.log_softmax(z / tau, 1)
            out["kd"][rows] = torch.special.xlogy(q, q).sum(1) - (q * log_p).sum(1)
            dz += (log_p.exp() * some - q) * (s["dkd"][rows].to(f64) / tau)[:, None]
        if train:
            out["dx"][rows] = dz @ W
            out["dW"] += dz.t() @ x
    return out
