"""The vocabulary head's losses and gradients against 64 bits."""
import pytest
import torch

import head_reference as R
from paper_2604_00785_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def make(T, d, V, K=0, masked=0.0, seed=0, known=6.0, std=0.05):
    g = torch.Generator().manual_seed(seed * 1000003 + T * 131 + d * 7 + V + K)
    a = {"W": (std * torch.randn(V, d, generator=g)).bfloat16()}
    target = torch.randint(0, V, (T,), generator=g)
    lift = known * torch.rand(T, 1, generator=g) / (std * std * d)
    a["x"] = (torch.randn(T, d, generator=g) + lift * a["W"][target].float()).bfloat16()
    live = torch.rand(T, generator=g) >= masked
    a["target"] = torch.where(live, target, -100).int()
    a["dloss"] = (torch.rand(T, generator=g) + 0.5) / T
    if K:
        n = min(K, V)
        ids = torch.stack([torch.randperm(V, generator=g)[:n] for _ in range(T)])
        if n < K:
            ids = torch.cat([ids, torch.full((T, K - n), -1)], 1)
        # the target among the entries in half of the rows
        for t in range(0, T, 2):
            if not bool((ids[t] == target[t]).any()):
                ids[t, t % n] = target[t]
        count = torch.randint(1, K + 1, (T, 1), generator=g)
        count[torch.rand(T, 1, generator=g) < 0.5] = K
        there = (torch.arange(K)[None] < count) & live[:, None]
        a["ids"] = torch.where(there, ids, -1).int()
        a["teacher"] = torch.where(there, 3 * torch.randn(T, K, generator=g), 0.0)
        a["dkd"] = (torch.rand(T, generator=g) + 0.5) / T
    return a


def run(a, tau=1.0, v_piece=0, train=True, junk=0xAB):
    t = {k: v.to(DEV) for k, v in a.items()}
    (T, d), V, K = a["x"].shape, a["W"].shape[0], a["ids"].shape[1] if "ids" in a else 0
    f = lambda: torch.full((T,), 7.0, device=DEV)  # noqa: E731
    out = {"loss": f(), "lse": f()}
    n = B.moe_head_fwd_workspace_bytes(T, d, V, K)
    if train:
        n = max(n, B.moe_head_bwd_workspace_bytes(T, d, V, K, v_piece))
    ws = torch.full((n,), junk, dtype=torch.uint8, device=DEV)
    if K:
        out.update(kd=f(), lse_t=f())
        B.moe_head_distill_fwd(t["x"], t["W"], t["target"], t["ids"], t["teacher"], tau, out["loss"], out["lse"], out["kd"], out["lse_t"], ws)
    else:
        B.moe_head_ce_fwd(t["x"], t["W"], t["target"], out["loss"], out["lse"], ws)
    if train:
        ws.fill_(junk)                                    # nothing is kept from one call to the next
        dx, dW = torch.full((T + 1, d), 7.0, dtype=BF, device=DEV), torch.full((V + 1, d), 7.0, dtype=BF, device=DEV)
        if K:
            B.moe_head_distill_bwd(t["x"], t["W"], t["target"], t["ids"], t["teacher"], tau, out["loss"], out["lse"], out["lse_t"],
                                   t["dloss"], t["dkd"], v_piece, dx[:T], dW[:V], ws)
        else:
            B.moe_head_ce_bwd(t["x"], t["W"], t["target"], out["loss"], out["lse"], t["dloss"], v_piece, dx[:T], dW[:V], ws)
        assert bool((dx[T] == 7).all()) and bool((dW[V] == 7).all())
        out.update(dx=dx[:T], dW=dW[:V])
    return out


def run_at_edge(a, edge, tau=1.0, v_piece=0):
    """Both directions with the tiles of every product at one edge, whatever the rule would take."""
    import ctypes
    lib = B.load()
    P, I, F = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    lib.moe_head_fwd.argtypes = [P] * 5 + [F] + [I] * 4 + [P] * 5 + [ctypes.c_size_t, P, P]
    lib.moe_head_bwd.argtypes = [P] * 5 + [F] + [P] * 5 + [I] * 5 + [P] * 3 + [ctypes.c_size_t, P, P]
    t = {k: v.to(DEV) for k, v in a.items()}
    (T, d), V, K = a["x"].shape, a["W"].shape[0], a["ids"].shape[1] if "ids" in a else 0
    n = max(B.moe_head_fwd_workspace_bytes(T, d, V, K), B.moe_head_bwd_workspace_bytes(T, d, V, K, v_piece))
    ws = torch.full((n,), 0xAB, dtype=torch.uint8, device=DEV)
    out = {k: torch.full((T,), 7.0, device=DEV) for k in ["loss", "lse"] + (["kd", "lse_t"] if K else [])}
    out.update(dx=torch.empty(T, d, dtype=BF, device=DEV), dW=torch.empty(V, d, dtype=BF, device=DEV))
    p = lambda o, k: o[k].data_ptr() if k in o else None  # noqa: E731
    head = [p(t, "x"), p(t, "W"), p(t, "target"), p(t, "ids"), p(t, "teacher"), tau]
    stream = torch.cuda.current_stream().cuda_stream
    fwd, bwd = (ctypes.c_int * 1)(edge), (ctypes.c_int * 2)(edge, edge)
    assert lib.moe_head_fwd(*head, T, d, V, K, *[p(out, k) for k in ("loss", "lse", "kd", "lse_t")], ws.data_ptr(), n, stream, ctypes.addressof(fwd)) == 0
    assert lib.moe_head_bwd(*head, *[p(out, k) for k in ("loss", "lse", "lse_t")], p(t, "dloss"), p(t, "dkd"), T, d, V, K, v_piece, p(out, "dx"),
                            p(out, "dW"), ws.data_ptr(), n, stream, ctypes.addressof(bwd)) == 0
    assert list(fwd) == [edge] and list(bwd) == [edge] * 2
    return out


def compare(a, got, tau=1.0):
    train = "dx" in got
    want, bound = R.head(a["x"], a["W"], a["target"], a.get("ids"), a.get("teacher"), tau, a["dloss"] if train else None, a.get("dkd"))
    for k in got:
        R.check(got[k], want[k], bound[k], k)
    for k in ("dx", "dW"):
        if k in got:
            # Two roundings to bf16, each uniform in half a step at most: 2^-8 sqrt(2 / 3) together where many of either are independent.
            # A token that hangs on its target alone has one rounding for its whole row of dx, so that takes many tokens.
            if a["x"].shape[0] < 16:
                continue
            R.check_norm_rel(got[k], want[k], R.HALF16 * (2 / 3) ** 0.5 * 1.05, k)
    return want


CE = [(1, 64, 1), (1, 64, 2), (1, 128, 1031), (2, 64, 63), (5, 192, 65), (16, 64, 128), (17, 128, 129), (31, 64, 257), (33, 320, 1000), (64, 64, 4097),
      (65, 128, 515), (100, 256, 300), (129, 64, 640), (200, 128, 1031), (257, 192, 777), (513, 64, 256), (40, 1024, 199)]


@pytest.mark.parametrize("T,d,V", CE)
def test_cross_entropy(T, d, V):
    print("cross entropy", T, d, V, flush=True)
    a = make(T, d, V)
    compare(a, run(a))


@pytest.mark.parametrize("T,d,V", [(300, 512, 20011), (1100, 128, 6001), (1500, 320, 1999)])
@pytest.mark.parametrize("masked", [0.0, 0.4])
def test_cross_entropy_of_many_tiles(T, d, V, masked):
    print("cross entropy", T, d, V, masked, flush=True)
    a = make(T, d, V, masked=masked)
    compare(a, run(a))


@pytest.mark.parametrize("T,d,V,K", [(1, 64, 5, 1), (1, 64, 3, 3), (3, 64, 200, 128), (2, 64, 7, 20), (17, 128, 300, 20), (64, 64, 1000, 7), (130, 192, 513, 64),
                                     (257, 64, 4099, 33), (700, 128, 2050, 3), (48, 64, 700, 300)])
@pytest.mark.parametrize("tau", [1.0, 0.7, 4.0])
def test_distillation(T, d, V, K, tau):
    print("distillation", T, d, V, K, tau, flush=True)
    a = make(T, d, V, K, masked=0.2 if T > 2 else 0.0)
    compare(a, run(a, tau), tau)


@pytest.mark.parametrize("edge", [128, 256])
@pytest.mark.parametrize("T,d,V,K,masked", [(1, 64, 1, 0, 0), (1, 192, 700, 0, 0), (17, 128, 129, 20, 0.2), (64, 64, 257, 0, 0), (65, 128, 5000, 3, 0), (128, 256, 640, 0, 0.5),
                                            (129, 64, 1031, 64, 0), (250, 128, 300, 100, 0.1), (256, 64, 256, 0, 0), (300, 320, 513, 33, 0.3), (600, 64, 3001, 0, 0.6),
                                            (520, 64, 200, 128, 0)])
def test_both_tile_edges(T, d, V, K, masked, edge):
    print("edge", edge, T, d, V, K, masked, flush=True)
    a = make(T, d, V, K, masked=masked, seed=15)
    if masked:
        a["target"][0] = 0                               # not all without a loss
    tau = 1.3 if K % 2 else 1.0
    compare(a, run_at_edge(a, edge, tau), tau)
    if V > 512:
        compare(a, run_at_edge(a, edge, tau, v_piece=512), tau)


def test_targets_and_entries_come_and_go_apart():
    """Rows with a target only, with entries only, with neither, and entries that do not count."""
    T, d, V, K = 96, 128, 777, 9
    a = make(T, d, V, K, seed=3)
    t = torch.arange(T)
    a["target"][t % 4 == 0] = torch.tensor([-100, -1, V, 2 ** 31 - 1] * (T // 16)).int()
    a["ids"][t % 3 == 0] = -1
    a["ids"][t % 5 == 1, 0] = V
    a["ids"][t % 5 == 2, 1] = 2 ** 31 - 1
    a["teacher"][t % 5 == 3, 2] = -float("inf")
    a["teacher"][t % 7 == 3] = -float("inf")
    for tau in (1.0, 1.5):
        compare(a, run(a, tau), tau)


@pytest.mark.parametrize("K", [0, 5])
def test_no_token_has_a_loss(K):
    a = make(70, 64, 300, K, seed=4)
    a["target"][:] = -100
    if K:
        a["ids"][:] = -1
    for k, v in run(a).items():
        assert bool((v == 0).all()), k


@pytest.mark.parametrize("live", [0, 1, 63, 64, 65, 199])
def test_one_token_has_a_loss(live):
    a = make(200, 64, 300, seed=5)
    keep = a["target"][live].clone()
    a["target"][:] = -100
    a["target"][live] = keep
    compare(a, run(a))


@pytest.mark.parametrize("T", [4097, 9000])
def test_many_tokens(T):
    """More tokens than a workgroup finds by itself."""
    a = make(T, 64, 130, masked=0.5, seed=6)
    compare(a, run(a))


@pytest.mark.parametrize("K,tau", [(0, 1.0), (11, 1.3)])
def test_pieces_of_the_vocabulary(K, tau):
    a = make(150, 128, 1500, K, masked=0.3, seed=7)
    whole = run(a, tau)
    compare(a, whole, tau)
    for piece in (256, 512, 1280):
        got = run(a, tau, v_piece=piece)
        compare(a, got, tau)
        assert torch.equal(got["dW"], whole["dW"]) and torch.equal(got["loss"], whole["loss"])


def test_losses_near_zero_and_far_away():
    """A target that is all but certain: its loss has a relative, not an absolute error.  And logits in the hundreds."""
    T, d, V = 64, 128, 900
    a = make(T, d, V, seed=8, known=0.0)
    lift = torch.linspace(5, 80, T)[:, None] / (0.05 ** 2 * d)
    a["x"] = (a["x"].float() + lift * a["W"][a["target"].long()].float()).bfloat16()
    got = run(a, train=False)
    want, bound = R.head(a["x"], a["W"], a["target"])
    R.check(got["loss"], want["loss"], bound["loss"] * want["loss"].clamp(max=1.0) + 1e-38, "loss")
    a["x"] = (a["x"].float() * 8).bfloat16()
    compare(a, run(a))


def test_student_is_the_teacher():
    """All columns are entries and the teacher's logits are the student's: a divergence of zero, and no gradient beyond the logits' error."""
    T, d, V = 20, 64, 40
    a = make(T, d, V, V, seed=9)
    a["ids"] = torch.arange(V).int().repeat(T, 1)
    a["teacher"] = (a["x"].to(R.F64) @ a["W"].to(R.F64).t()).float()
    a["target"][:] = -100
    got = run(a, 2.0)
    want, bound = R.head(a["x"], a["W"], a["target"], a["ids"], a["teacher"], 2.0, a["dloss"], a["dkd"])
    assert bool((got["kd"].cpu() >= -1e-7).all()) and float(got["kd"].abs().max()) <= float(bound["kd"].max())
    R.check(got["dx"], want["dx"], bound["dx"], "dx")
    R.check(got["dW"], want["dW"], bound["dW"], "dW")


def test_gradients_are_differences_of_forward_passes():
    T, d, V, K, tau = 24, 64, 300, 6, 1.5
    a = make(T, d, V, K, seed=10)
    got = run(a, tau)
    weight = lambda o: float((o["loss"].cpu().to(R.F64) * a["dloss"] + o["kd"].cpu().to(R.F64) * a["dkd"]).sum())  # noqa: E731
    g = torch.Generator().manual_seed(1)
    for name, grad, h in (("x", "dx", 0.02), ("W", "dW", 0.002)):
        step = h * torch.randn(a[name].shape, generator=g)
        up, down = dict(a), dict(a)
        up[name], down[name] = (a[name].float() + step).bfloat16(), (a[name].float() - step).bfloat16()
        moved = up[name].to(R.F64) - down[name].to(R.F64)
        change = weight(run(up, tau, train=False)) - weight(run(down, tau, train=False))
        slope = float((got[grad].cpu().to(R.F64) * moved).sum())
        size = float((got[grad].cpu().to(R.F64) * moved).norm())
        # the rounding of the gradient's elements, the points not lying evenly about a (bf16), and a third order in the step
        assert abs(change - slope) <= 0.02 * size + 0.02 * abs(slope) + 1e-5, (name, change, slope)


@pytest.mark.parametrize("K", [0, 9])
def test_the_same_bits_every_time_and_on_another_stream(K):
    a = make(333, 128, 1200, K, masked=0.2, seed=11)
    first = run(a, 1.5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run(a, 1.5, junk=0)
    side.synchronize()
    for k in first:
        assert torch.equal(first[k], again[k]), k


def test_a_captured_step_gives_the_eager_results():
    T, d, V, K, tau = 150, 128, 900, 7, 1.5
    a = [make(T, d, V, K, masked=0.2, seed=s) for s in (12, 13)]
    t = {k: v.to(DEV) for k, v in a[0].items()}
    f = lambda: torch.empty(T, device=DEV)  # noqa: E731
    loss, lse, kd, lse_t, dx, dW = f(), f(), f(), f(), torch.empty(T, d, dtype=BF, device=DEV), torch.empty(V, d, dtype=BF, device=DEV)
    ws = torch.empty(max(B.moe_head_fwd_workspace_bytes(T, d, V, K), B.moe_head_bwd_workspace_bytes(T, d, V, K)), dtype=torch.uint8, device=DEV)

    def step():
        B.moe_head_distill_fwd(t["x"], t["W"], t["target"], t["ids"], t["teacher"], tau, loss, lse, kd, lse_t, ws)
        B.moe_head_distill_bwd(t["x"], t["W"], t["target"], t["ids"], t["teacher"], tau, loss, lse, lse_t, t["dloss"], t["dkd"], 0, dx, dW, ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(4):
        for k, v in a[n % 2].items():
            t[k].copy_(v)
        want = run(a[n % 2], tau)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in dict(loss=loss, lse=lse, kd=kd, lse_t=lse_t, dx=dx, dW=dW).items():
            assert torch.equal(v, want[k]), (n, k)


def test_gradients_may_be_negative_zero_or_large():
    """dloss and dkd are any numbers: zero for a token leaves no trace, a sign turns the gradient."""
    a = make(40, 64, 200, 5, seed=14)
    a["dloss"][::3] = 0
    a["dkd"][::2] = 0
    a["dloss"][1::3] *= -3e4
    compare(a, run(a, 1.5), 1.5)


@pytest.mark.parametrize("T,K", [(60, 0), (60, 7), (500, 0), (500, 7)])
def test_nothing_of_a_token_without_a_loss_is_looked_at(T, K):
    """NaN wherever a masked token or an entry that does not count has a number."""
    a = make(T, 64, 300, K, masked=0.4, seed=16)
    out = a["target"] < 0
    a["target"][0], out[0] = 5, False
    clean = compare(a, run(a, 1.5), 1.5)
    nan = float("nan")
    a["x"][out] = nan
    a["dloss"][out] = nan
    if K:
        a["dkd"][out] = nan
        a["teacher"][a["ids"] < 0] = nan
    got = run(a, 1.5)
    a["x"][out] = 0
    a["dloss"][out] = 0
    if K:
        a["dkd"][out] = 0
        a["teacher"][a["ids"] < 0] = 0
    compare(a, got, 1.5)
    assert torch.equal(clean["loss"], R.head(a["x"], a["W"], a["target"])[0]["loss"])


@pytest.mark.parametrize("T,masked", [(64, 0.0), (65, 0.0), (128, 0.0), (200, 0.6), (255, 0.55), (600, 0.85)])
@pytest.mark.parametrize("K", [0, 9])
def test_weight_gradient_of_few_tokens_is_rounded_once(T, masked, K):
    """With up to 128 losses, what rounding the logits' gradient loses goes into dW as well: 2 terms leave 2^-18 of it, the logits' errors some 1e-5,
    and what remains is the rounding of dW itself, 2^-9 / sqrt(3) and more of its norm: a twentieth of that is left for all else."""
    a = make(T, 256, 3000, K, masked, seed=5)
    assert int((a["target"] >= 0).sum()) <= 128
    got = run(a)
    want, _ = R.head(a["x"], a["W"], a["target"], a.get("ids"), a.get("teacher"), 1.0, a["dloss"], a.get("dkd"))
    once = float((want["dW"].bfloat16().double() - want["dW"]).norm())
    off = float((got["dW"].cpu().double() - want["dW"]).norm())
    assert off <= 1.05 * once, (off, once)


def test_offsets_past_32_bits():
    """A gradient of the logits of 5.8 GB (and 2.9e9 elements), checked at tokens and columns from all over it."""
    T, d, V = 72000, 64, 40001
    g = torch.Generator(device=DEV).manual_seed(17)
    x = torch.randn(T, d, generator=g, device=DEV).bfloat16()
    W = (0.1 * torch.randn(V, d, generator=g, device=DEV)).bfloat16()
    target = torch.randint(0, V, (T,), generator=g, device=DEV).int()
    dloss = torch.rand(T, generator=g, device=DEV) / T
    loss, lse = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    dx, dW = torch.empty(T, d, dtype=BF, device=DEV), torch.empty(V, d, dtype=BF, device=DEV)
    piece = (V + 255) // 256 * 256
    ws = torch.empty(max(B.moe_head_fwd_workspace_bytes(T, d, V), B.moe_head_bwd_workspace_bytes(T, d, V, 0, piece)), dtype=torch.uint8, device=DEV)
    assert T * piece * 2 > 2 ** 32 and ws.numel() > T * piece * 2
    B.moe_head_ce_fwd(x, W, target, loss, lse, ws)
    B.moe_head_ce_bwd(x, W, target, loss, lse, dloss, piece, dx, dW, ws)
    rows = torch.cat([torch.arange(0, T, 1999), torch.tensor([T - 1])])
    few = {"x": x[rows.to(DEV)].cpu(), "W": W.cpu(), "target": target[rows.to(DEV)].cpu(), "dloss": dloss[rows.to(DEV)].cpu()}
    want, bound = R.head(few["x"], few["W"], few["target"], dloss=few["dloss"])
    for k, v in (("loss", loss), ("lse", lse), ("dx", dx)):
        R.check(v[rows.to(DEV)], want[k], bound[k], k)
    # columns: the gradient over all tokens, in 64 bits, with the log of the sums checked above
    cols = torch.cat([torch.arange(0, V, 4003), torch.tensor([V - 1])]).to(DEV)
    z = x.double() @ W[cols].double().t()
    dz = (z - lse.double()[:, None]).exp() - (target[:, None] == cols[None, :]).double()
    dz *= dloss.double()[:, None]
    ref = dz.t() @ x.double()
    # (the factor of dz's rounding, its exponential's and the sum's: T terms)
    off = (R.HALF16 + 2.0 ** -16 + T * R.HALF32) * (dz.abs().t() @ x.double().abs()) + R.HALF16 * ref.abs()
    R.check(dW[cols], ref.cpu(), off.cpu(), "dW")
