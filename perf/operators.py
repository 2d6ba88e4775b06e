"""What a training program asks of the sequence operators, as cases that can be timed and checked.

Linear attention with a decay for each head is the memory of a policy: whole sequences in training (forward and
backward), one step of every environment while acting.  Layer norm stands before and behind it.  The sizes are those of
the repository's workloads (64 and 4096 environments, 24 steps, memories 256 wide as four heads of 64, layers of 512, 235 observations,
a quarter of the environments per minibatch), long sequences of a few environments, and irregular sizes between them.
With `own` false, `run` computes the same in elementary torch operations.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-5
CHUNK = 64                         # steps that the plain form takes together


# ---- the cases ------------------------------------------------------------------------------------------------------
def listed():
    return [
        # acting in a small run or an evaluation: one step of 64 environments, latency counts
        dict(name="step_64", kind="step", N=64, H=4, Dk=32, Dv=32, dtype="fp32", done_p=0.02),
        # acting in the standard training run: a memory of four heads of 64 per environment, episodes end here and there
        dict(name="step_4096", kind="step", N=4096, H=4, Dk=64, Dv=64, dtype="fp32", done_p=0.01),
        # a whole roll-out through the memory, from the states that its first step started from
        dict(name="forward_rollout", kind="forward", T=24, N=4096, H=4, Dk=64, Dv=64, dtype="fp32", done_p=0.01, s0=True, ragged=False),
        # a long history of two environments in bf16, heads of 128
        dict(name="forward_long", kind="forward", T=8192, N=2, H=8, Dk=128, Dv=128, dtype="bf16", done_p=0.0, s0=False, ragged=False),
        # padded trajectories of different lengths, sizes that fit no tile
        dict(name="forward_ragged", kind="forward", T=777, N=37, H=3, Dk=40, Dv=72, dtype="fp16", done_p=0.004, s0=True, ragged=True),
        # gradients of one minibatch of the standard training run: a quarter of the environments, all steps
        dict(name="backward_rollout", kind="backward", T=24, N=1024, H=4, Dk=64, Dv=64, dtype="fp32", done_p=0.01, s0=True, ragged=False),
        # gradients over long sequences in bf16
        dict(name="backward_long", kind="backward", T=4096, N=4, H=8, Dk=64, Dv=64, dtype="bf16", done_p=0.0, s0=False, ragged=False),
        # gradients of a few padded trajectories with narrow odd heads
        dict(name="backward_ragged", kind="backward", T=333, N=5, H=2, Dk=24, Dv=20, dtype="fp32", done_p=0.01, s0=True, ragged=True),
        # the norm before the memory while a small run acts
        dict(name="norm_64", kind="norm", rows=64, cols=128, dtype="fp32"),
        # the norm over every step of the standard roll-out
        dict(name="norm_rollout", kind="norm", rows=98304, cols=512, dtype="bf16"),
        # gradients of the norm of height-scan observations over one minibatch
        dict(name="norm_backward_rough", kind="norm_backward", rows=24576, cols=235, dtype="fp32"),
        # gradients of a wide norm in bf16
        dict(name="norm_backward_wide", kind="norm_backward", rows=8192, cols=4096, dtype="bf16"),
    ]


def draw(rng):
    spread = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    dim = lambda: rng.choice([32, 64, 128, rng.randint(8, 128)])  # noqa: E731
    kind = rng.choice(["step", "forward", "forward", "backward", "backward", "norm", "norm_backward"])
    dtype = rng.choice(["fp32", "fp32", "bf16", "fp16"])
    most = [work(c) for c in listed() if c["kind"] == kind]
    while True:
        if kind == "step":
            c = dict(kind=kind, N=spread(64, 8192), H=rng.randint(1, 12), Dk=dim(), Dv=dim(), dtype=dtype, done_p=rng.choice([0.0, 0.01]))
        elif kind in ("forward", "backward"):
            T, ragged = spread(8, 8192), rng.random() < 0.35
            c = dict(kind=kind, T=T, N=spread(2, 4096), H=rng.randint(1, 12), Dk=dim(), Dv=dim(), dtype=dtype,
                     done_p=rng.choice([0.0, 0.01, 1.0 / T]), s0=rng.random() < 0.5, ragged=ragged)
            if c["T"] * c["N"] < 1024:
                continue
        else:
            c = dict(kind=kind, rows=spread(64, 131072), cols=spread(24, 8192), dtype=dtype)
        w = work(c)
        if all(w[m] <= max(x[m] for x in most) for m in w):
            return c


def work(case):
    kind, size = case["kind"], torch.empty(0, dtype=TYPES[case["dtype"]]).element_size()
    if kind.startswith("norm"):
        n, back = case["rows"] * case["cols"], kind == "norm_backward"
        return {"bytes": n * size * (3 if back else 2) + 8 * case["rows"] + (12 if back else 8) * case["cols"], "flops": n * (12 if back else 8)}
    N, H, Dk, Dv = (case[x] for x in ("N", "H", "Dk", "Dv"))
    state, heads = 4 * N * H * Dk * Dv, N * H
    if kind == "step":
        return {"bytes": 2 * state + heads * size * (2 * Dk + 2 * Dv) + N, "flops": 5 * heads * Dk * Dv}
    tokens = heads * case["T"] * (0.5 if case["ragged"] else 1.0)       # lengths are uniform
    if kind == "forward":
        b = tokens * size * (2 * Dk + Dv) + heads * case["T"] * size * Dv + state * (2 if case["s0"] else 1)
        return {"bytes": b, "flops": 4 * tokens * Dk * Dv}
    b = tokens * size * (2 * Dk + 2 * Dv) + heads * case["T"] * size * (2 * Dk + Dv) + state * (3 if case["s0"] else 2)
    return {"bytes": b, "flops": 10 * tokens * Dk * Dv}


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _inputs(case, seed):
    """Everything that the case's arithmetic depends on, on the GPU, from the seed alone."""
    g = torch.Generator("cuda")
    g.manual_seed(1000003 * seed + 17)
    dt = TYPES[case["dtype"]]
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    if case["kind"].startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        x = (normal(rows, cols) * (0.5 + 2 * torch.rand(rows, 1, generator=g, device="cuda")) + 0.5 * normal(rows, 1)).to(dt)
        return dict(x=x, dy=normal(rows, cols).to(dt), weight=1 + 0.2 * normal(cols), bias=0.1 * normal(cols))
    step = case["kind"] == "step"
    T, N, H, Dk, Dv = 1 if step else case["T"], case["N"], case["H"], case["Dk"], case["Dv"]
    # one product makes q, k and v of a step side by side
    qkv = normal(T, N, H * (2 * Dk + Dv)).to(dt)
    q, k, v = qkv.split([H * Dk, H * Dk, H * Dv], dim=2)
    i = dict(q=q.unflatten(2, (H, Dk)), k=k.unflatten(2, (H, Dk)), v=v.unflatten(2, (H, Dv)))
    # memories of about 4 to 250 steps
    i["log_decay"] = torch.log1p(-torch.exp2(-torch.linspace(2, 8, H, dtype=torch.float64, device="cuda"))).float()
    i["dones"] = (torch.rand(T, N, generator=g, device="cuda") < case["done_p"]).to(torch.uint8) if case["done_p"] else None
    i["s0"] = 2 * normal(N, H, Dk, Dv) if step or case["s0"] else None
    i["lengths"] = None
    if not step and case["ragged"]:
        i["lengths"] = torch.randint(0, T + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
        i["lengths"][0] = T
    if case["kind"] == "backward":
        i["do"], i["ds_last"] = normal(T, N, H, Dv).to(dt), normal(N, H, Dk, Dv)
    i["scale"] = 1.0 / math.sqrt(Dk)
    return i


def prepare(case, seed):
    """Inputs, and the buffers and workspace that a program keeps from call to call."""
    i = _inputs(case, seed)
    s = dict(case=dict(case), i=i)
    new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    dt = TYPES[case["dtype"]]
    if case["kind"].startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        x = i["x"].float()
        s["mean"] = x.mean(1) if case["kind"] == "norm_backward" else new(rows)
        s["rstd"] = (x - x.mean(1, keepdim=True)).square().mean(1).add(EPS).rsqrt() if case["kind"] == "norm_backward" else new(rows)
        s["out"] = new(rows, cols, dtype=dt)
        s["dweight"], s["dbias"] = new(cols), new(cols)
    else:
        N, H, Dk, Dv = (case[x] for x in ("N", "H", "Dk", "Dv"))
        T = case.get("T", 1)
        s["state"] = new(N, H, Dk, Dv)
        if case["kind"] == "backward":
            s["dq"], s["dk"], s["dv"] = new(T, N, H, Dk, dtype=dt), new(T, N, H, Dk, dtype=dt), new(T, N, H, Dv, dtype=dt)
        else:
            s["o"] = new(T, N, H, Dv, dtype=dt)
    if own:
        import paper_2509_10771_amd as rx
        s["rx"] = rx
        if case["kind"] == "norm_backward":
            s["ws"] = rx.workspace(rx.rslx_layer_norm_backward_workspace_bytes(case["rows"], case["cols"]))
        elif case["kind"] != "norm":
            step = case["kind"] == "step"
            s["la"] = rx.LinearAttn(dt, T, N, H, Dk, Dv, i["log_decay"], i["scale"], None if step else i["dones"], i["lengths"])
            if case["kind"] == "forward":
                s["ws"] = rx.workspace(rx.rslx_linear_attention_workspace_bytes(s["la"]))
            elif case["kind"] == "backward":
                s["ws"] = rx.workspace(rx.rslx_linear_attention_backward_workspace_bytes(s["la"]))
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    rx, i, kind = s["rx"], s["i"], s["case"]["kind"]
    if kind == "norm":
        rx.rslx_layer_norm(i["x"], i["weight"], i["bias"], EPS, s["out"], s["mean"], s["rstd"])
        return dict(y=s["out"], mean=s["mean"], rstd=s["rstd"])
    if kind == "norm_backward":
        rx.rslx_layer_norm_backward(i["dy"], i["x"], i["weight"], s["mean"], s["rstd"], s["out"], s["dweight"], s["dbias"], s["ws"])
        return dict(dx=s["out"], dweight=s["dweight"], dbias=s["dbias"])
    if kind == "step":
        rx.rslx_linear_attention_step(s["la"], i["q"], i["k"], i["v"], i["dones"], i["s0"], s["state"], s["o"])
        return dict(o=s["o"], state=s["state"])
    if kind == "forward":
        rx.rslx_linear_attention(s["la"], i["q"], i["k"], i["v"], i["s0"], s["o"], s["state"], s["ws"])
        return dict(o=s["o"], state=s["state"])
    rx.rslx_linear_attention_backward(s["la"], i["q"], i["k"], i["v"], i["s0"], i["do"], i["ds_last"], s["dq"], s["dk"], s["dv"], s["state"],
                                      s["ws"])
    return dict(dq=s["dq"], dk=s["dk"], dv=s["dv"], ds0=s["state"])


def _run_plain(s):
    i, case = s["i"], s["case"]
    kind, dt = case["kind"], TYPES[case["dtype"]]
    if kind.startswith("norm"):
        x = i["x"].float()
        if kind == "norm":
            mean = x.mean(1)
            c = x - mean[:, None]
            rstd = (c * c).mean(1).add(EPS).rsqrt()
            return dict(y=(c * rstd[:, None] * i["weight"] + i["bias"]).to(dt), mean=mean, rstd=rstd)
        dy, rstd = i["dy"].float(), s["rstd"][:, None]
        xh = (x - s["mean"][:, None]) * rstd
        g = dy * i["weight"]
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        return dict(dx=dx.to(dt), dweight=(dy * xh).sum(0), dbias=dy.sum(0))
    if kind == "step":
        q, k, v = (i[x][0].float() for x in ("q", "k", "v"))
        state = i["s0"] * torch.exp(i["log_decay"])[:, None, None]
        if i["dones"] is not None:
            state = torch.where(i["dones"][0].bool()[:, None, None, None], torch.zeros_like(state), state)
        state = state + k[..., None] * v[..., None, :]
        return dict(o=(i["scale"] * (q[..., None] * state).sum(2)).to(dt)[None], state=state)
    T, N, H, Dk, Dv = (case[x] for x in ("T", "N", "H", "Dk", "Dv"))
    # heads first, steps that do not exist taken out
    t = torch.arange(T, device="cuda")
    length = torch.full((N,), T, device="cuda") if i["lengths"] is None else i["lengths"].long()
    there = t[None] < length[:, None]                                            # [N, T]
    first = lambda x: torch.where(there[:, None, :, None], x.permute(1, 2, 0, 3), torch.zeros((), dtype=x.dtype, device="cuda")).float()  # noqa: E731
    last = lambda x: x.permute(2, 0, 1, 3).to(dt).contiguous()  # noqa: E731
    q, k, v = first(i["q"]), first(i["k"]), first(i["v"])
    ended = torch.zeros(N, T, dtype=torch.long, device="cuda") if i["dones"] is None else i["dones"].t().long() * there
    after = ended.cumsum(1)                                                      # episodes ended up to and with step t
    episode, now = after - ended, length - 1                                     # episode of step t
    final = after[:, -1]                                                         # episode that the last state belongs to
    zero = torch.zeros(N, H, Dk, Dv, device="cuda")
    s0 = zero if i["s0"] is None else i["s0"]
    first_episode = torch.zeros(N, dtype=torch.long, device="cuda")
    # positions of the forward walk, and those of the walk from the end
    there_at, back_at = t.expand(N, T), torch.clamp(now[:, None] - t, min=0)
    if kind == "forward":
        o, state = _walk(q, k, v, i["log_decay"], episode, there_at, first_episode, s0, 1, final, length, there)
        return dict(o=last(i["scale"] * o), state=state)
    do = first(i["do"])
    turn = lambda x: torch.where(there[:, None, :, None], x.gather(2, back_at[:, None, :, None].expand_as(x)), torch.zeros((), device="cuda"))  # noqa: E731
    dq, _ = _walk(do, v, k, i["log_decay"], episode, there_at, first_episode, s0.transpose(2, 3), 1, final, length, there)
    rq, rk, rv, rdo, repisode = turn(q), turn(k), turn(v), turn(do), episode.gather(1, back_at)
    zl = i["ds_last"] / i["scale"]
    dv, ds0 = _walk(rk, rq, rdo, i["log_decay"], repisode, there_at, final, zl, 0, first_episode, length, there)
    dk, _ = _walk(rv, rdo, rq, i["log_decay"], repisode, there_at, final, zl.transpose(2, 3), 0, first_episode, length, there)
    return dict(dq=last(i["scale"] * dq), dk=last(i["scale"] * turn(dk)), dv=last(i["scale"] * turn(dv)), ds0=i["scale"] * ds0)


def _walk(a, b, c, log_decay, episode, position, episode0, s0, lead, episode1, length, there):
    """o_i = sum over j <= i of the same episode of l^(i - j) (a_i . b_j) c_j, with the state s0 of episode0 before the first
    position (weight l^(i + lead)), and the state of episode1 behind the last one (weights l^(length - lead - j)); chunk by chunk, the
    chunks' states joined by one product."""
    N, H, T, D = a.shape
    E = c.shape[-1]
    C = min(CHUNK, T)
    n = -(-T // C)
    pad = n * C - T
    split = lambda x: torch.nn.functional.pad(x, (0, 0, 0, pad)).unflatten(2, (n, C))  # noqa: E731
    A, B, V = split(a), split(b), split(c)    # [N, H, n, C, .]
    ep = torch.nn.functional.pad(episode, (0, pad), value=-1).view(N, n, C)
    ld = log_decay.double()
    t = torch.arange(C, device=a.device)
    gap = (t[:, None] - t[None, :]).clamp(min=0)
    weight = (torch.exp(ld[:, None, None] * gap) * (t[:, None] >= t[None, :])).float()    # [H, C, C]
    same = ep[..., :, None] == ep[..., None, :]    # [N, n, C, C]
    o = ((A @ B.transpose(-1, -2)) * weight[None, :, None] * same[:, None]) @ V
    # what every chunk leaves behind itself, for the episode that goes on there
    begins = ep[:, :, 0]
    goes_on = torch.cat([begins[:, 1:], torch.full_like(begins[:, :1], -2)], 1)
    tail = torch.exp(ld[:, None] * (C - lead - t)).float()    # [H, C]
    left = (B * (tail[None, :, None] * (ep == goes_on[..., None])[:, None])[..., None]).transpose(-1, -2) @ V
    at = torch.arange(n, device=a.device)
    apart = at[:, None] - 1 - at[None, :]
    join = torch.exp(ld[:, None, None] * C * apart.clamp(min=0)) * (apart >= 0)    # [H, n, n]
    passes = begins[:, :, None] == goes_on[:, None, :]
    join = (join[None] * passes[:, None]).float()    # [N, H, n, n]
    enters = (join @ left.flatten(3)).view(N, H, n, D, E)
    start = torch.exp(ld[:, None] * C * at)[None] * (begins == episode0[:, None])[:, None]    # [N, H, n]
    enters = enters + start.float()[..., None, None] * s0[:, :, None]
    head = torch.exp(ld[:, None] * (t + lead)).float()
    o = o + ((A * (head[None, :, None] * (ep == begins[..., None])[:, None])[..., None]) @ enters)
    # the state behind the last position, from every step of its episode
    w = torch.exp(ld[:, None] * (length[:, None, None] - lead - position[:, None]).clamp(min=0)) * ((episode == episode1[:, None]) & there)[:, None]
    state = (b * w.float()[..., None]).transpose(-1, -2) @ c
    w0 = torch.exp(ld * length[:, None]) * (episode0 == episode1)[:, None]
    return o.flatten(2, 3)[:, :, :T], state + w0.float()[..., None, None] * s0


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------
def exact(case, seed):
    i, kind = _inputs(case, seed), case["kind"]
    if kind.startswith("norm"):
        x = i["x"].double()
        n = x.shape[1]
        m = x.sum(1, keepdim=True) / n
        var = ((x - m) ** 2).sum(1, keepdim=True) / n
        r = 1.0 / torch.sqrt(var + EPS)
        if kind == "norm":
            return dict(y=(x - m) * r * i["weight"].double() + i["bias"].double(), mean=m[:, 0], rstd=r[:, 0])
        dy, w = i["dy"].double(), i["weight"].double()
        c = x - m
        # through the mean and the variance
        dxh = dy * w
        dvar = (dxh * c).sum(1, keepdim=True) * (-0.5) * r ** 3
        dx = dxh * r + dvar * 2 * c / n
        dx = dx - (dxh * r).sum(1, keepdim=True) / n
        return dict(dx=dx, dweight=(dy * c * r).sum(0), dbias=dy.sum(0))
    T = 1 if kind == "step" else case["T"]
    N, H, Dk, Dv = (case[x] for x in ("N", "H", "Dk", "Dv"))
    if T * N * H * Dk * Dv > 1.5e11 or T > 20000:
        return None
    lam = torch.exp(i["log_decay"].double())[None, :, None, None]
    ends = torch.zeros(T, N, dtype=torch.bool, device="cuda") if i["dones"] is None else i["dones"].bool()
    length = torch.full((N,), T, device="cuda") if i["lengths"] is None else i["lengths"].long()
    col = lambda x: x[:, None, None, None]  # noqa: E731
    S = torch.zeros(N, H, Dk, Dv, dtype=torch.float64, device="cuda") if i["s0"] is None else i["s0"].double()
    if kind == "step":
        S = torch.where(col(ends[0]), torch.zeros_like(S), S) * lam + i["k"][0].double()[..., None] * i["v"][0].double()[..., None, :]
        return dict(o=(i["scale"] * (i["q"][0].double()[:, :, None] @ S)[:, :, 0])[None], state=S)
    back = kind == "backward"
    plain = not ends.any() and i["lengths"] is None
    out = torch.zeros(T, N, H, Dk if back else Dv, dtype=torch.float64, device="cuda")
    for t in range(T):
        new = S * lam
        new += i["k"][t].double()[..., None] * i["v"][t].double()[..., None, :]
        here = t < length
        r = (new @ i["do"][t].double()[..., None])[..., 0] if back else (i["q"][t].double()[:, :, None] @ new)[:, :, 0]
        out[t] = r if plain else r * here[:, None, None]
        if not plain:
            new = torch.where(col(ends[t]), torch.zeros_like(new), new)
            new = torch.where(col(here), new, S)
        S = new
    if not back:
        return dict(o=i["scale"] * out, state=S)
    dk, dv = (torch.zeros(T, N, H, d, dtype=torch.float64, device="cuda") for d in (Dk, Dv))
    dS = i["ds_last"].double()
    for t in range(T - 1, -1, -1):
        here = t < length
        new = dS if plain else torch.where(col(ends[t]), torch.zeros_like(dS), dS)
        new = new + i["scale"] * i["q"][t].double()[..., None] * i["do"][t].double()[..., None, :]
        a, b = (new @ i["v"][t].double()[..., None])[..., 0], (i["k"][t].double()[:, :, None] @ new)[:, :, 0]
        dk[t], dv[t] = (a, b) if plain else (a * here[:, None, None], b * here[:, None, None])
        new *= lam
        dS = new if plain else torch.where(col(here), new, dS)
    return dict(dq=i["scale"] * out, dk=dk, dv=dv, ds0=dS)
