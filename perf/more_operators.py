"""What a training program asks of the operators around a gated memory, as cases that can be timed and checked.

A gated linear recurrence is a policy's memory (whole sequences in training, one step of every environment while acting), a root-mean-square
norm with the residual's addition stands before and behind it, and the Muon step trains the matrices between them.  The sizes are those of the
repository's workloads (64 and 4096 environments, 24 steps, memories 256 wide, layers of 512, 256 and 128, 235 observations, a quarter of the
environments per minibatch), long sequences of a few environments, and irregular sizes between them.  With `own` false, `run` computes the same
in elementary torch operations.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-5
E4M3_MAX = 448.0
NS = (3.4445, -4.7750, 2.0315)     # coefficients of the Newton-Schulz step
NETS = "48x512,512x256,256x128,128x12,48x512,512x256,256x128,128x1"


# ---- the cases ------------------------------------------------------------------------------------------------------
def listed():
    return [
        # acting in a small run or an evaluation: one step of 64 environments, latency counts
        dict(name="step_64", kind="step", N=64, D=256, dtype="fp32", done_p=0.02),
        # a whole roll-out of the standard training run through the memory, from the states that its first step started from
        dict(name="forward_rollout", kind="forward", T=24, N=4096, D=256, dtype="fp32", done_p=0.01, s0=True, ragged=False),
        # a long history of four environments in bf16
        dict(name="forward_long", kind="forward", T=8192, N=4, D=1024, dtype="bf16", done_p=0.0, s0=False, ragged=False),
        # gradients of one minibatch of the standard training run: a quarter of the environments, all steps
        dict(name="backward_rollout", kind="backward", T=24, N=1024, D=256, dtype="fp32", done_p=0.01, s0=True, ragged=False),
        # gradients over long sequences in bf16
        dict(name="backward_long", kind="backward", T=4096, N=4, D=1024, dtype="bf16", done_p=0.0, s0=False, ragged=False),
        # gradients of padded trajectories of different lengths, sizes that fit no tile
        dict(name="backward_ragged", kind="backward", T=777, N=37, D=203, dtype="fp16", done_p=0.004, s0=True, ragged=True),
        # the norm behind the memory while a small run acts
        dict(name="norm_64", kind="norm", rows=64, cols=256, dtype="fp32", residual=True, e4m3=False),
        # the norm over every step of the standard roll-out, its output kept in a byte a value
        dict(name="norm_rollout_e4m3", kind="norm", rows=98304, cols=512, dtype="bf16", residual=True, e4m3=True),
        # gradients of the norm of height-scan observations over one minibatch
        dict(name="norm_backward_rough", kind="norm_backward", rows=24576, cols=235, dtype="fp32", residual=True),
        # one optimiser step of the standard actor and critic
        dict(name="muon_nets", kind="muon", shapes=NETS, steps=5),
        # matrices that fit no tile, tall and wide
        dict(name="muon_ragged", kind="muon", shapes="777x333,235x512,333x1001,30x100", steps=5),
        # one large matrix
        dict(name="muon_large", kind="muon", shapes="2048x4096", steps=5),
    ]


def draw(rng):
    spread = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    kind = rng.choice(["step", "forward", "forward", "backward", "backward", "norm", "norm_backward", "muon", "muon"])
    dtype = rng.choice(["fp32", "fp32", "bf16", "fp16"])
    most = [work(c) for c in listed() if c["kind"] == kind]
    if kind == "step":
        most = [dict(bytes=1e8, flops=1e9)]                       # up to 8192 environments
    while True:
        if kind == "step":
            c = dict(kind=kind, N=spread(64, 8192), D=rng.choice([128, 256, 512, rng.randint(24, 1024)]), dtype=dtype, done_p=rng.choice([0.0, 0.01]))
        elif kind in ("forward", "backward"):
            T, ragged = spread(8, 8192), rng.random() < 0.35
            c = dict(kind=kind, T=T, N=spread(2, 4096), D=rng.choice([128, 256, 512, 1024, rng.randint(24, 1024)]), dtype=dtype,
                     done_p=rng.choice([0.0, 0.01, 1.0 / T]), s0=rng.random() < 0.5, ragged=ragged)
            if T * c["N"] < 1024:
                continue
        elif kind == "muon":
            dim = lambda: rng.choice([128, 256, 512, spread(12, 2048)])  # noqa: E731
            c = dict(kind=kind, shapes=",".join("%dx%d" % (dim(), dim()) for _ in range(rng.randint(1, 12))), steps=5)
        else:
            c = dict(kind=kind, rows=spread(64, 131072), cols=spread(24, 8192), dtype=dtype, residual=rng.random() < 0.7)
            if kind == "norm":
                c["e4m3"] = rng.random() < 0.4
        w = work(c)
        if all(w[m] <= max(x[m] for x in most) for m in w):
            return c


def _shapes(case):
    return [tuple(int(n) for n in s.split("x")) for s in case["shapes"].split(",")]


def work(case):
    kind = case["kind"]
    if kind == "muon":
        flops = sum(case["steps"] * (3 * min(s) ** 2 * max(s) + min(s) ** 3) for s in _shapes(case))     # symmetric products by half
        return {"bytes": sum(20 * a * b for a, b in _shapes(case)), "flops": flops}
    size = torch.empty(0, dtype=TYPES[case["dtype"]]).element_size()
    if kind.startswith("norm"):
        n, more = case["rows"] * case["cols"], 1 if case["residual"] else 0
        if kind == "norm":
            y = n + 4 * case["rows"] if case["e4m3"] else n * size
            return {"bytes": n * size * (1 + 2 * more) + y + 4 * case["rows"] + 4 * case["cols"], "flops": n * 6}
        return {"bytes": n * size * (3 + more) + 4 * case["rows"] + 8 * case["cols"], "flops": n * 10}
    N, D = case["N"], case["D"]
    if kind == "step":
        return {"bytes": N * D * (3 * size + 8) + N, "flops": 10 * N * D}
    tokens, all_tokens = N * D * case["T"] * (0.5 if case["ragged"] else 1.0), N * D * case["T"]       # lengths are uniform
    states = 4 * N * D * (2 if case["s0"] else 1)
    if kind == "forward":
        return {"bytes": size * (2 * tokens + all_tokens) + states, "flops": 10 * tokens}
    return {"bytes": size * (3 * tokens + 2 * all_tokens) + states + 4 * N * D, "flops": 25 * tokens}


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _inputs(case, seed):
    """Everything that the case's arithmetic depends on, on the GPU, from the seed alone."""
    g = torch.Generator("cuda")
    g.manual_seed(1000003 * seed + 29)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    kind = case["kind"]
    if kind == "muon":
        # weights, gradients and momenta of all matrices in one flat buffer each
        n = sum(a * b for a, b in _shapes(case))
        w, grad, m = 0.05 * normal(n), 1e-3 * normal(n), 5e-3 * normal(n)
        at, mats = 0, []
        for a, b in _shapes(case):
            mats.append(tuple(t[at:at + a * b].view(a, b) for t in (w, grad, m)))
            at += a * b
        return dict(mats=mats, lr=0.02, beta=0.95, decay=0.01, scales=[math.sqrt(max(1.0, b / a)) for a, b in _shapes(case)])
    dt = TYPES[case["dtype"]]
    if kind.startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        x = (normal(rows, cols) * (0.5 + 2 * torch.rand(rows, 1, generator=g, device="cuda"))).to(dt)
        return dict(x=x, residual=normal(rows, cols).to(dt) if case["residual"] else None, dy=normal(rows, cols).to(dt), weight=1 + 0.2 * normal(cols))
    step = kind == "step"
    T, N, D = 1 if step else case["T"], case["N"], case["D"]
    # one product makes candidates and gates of a step side by side; memories of about 2 to 250 steps
    xg = normal(T, N, 2 * D)
    xg[..., D:] += torch.linspace(0, 5.5, D, device="cuda")
    xg = xg.to(dt)
    i = dict(x=xg[..., :D], g=xg[..., D:])
    i["dones"] = (torch.rand(T, N, generator=g, device="cuda") < case["done_p"]).to(torch.uint8) if case["done_p"] else None
    i["s0"] = normal(N, D) if step or case["s0"] else None
    i["lengths"] = None
    if not step and case["ragged"]:
        i["lengths"] = torch.randint(0, T + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
        i["lengths"][0] = T
    if kind == "backward":
        i["dh"], i["ds_last"] = normal(T, N, D).to(dt), normal(N, D)
    return i


def prepare(case, seed):
    """Inputs, and the buffers and workspace that a program keeps from call to call."""
    i = _inputs(case, seed)
    s = dict(case=dict(case), i=i)
    new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    kind = case["kind"]
    if kind == "muon":
        s["out"] = [(torch.empty_like(w), torch.empty_like(m)) for w, _, m in i["mats"]]
    elif kind.startswith("norm"):
        rows, cols, dt = case["rows"], case["cols"], TYPES[case["dtype"]]
        if kind == "norm":
            s["total"] = new(rows, cols, dtype=dt) if case["residual"] else None
            s["y"] = new(rows, cols, dtype=torch.float8_e4m3fn if case["e4m3"] else dt)
            s["scales"], s["rstd"] = new(rows), new(rows)
        else:
            s["rstd"] = i["x"].float().square().mean(1).add(EPS).rsqrt()
            s["dx"], s["dweight"] = new(rows, cols, dtype=dt), new(cols)
    else:
        T, N, D, dt = case.get("T", 1), case["N"], case["D"], TYPES[case["dtype"]]
        s["state"] = new(N, D)
        for name in ("dx", "dg") if kind == "backward" else ("h",):
            s[name] = new(T, N, D, dtype=dt)
    if own:
        import paper_2509_10771_amd as rx
        s["rx"] = rx
        if kind == "muon":
            s["muon"] = rx.Muon([(w, wo, g, m, mo, k) for (w, g, m), (wo, mo), k in zip(i["mats"], s["out"], i["scales"])], lr=i["lr"], momentum=i["beta"],
                                nesterov=True, weight_decay=i["decay"], steps=case["steps"])
            s["ws"] = rx.workspace(rx.rslx_muon_step_workspace_bytes(s["muon"]))
        elif kind == "norm_backward":
            s["ws"] = rx.workspace(rx.rslx_rms_norm_backward_workspace_bytes(case["rows"], case["cols"]))
        elif kind != "norm":
            step = kind == "step"
            s["gr"] = rx.GatedRec(dt, T, N, D, None if step else i["dones"], i["lengths"])
            if kind == "forward":
                s["ws"] = rx.workspace(rx.rslx_gated_recurrence_workspace_bytes(s["gr"]))
            elif kind == "backward":
                s["ws"] = rx.workspace(rx.rslx_gated_recurrence_backward_workspace_bytes(s["gr"]))
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    rx, i, kind = s["rx"], s["i"], s["case"]["kind"]
    if kind == "muon":
        rx.rslx_muon_step(s["muon"], s["ws"])
        return dict(w=[w for w, _ in s["out"]], m=[m for _, m in s["out"]])
    if kind == "norm":
        if s["case"]["e4m3"]:
            rx.rslx_rms_norm_e4m3(i["x"], i["residual"], i["weight"], EPS, s["total"], s["y"], s["scales"], s["rstd"])
            out = dict(y=s["y"], scales=s["scales"], rstd=s["rstd"])
        else:
            rx.rslx_rms_norm(i["x"], i["residual"], i["weight"], EPS, s["total"], s["y"], s["rstd"])
            out = dict(y=s["y"], rstd=s["rstd"])
        return dict(out, total=s["total"]) if i["residual"] is not None else out
    if kind == "norm_backward":
        rx.rslx_rms_norm_backward(i["dy"], i["x"], i["weight"], s["rstd"], i["residual"], s["dx"], s["dweight"], s["ws"])
        return dict(dx=s["dx"], dweight=s["dweight"])
    if kind == "step":
        rx.rslx_gated_recurrence_step(s["gr"], i["x"], i["g"], i["dones"], i["s0"], s["state"], s["h"])
        return dict(h=s["h"], state=s["state"])
    if kind == "forward":
        rx.rslx_gated_recurrence(s["gr"], i["x"], i["g"], i["s0"], s["h"], s["state"], s["ws"])
        return dict(h=s["h"], state=s["state"])
    rx.rslx_gated_recurrence_backward(s["gr"], i["x"], i["g"], i["s0"], i["dh"], i["ds_last"], s["dx"], s["dg"], s["state"], s["ws"])
    return dict(dx=s["dx"], dg=s["dg"], ds0=s["state"])


def _run_plain(s):
    i, case = s["i"], s["case"]
    kind = case["kind"]
    if kind == "muon":
        return _muon_plain(s)
    dt = TYPES[case["dtype"]]
    if kind == "norm":
        z = i["x"].float()
        if i["residual"] is not None:
            z = z + i["residual"].float()
        rstd = (z * z).mean(1).add(EPS).rsqrt()
        y = z * rstd[:, None] * i["weight"]
        if case["e4m3"]:
            scales = y.abs().amax(1) / E4M3_MAX
            out = dict(y=(y / scales[:, None]).to(torch.float8_e4m3fn), scales=scales, rstd=rstd)
        else:
            out = dict(y=y.to(dt), rstd=rstd)
        return dict(out, total=z.to(dt)) if i["residual"] is not None else out
    if kind == "norm_backward":
        dy, rstd = i["dy"].float(), s["rstd"][:, None]
        h, k = i["x"].float() * rstd, dy * i["weight"]
        dx = rstd * (k - h * (k * h).mean(1, keepdim=True))
        if i["residual"] is not None:
            dx = dx + i["residual"].float()
        return dict(dx=dx.to(dt), dweight=(dy * h).sum(0))
    x, g = i["x"].float(), i["g"].float()
    e = torch.exp(-g.abs())
    low, high = e / (1 + e), 1 / (1 + e)
    f, f1 = torch.where(g >= 0, high, low), torch.where(g >= 0, low, high)     # sigmoid(g) and 1 - sigmoid(g)
    if kind == "step":
        before = i["s0"] if i["dones"] is None else torch.where(i["dones"][0].bool()[:, None], torch.zeros_like(i["s0"]), i["s0"])
        state = f[0] * before + f1[0] * x[0]
        return dict(h=state[None].to(dt), state=state)
    T, N, D = x.shape
    there = None
    keep = torch.ones(T, N, 1, device="cuda") if i["dones"] is None else 1.0 - i["dones"].float()[..., None]
    if i["lengths"] is not None:                                                # steps that do not exist hand the state on
        there = (torch.arange(T, device="cuda")[:, None] < i["lengths"].long()[None])[..., None]
        f, f1 = torch.where(there, f, torch.ones_like(f)), torch.where(there, f1, torch.zeros_like(f1))
        keep = torch.where(there, keep, torch.ones_like(keep))
    s0 = torch.zeros(N, D, device="cuda") if i["s0"] is None else i["s0"]
    before = torch.cat([torch.ones_like(keep[:1]), keep[:-1]])
    b = f1 * x
    b[0] += f[0] * s0
    h = _scan(f * before, b)
    if kind == "forward":
        out = h if there is None else torch.where(there, h, torch.zeros_like(h))
        return dict(h=out.to(dt), state=keep[-1] * h[-1])
    dh = i["dh"].float()
    if there is not None:
        dh = torch.where(there, dh, torch.zeros_like(dh))
    dh = dh.clone()
    dh[-1] += keep[-1] * i["ds_last"]
    d = _scan(torch.cat([keep[:-1] * f[1:], torch.ones_like(f[:1])]).flip(0), dh.flip(0)).flip(0)
    entered = torch.cat([s0[None], keep[:-1] * h[:-1]])
    dx, dg = f1 * d, d * f * f1 * (entered - x)
    return dict(dx=dx.to(dt), dg=dg.to(dt), ds0=f[0] * d[0])


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t over the first dimension, h_{-1} = 0, by doubling."""
    T, d = a.shape[0], 1
    while d < T:
        b = torch.cat([b[:d], b[d:] + a[d:] * b[:-d]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _muon_plain(s):
    i = s["i"]
    ws, ms = [], []
    for (w, grad, m), scale in zip(i["mats"], i["scales"]):
        m = i["beta"] * m + grad
        u = grad + i["beta"] * m
        x = u / (u * u).sum().sqrt()
        tall = x.shape[0] > x.shape[1]
        if tall:
            x = x.t()
        for _ in range(s["case"]["steps"]):
            a = x @ x.t()
            x = NS[0] * x + (NS[1] * a + NS[2] * (a @ a)) @ x
        ws.append((1 - i["lr"] * i["decay"]) * w - i["lr"] * scale * (x.t() if tall else x))
        ms.append(m)
    return dict(w=ws, m=ms)


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------
def exact(case, seed):
    i, kind = _inputs(case, seed), case["kind"]
    if kind == "muon":
        ws, ms = [], []
        for (w, grad, m), scale in zip(i["mats"], i["scales"]):
            grad = grad.double()
            m = i["beta"] * m.double() + grad
            x = grad + i["beta"] * m
            x = x / torch.linalg.matrix_norm(x)
            wide = x.shape[0] < x.shape[1]
            for _ in range(case["steps"]):
                # from the other side of the product: X (a + b X^T X + c (X^T X)^2), term by term
                r = (lambda y: x @ (x.t() @ y)) if wide else (lambda y: (y @ x.t()) @ x)
                first = r(x)
                x = NS[0] * x + NS[1] * first + NS[2] * r(first)
            ws.append(w.double() * (1 - i["lr"] * i["decay"]) - i["lr"] * scale * x)
            ms.append(m)
        return dict(w=ws, m=ms)
    if kind.startswith("norm"):
        x, w = i["x"].double(), i["weight"].double()
        n = x.shape[1]
        if kind == "norm":
            z = x if i["residual"] is None else x + i["residual"].double()
            r = 1.0 / torch.sqrt((z ** 2).sum(1) / n + EPS)
            y = z * w * r[:, None]
            if case["e4m3"]:
                scales = y.abs().max(1).values / E4M3_MAX
                out = dict(y=y / scales[:, None], scales=scales, rstd=r)
            else:
                out = dict(y=y, rstd=r)
            return dict(out, total=z) if i["residual"] is not None else out
        # through the mean of the squares
        dy = i["dy"].double()
        r = 1.0 / torch.sqrt((x ** 2).sum(1, keepdim=True) / n + EPS)
        dr = (dy * w * x).sum(1, keepdim=True)
        dx = dy * w * r - dr * r ** 3 * x / n
        return dict(dx=dx if i["residual"] is None else dx + i["residual"].double(), dweight=(dy * x * r).sum(0))
    T = 1 if kind == "step" else case["T"]
    N, D = case["N"], case["D"]
    if T * N * D > 4e8:
        return None
    gate = lambda t: torch.sigmoid(i["g"][t].double())  # noqa: E731
    rest = lambda t: torch.sigmoid(-i["g"][t].double())  # noqa: E731
    ends = torch.zeros(T, N, dtype=torch.bool, device="cuda") if i["dones"] is None else i["dones"].bool()
    h = torch.zeros(N, D, dtype=torch.float64, device="cuda") if i["s0"] is None else i["s0"].double()
    if kind == "step":
        h = h.masked_fill(ends[0][:, None], 0.0) * gate(0) + rest(0) * i["x"][0].double()
        return dict(h=h[None], state=h)
    length = torch.full((N,), T, device="cuda") if i["lengths"] is None else i["lengths"].long()
    back = kind == "backward"
    out = torch.zeros(T, N, D, dtype=torch.float64, device="cuda")              # outputs, or the states that steps start from
    for t in range(T):
        here = (t < length)[:, None]
        new = gate(t) * h + rest(t) * i["x"][t].double()
        out[t] = h if back else new * here
        h = torch.where(here, new.masked_fill(ends[t][:, None], 0.0), h)
    if not back:
        return dict(h=out, state=h)
    dx, dg = (torch.zeros(T, N, D, dtype=torch.float64, device="cuda") for _ in range(2))
    d = i["ds_last"].double()                                                    # of the state behind step t
    for t in range(T - 1, -1, -1):
        here = (t < length)[:, None]
        new = d.masked_fill(ends[t][:, None], 0.0) + i["dh"][t].double()
        f = gate(t)
        dx[t] = rest(t) * new * here
        dg[t] = new * (out[t] - i["x"][t].double()) * f * rest(t) * here
        d = torch.where(here, new * f, d)
    return dict(dx=dx, dg=dg, ds0=d)
