"""The ends of a training step, and of scoring, around the routed stack: what is timed and compared.

Three operators: the language-model loss over a large vocabulary with its gradients (`hero_lm_loss`), the final
RMSNorm before it with its backward (`hero_final_norm`, `hero_final_norm_backward`), and the clipping of all router
and adapter gradients by their global norm (`hero_grad_clip`, `hero_grad_norm`).  `run` computes them in elementary
torch operations, or, where `own` is true, through the binding's entry points.

Shapes are those of the repository's workloads (Llama-3.1-8B, Llama-2-13B, the tiny fp32 stack, the rank-896
adapters) and generic ones.  Hidden rows are noise plus a share of their target's head row, so that the tokens' losses
spread from those of a sure model to those of a lost one; targets follow instruction tuning, where the prompt at the
head of each sequence carries none (-1).  Gradients are Gaussians whose scale differs from tensor to tensor.
"""
import math

import torch

own = False

DEV = "cuda:0"
SEQ = 2048        # tokens of one training sequence
EPS_NORM = 1e-5
ROUTER = dict(d_e=256, d_h=48, d_a=16, d_p=64, d_m=128, d_s=64, d_head=256)
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _loss(name, T, d, vocab, dtype="bf16", keep=1.0, dx=True, dw=False, mean=True):
    return dict(name=name, op="lm_loss", T=T, d=d, vocab=vocab, dtype=dtype, keep=keep, dx=dx, dw=dw, mean=mean)


def _norm(name, T, d, dtype="bf16", backward=False, dgain=False):
    return dict(name=name, op="final_norm", T=T, d=d, dtype=dtype, backward=backward, dgain=dgain)


def _clip(name, d, d_r, layers, dtype="f32", max_norm=1.0, clip=True, odd=0):
    return dict(name=name, op="grad_clip", d=d, d_r=d_r, layers=layers, dtype=dtype, max_norm=max_norm, clip=clip, odd=odd)


def listed():
    return [
        # one decoded token's log-likelihood (latency, and one pass over a small head)
        _loss("score_1_token", 1, 2048, 32000, dx=False, mean=False),
        # the tiny fp32 stack's training step, a vocabulary of odd size, head trained along
        _loss("step_f32_64_tokens", 64, 256, 2003, dtype="f32", dw=True),
        # a short sequence's gradient: few rows against the whole head
        _loss("step_8b_96_tokens", 96, 4096, 128256),
        # perplexity of a prompt: per-token losses, no gradient
        _loss("score_8b_1000_tokens", 1000, 4096, 128256, dx=False, mean=False),
        # a ragged batch at a small width, odd vocabulary, a third of the tokens prompt, head trained along
        _loss("step_ragged_1777_tokens", 1777, 1024, 50257, keep=0.66, dw=True),
        # instruction tuning with the frozen head of the 8B backbone: half of the tokens are prompt
        _loss("step_8b_4096_tokens", 4096, 4096, 128256, keep=0.5),
        # the largest: four sequences of 2048 that all count
        _loss("step_8b_8192_tokens", 8192, 4096, 128256),
        # the norm of one decoded token
        _norm("norm_8b_1_token", 1, 4096),
        # backward of the norm over a batch at the 13B width, its gain trained along
        _norm("norm_backward_13b_8192", 8192, 5120, backward=True, dgain=True),
        # gradients of the tiny fp32 stack: many small tensors
        _clip("clip_tiny", 256, 16, 4),
        # router and adapters of the 8B workload, 32 layers of rank 64
        _clip("clip_8b_rank64", 4096, 64, 32),
        # the rank-896 operating point in 16 layers, with one tensor of odd size
        _clip("clip_8b_rank896", 4096, 896, 16, odd=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lm_loss", "lm_loss", "final_norm", "grad_clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "lm_loss":
        T, d, vocab = _log(rng, 1, 8192), 256 * _log(rng, 1, 20), _log(rng, 1000, 128256)
        dx, dw = rng.choice([(False, False), (True, False), (True, False), (True, True), (False, True)])
        most = 2.0e12 if dtype == "f32" else 8.0e12   # products of one pass: at most those of the largest listed case
        T = max(1, min(T, int(most / (2.0 * vocab * d * (1 + dx + dw)))))
        c = _loss("", T, d, vocab, dtype, rng.choice([1.0, 0.9, 0.5, 0.2]), dx, dw, rng.random() < 0.7)
    elif op == "final_norm":
        backward = rng.random() < 0.6
        c = _norm("", _log(rng, 1, 8192), 256 * _log(rng, 1, 20), dtype, backward, backward and rng.random() < 0.5)
    else:
        c = _clip("", 256 * _log(rng, 1, 16), 32 * _log(rng, 1, 28), rng.randint(1, 16), dtype, _log(rng, 1, 1000) / 100.0,
                  rng.random() < 0.7, rng.choice([0, 1, 3, 77]))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _targets(case, g):
    """Targets, -1 over the prompt of each sequence; the share that counts is exact."""
    T = case["T"]
    y = torch.randint(0, case["vocab"], (T,), generator=g, device=DEV, dtype=torch.int32)
    pos = torch.arange(T, device=DEV)
    length = torch.where(pos // SEQ < T // SEQ, SEQ, T % SEQ)
    return torch.where(pos % SEQ < (length * (1.0 - case["keep"])).floor(), torch.full_like(y, -1), y)


def _counted(case):
    T, lost = case["T"], lambda n: math.floor(n * (1.0 - case["keep"]))
    return T - (T // SEQ) * lost(SEQ) - lost(T % SEQ)


def _grad_shapes(case):
    """Router, adapters (W_1, W_2 of every layer) and the layers' decays; the last one with `odd` elements more."""
    d, r, R = case["d"], case["d_r"], ROUTER
    router = [(R["d_e"], d), (R["d_h"], R["d_e"]), (R["d_p"], 6), (R["d_a"], R["d_p"])] + 4 * [(R["d_m"], R["d_s"])] + [
        (R["d_m"], R["d_m"]), (R["d_head"], (R["d_s"] + R["d_m"] + 8) // 8 * 8), (R["d_head"],), (R["d_head"], d), (R["d_head"],)]
    return router + case["layers"] * [(r, d), (d, r)] + [(case["layers"] + case["odd"],)]


def _offsets(sizes):
    """Each tensor's place in one buffer, at multiples of 64 elements, and the buffer's length."""
    at, starts = 0, []
    for n in sizes:
        starts.append(at)
        at += (n + 63) // 64 * 64
    return starts, at


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rnd = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    if case["op"] == "lm_loss":
        T, d, V, dt = case["T"], case["d"], case["vocab"], DT[case["dtype"]]
        w = rnd(V, d).mul_(1.5 / math.sqrt(d)).to(dt)
        y = _targets(case, g)
        share = 10.0 * torch.rand(T, 1, generator=g, device=DEV)
        x = rnd(T, d) + share / 1.5 * w[y.clamp(min=0).long()].float()
        x = x * torch.rsqrt(x.square().mean(1, keepdim=True)) * (0.75 + 0.5 * torch.rand(d, generator=g, device=DEV))
        s = dict(case=case, w=w, x=x.to(dt), y=y)
        if case["dx"] and not case["dw"]:   # a frozen head is laid out once: its transpose, rows padded to 64 with zeros
            s["w_t"] = torch.zeros(d, (V + 63) // 64 * 64, dtype=dt, device=DEV)
            s["w_t"][:, :V] = w.t()
        return s
    if case["op"] == "final_norm":
        T, d, dt = case["T"], case["d"], DT[case["dtype"]]
        s = dict(case=case, h=(rnd(T, d) * (0.5 + 4.0 * torch.rand(T, 1, generator=g, device=DEV))).to(dt),
                 gain=(0.75 + 0.5 * torch.rand(d, generator=g, device=DEV)).to(dt))
        if case["backward"]:
            s["dx"] = (rnd(T, d) * (1e-3 * torch.rand(T, 1, generator=g, device=DEV))).to(dt)
        return s
    # scales from 1e-6 to 1e-2: the global norm of a large model's lands on either side of the usual limits
    dt = DT[case["dtype"]]
    grads = [rnd(*shape).mul_(10.0 ** (-6.0 + 4.0 * float(torch.rand((), generator=g, device=DEV)))).to(dt)
             for shape in _grad_shapes(case)]
    return dict(case=case, grads=grads)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    if own:
        return _own(state)
    return {"lm_loss": _plain_loss, "final_norm": _plain_norm, "grad_clip": _plain_clip}[state["case"]["op"]](state)


def _plain_loss(s):
    case, V = s["case"], s["case"]["vocab"]
    counts = (s["y"] >= 0) & (s["y"] < V)
    rows = counts.nonzero()[:, 0]
    x, w, y = s["x"][rows].float(), s["w"].float(), s["y"][rows].long()
    logits = x @ w.t()
    m = logits.max(1, keepdim=True).values
    e = (logits - m).exp()
    z = e.sum(1, keepdim=True)
    nll = (z.log() + m)[:, 0] - logits.gather(1, y[:, None])[:, 0]
    share = 1.0 / max(1, rows.numel()) if case["mean"] else 1.0
    token = torch.zeros(case["T"], device=DEV)
    token[rows] = nll
    out = {"loss": (nll.double().sum() * share).float().reshape(1), "token_loss": token}
    if case["dx"] or case["dw"]:
        p = e.div_(z)
        p[torch.arange(rows.numel(), device=DEV), y] -= 1.0
        p *= share
        if case["dx"]:
            dx = torch.zeros(case["T"], case["d"], device=DEV)
            dx[rows] = p @ w
            out["dx"] = dx.to(s["x"].dtype)
        if case["dw"]:
            out["dw"] = (p.t() @ x).to(s["w"].dtype)
    return out


def _plain_norm(s):
    h, gain = s["h"].float(), s["gain"].float()
    r = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS_NORM)
    if not s["case"]["backward"]:
        return {"x": (h * r * gain).to(s["h"].dtype)}
    dx = s["dx"].float()
    u = dx * gain
    out = {"dh": (r * (u - h * r * r * (h * u).mean(1, keepdim=True))).to(s["h"].dtype)}
    if s["case"]["dgain"]:
        out["dgain"] = (dx.double() * (h * r).double()).sum(0).float()
    return out


def _plain_clip(s):
    case, grads = s["case"], s["grads"]
    norm = torch.stack([g.double().square().sum() for g in grads]).sum().sqrt()
    out = {"norm": norm.float().reshape(1)}
    if case["clip"]:
        c = (case["max_norm"] / norm).clamp(max=1.0).float()
        out["grads"] = torch.cat([torch.nn.functional.pad((g.float() * c).to(g.dtype).reshape(-1), (0, -g.numel() % 64))
                                  for g in grads])
    return out


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _dims(case, H):
    return H.hero_dims(d=case["d"], d_ff=2 * case["d"], d_r=64, L_R=32, dtype=H.HERO_BF16 if case["dtype"] == "bf16" else H.HERO_F32,
                       eps_norm=EPS_NORM, eps=1e-6, T_hist=0.9, **ROUTER)


def _own(s):
    from paper_2609_08189_amd import hero as H
    case, stream = s["case"], torch.cuda.current_stream().cuda_stream
    plan = s.get("plan")
    if plan is None:   # structs, output buffers and workspace, as a program keeps them for its shapes
        plan = s["plan"] = {"lm_loss": _loss_plan, "final_norm": _norm_plan, "grad_clip": _clip_plan}[case["op"]](s, H)
    out, ws = plan["out"], plan["ws"]
    if case["op"] == "lm_loss":
        if case["dx"] and case["dw"]:   # a trained head changes from step to step, and its transposed copy with it
            H.check(H.hero_lm_head_weights_make(plan["dims"], case["vocab"], s["w"], plan["w_t"], stream), "hero_lm_head_weights_make")
        H.check(H.hero_lm_loss(plan["dims"], case["vocab"], case["T"], s["x"], plan["head"], s["y"],
                               H.HERO_LOSS_MEAN if case["mean"] else H.HERO_LOSS_SUM, 1.0, plan["outs"], ws, ws.numel(), stream),
                "hero_lm_loss")
    elif case["op"] == "final_norm" and case["backward"]:
        H.check(H.hero_final_norm_backward(plan["dims"], case["T"], s["h"], s["dx"], s["gain"], out["dh"], out.get("dgain"), ws,
                                           ws.numel(), stream), "hero_final_norm_backward")
    elif case["op"] == "final_norm":
        H.check(H.hero_final_norm(plan["dims"], case["T"], s["h"], s["gain"], out["x"], stream), "hero_final_norm")
    elif case["clip"]:
        H.check(H.hero_grad_clip(plan["tensors"], case["max_norm"], out["norm"], ws, ws.numel(), stream), "hero_grad_clip")
    else:
        H.check(H.hero_grad_norm(plan["tensors"], out["norm"], ws, ws.numel(), stream), "hero_grad_norm")
    return out


def _bytes(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)


def _loss_plan(s, H):
    case, dims = s["case"], _dims(s["case"], H)
    out = {"loss": torch.empty(1, device=DEV), "token_loss": torch.empty(case["T"], device=DEV)}
    if case["dx"]:
        out["dx"] = torch.empty_like(s["x"])
    if case["dw"]:
        out["dw"] = torch.empty_like(s["w"])
    w_t = s.get("w_t")
    if case["dx"] and w_t is None:
        w_t = torch.empty(case["d"], (case["vocab"] + 63) // 64 * 64, dtype=s["w"].dtype, device=DEV)
    outs = H.hero_lm_loss_out(*[H.ptr(out.get(k)) for k in ("loss", "token_loss", "dx", "dw")])
    return dict(dims=dims, out=out, outs=outs, w_t=w_t, head=H.hero_lm_head(H.ptr(s["w"]), H.ptr(w_t)),
                ws=_bytes(H.hero_lm_loss_workspace_size(dims, case["vocab"], case["T"], case["dx"], case["dw"])))


def _norm_plan(s, H):
    case, dims = s["case"], _dims(s["case"], H)
    if not case["backward"]:
        return dict(dims=dims, out={"x": torch.empty_like(s["h"])}, ws=None)
    out = {"dh": torch.empty_like(s["h"])}
    if case["dgain"]:
        out["dgain"] = torch.empty(case["d"], device=DEV)
    return dict(dims=dims, out=out, ws=_bytes(H.hero_final_norm_backward_workspace_size(dims, case["T"])))


def _clip_plan(s, H):
    case, grads = s["case"], s["grads"]
    out = {"norm": torch.empty(1, device=DEV)}
    starts, total = _offsets([g.numel() for g in grads])
    if case["clip"]:
        out["grads"] = torch.zeros(total, dtype=grads[0].dtype, device=DEV)
    at = lambda i: H.ptr(out["grads"]) + starts[i] * grads[0].element_size() if case["clip"] else None  # noqa: E731
    kind = H.HERO_BF16 if case["dtype"] == "bf16" else H.HERO_F32
    tensors = H.hero_grad_tensors([(H.ptr(g), at(i), g.numel(), kind) for i, g in enumerate(grads)])
    return dict(out=out, tensors=tensors, ws=_bytes(H.hero_grad_norm_workspace_size(tensors)))


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its values in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "lm_loss":
        T, d, V, n = case["T"], case["d"], case["vocab"], _counted(case)
        products = 1 + case["dx"] + case["dw"]
        return {"bytes": es * (n * d + V * d + T * d * case["dx"] + V * d * case["dw"]) + 8 * T + 4,
                "flops": 2.0 * n * V * d * products}
    if case["op"] == "final_norm":
        T, d = case["T"], case["d"]
        return {"bytes": es * (T * d * (3 if case["backward"] else 2) + d) + 4 * d * case["dgain"],
                "flops": T * d * (8.0 if case["backward"] else 4.0)}
    n = sum(math.prod(shape) for shape in _grad_shapes(case))
    return {"bytes": es * n * (2 if case["clip"] else 1) + 4, "flops": n * (3.0 if case["clip"] else 2.0)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "lm_loss":
        V, T = case["vocab"], case["T"]
        y = s["y"].long()
        live = ((y >= 0) & (y < V)).double()
        n = float(live.sum())
        unit = case["mean"] and 1.0 / max(n, 1.0) or 1.0
        X, W = s["x"].double(), s["w"].double()
        L = torch.mm(X, W.T.contiguous())
        lse = torch.logsumexp(L, dim=1)
        hot = torch.arange(T, device=DEV), y.clamp(0, V - 1)
        nll = torch.where(live > 0, lse - L[hot], torch.zeros_like(lse))
        out = {"loss": (nll.sum() * unit).reshape(1), "token_loss": nll}
        G = torch.exp(L - lse[:, None])
        G[hot] = torch.expm1(L[hot] - lse)
        G *= (live * unit)[:, None]
        if case["dx"]:
            out["dx"] = torch.mm(G, W)
        if case["dw"]:
            out["dw"] = torch.mm(G.T.contiguous(), X)
        return out
    if case["op"] == "final_norm":
        h, w, d = s["h"].double(), s["gain"].double(), case["d"]
        rms = (h.pow(2).sum(1) / d + EPS_NORM).sqrt()[:, None]
        if not case["backward"]:
            return {"x": w * h / rms}
        dx = s["dx"].double()
        out = {"dh": w * dx / rms - h * ((w * dx * h).sum(1)[:, None] / (d * rms ** 3))}
        if case["dgain"]:
            out["dgain"] = torch.einsum("td,td->d", dx, h / rms)
        return out
    flat = [g.double().flatten() for g in s["grads"]]
    norm = math.sqrt(sum(float(torch.dot(v, v)) for v in flat))
    out = {"norm": torch.tensor([norm], dtype=torch.float64)}
    if case["clip"]:
        starts, total = _offsets([v.numel() for v in flat])
        out["grads"] = torch.zeros(total, dtype=torch.float64, device=DEV)
        for at, v in zip(starts, flat):
            out["grads"][at:at + v.numel()] = v * (case["max_norm"] / norm if norm > case["max_norm"] else 1.0)
    return out
