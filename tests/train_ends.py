"""The ends of a training step on the GPU for the tests: buffers, calls and error bounds."""
import numpy as np
import torch

from paper_2609_08189_amd import hero as H

DEV = "cuda:0"
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}   # torch.finfo(dtype).eps / 2
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
GUARD = 4096                                          # bytes kept around every output


def dims(d, dtype="bf16", eps_norm=1e-5):
    return H.hero_dims(d=d, d_ff=2 * d, d_r=64, L_R=4, d_m=64, d_s=64, d_h=48, d_a=16, d_e=256, d_p=64, d_head=256,
                       dtype=H.HERO_BF16 if dtype == "bf16" else H.HERO_F32, eps_norm=eps_norm, eps=1e-6, T_hist=0.9)


def stream():
    return torch.cuda.current_stream().cuda_stream


class Guarded:
    """A tensor whose surroundings show a write out of its range; filled with 0xFF (NaN) first."""

    def __init__(self, shape, dtype):
        n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        self.n = n
        self.raw = torch.full((n + 2 * GUARD,), 0xFF, dtype=torch.uint8, device=DEV)
        self.t = self.raw[GUARD:GUARD + n].view(dtype).view(shape)

    def poison(self):
        self.raw.fill_(0xFF)

    def whole(self):
        r = self.raw
        return bool((r[:GUARD] == 0xFF).all()) and bool((r[GUARD + self.n:] == 0xFF).all())


def f64(t):
    return t.detach().cpu().double().numpy()


class Loss:
    """hero_lm_loss on given x [T][d], w [vocab][d] (torch, on the GPU) and targets."""

    def __init__(self, x, w, y, dx=True, dw=True, mean=True, scale=1.0):
        self.x, self.w, self.scale, self.mean = x, w, scale, mean
        self.T, self.d, self.V = x.shape[0], x.shape[1], w.shape[0]
        self.dtype = "bf16" if x.dtype == torch.bfloat16 else "f32"
        self.dims = dims(self.d, self.dtype)
        self.y = torch.as_tensor(np.asarray(y), dtype=torch.int32).to(DEV)
        self.out = {"loss": Guarded((1,), torch.float32), "token_loss": Guarded((self.T,), torch.float32)}
        if dx:
            self.out["dx"] = Guarded(tuple(x.shape), x.dtype)
        if dw:
            self.out["dw"] = Guarded(tuple(w.shape), w.dtype)
        self.w_t = None
        if dx:
            self.w_t = Guarded((self.d, (self.V + 63) // 64 * 64), w.dtype)
            H.check(H.hero_lm_head_weights_make(self.dims, self.V, w, self.w_t.t, stream()), "hero_lm_head_weights_make")
        self.ws = Guarded((H.hero_lm_loss_workspace_size(self.dims, self.V, self.T, dx, dw),), torch.uint8)
        p = lambda k: self.out[k].t.data_ptr() if k in self.out else None  # noqa: E731
        self.outs = H.hero_lm_loss_out(p("loss"), p("token_loss"), p("dx"), p("dw"))
        self.head = H.hero_lm_head(w.data_ptr(), self.w_t.t.data_ptr() if dx else None)

    def run(self):
        H.check(H.hero_lm_loss(self.dims, self.V, self.T, self.x, self.head, self.y,
                               H.HERO_LOSS_MEAN if self.mean else H.HERO_LOSS_SUM, self.scale, self.outs, self.ws.t,
                               self.ws.n, stream()), "hero_lm_loss")
        return self

    def results(self):
        torch.cuda.synchronize()
        for k, v in {**self.out, "ws": self.ws}.items():
            assert v.whole(), f"{k}: written out of range"
        return {k: f64(v.t) for k, v in self.out.items()}


def loss_bounds(x, w, y, scale, mean, dtype):
    """Bounds of |result - 64 bits| by the roundings on the way, from the same inputs in 64 bits.

    u: half a step of the stored exponentials and outputs; g = n 2^-24: n fp32 additions in any order.
      logit      d 2^-24 sum |x W|, of the column and of the target: a relative error of e = exp(l - ref); fp32 products
                 may be six bf16 products of three-term operands, six additions each (a: 6), that leave out 3 2^-24
      exp        a step or two, and the rounding of its argument: 2^-22 (|l - ref| + 4)
      S          the sum's order: at most V / 64 + 64 additions one after another
      dx         e stored in u, twice where a reference moved (a logit 60 above the target's); V additions
      dW         p stored in u, or e divided by its row's sum and stored a second time, and where a reference moved a
                 third; the target's p - 1 once; N additions
      below 2^-126 an exponential may be zero: e is at least one somewhere in each row's sum, so p loses at most 2^-126 a
                 column, dx 2^-126 sum |W| and dW 2^-126 sum |x| (times the unit), and a result itself at most 2^-126
    """
    u, s24, tiny = HALF_STEP[dtype], 2.0 ** -24, 2.0 ** -126
    a = 6 if dtype == "f32" else 1
    T, d = x.shape
    V = w.shape[0]
    rows = np.flatnonzero((y >= 0) & (y < V))
    n = len(rows)
    unit = abs(scale) / (max(n, 1) if mean else 1)
    tok, dx, dw = np.zeros(T), np.zeros((T, d)), np.zeros((V, d))
    if n == 0:
        return 0.0, tok, dx, dw
    xr, at = x[rows], (np.arange(n), y[rows])
    l = xr @ w.T
    lt = l[at]
    size = np.max(np.abs(xr) @ np.abs(w).T, axis=1)
    top = np.maximum(l.max(axis=1), lt)
    ref = np.where(top - lt > 59.0, top, lt)
    p = np.exp(l - top[:, None])
    z = p.sum(axis=1)
    p /= z[:, None]
    rest = 1.0 - p[at]
    eps = 2 * (a * d + 3) * s24 * size + 4 * s24 * (np.max(np.abs(l - ref[:, None]), axis=1) + 4)
    eps = np.expm1(eps) + (V / 64 + 64) * s24
    p[at] = 0.0
    nll = np.log(z) + top - lt
    tok[rows] = np.minimum(1.0, p.sum(axis=1) * 1.001 + 1e-30) * eps + 8 * s24 * np.abs(nll) + 2 * d * s24 * size * rest
    ue = u * np.where(top - lt > 59.0, 2.01, 1.01)
    dx[rows] = unit * (((ue + eps + (a * V + 3) * s24)[:, None] * p) @ np.abs(w) + (rest * (eps + 8 * s24))[:, None] * np.abs(w[y[rows]]))
    dx[rows] += tiny + unit * tiny * np.abs(w).sum(0)
    g = p * (ue + 1.01 * u + eps + (a * n + 3) * s24)[:, None]
    g[at] = rest * (1.01 * u + eps + (a * n + 3) * s24)
    dw = unit * (g.T @ np.abs(xr)) + tiny + unit * tiny * np.abs(xr).sum(0)
    return float(tok.sum() * unit + 2 * s24 * unit * np.abs(nll).sum()), tok, dx, dw


def check_loss(c, ref, bounds, got=None):
    """Every output of a Loss against O.lm_loss's, element by element; returns the worst share of its bound."""
    got = got or c.results()
    u = HALF_STEP[c.dtype]
    b = dict(zip(("loss", "token_loss", "dx", "dw"), bounds))
    worst = {}
    for k, v in got.items():
        r = np.asarray(getattr(ref, k)).reshape(v.shape)
        tol = b[k] + (1.01 * u if k in ("dx", "dw") else 2.0 ** -24) * np.abs(r) + 1e-300   # a bound of zero: an exact zero
        assert np.all(np.isfinite(v)), k
        share = np.abs(v - r) / tol
        worst[k] = float(share.max())
        assert worst[k] <= 1.0, f"{k}: {worst[k]:.2f} of its bound at {np.unravel_index(share.argmax(), share.shape)}"
    return worst
