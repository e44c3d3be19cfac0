"""hero_final_norm and its backward against the oracle in 64 bits.

Bounds: an output's own rounding (half a step u of its type) and fp32 arithmetic: r from a sum of d squares, at most
d / 64 + 16 additions one after another, halved by the root, and a few products: (d / 64 + 24) 2^-24 of the terms."""
import numpy as np
import pytest

from oracle import hero_oracle as O

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _rows(T, d, dtype, seed):
    import torch
    from tests import train_ends as E
    rng = np.random.default_rng(seed)
    put = lambda a: torch.from_numpy(a.astype(np.float32)).to(E.DEV).to(E.TORCH[dtype])  # noqa: E731
    h = put(rng.standard_normal((T, d)) * rng.uniform(0.1, 5.0, (T, 1)))
    return h, put(rng.standard_normal((T, d)) * 10.0 ** rng.uniform(-6, 0, (T, 1))), put(rng.uniform(0.5, 1.5, d))


CASES = [(1, 256), (2, 1280), (3, 4096), (5, 8192), (7, 8448), (2, 32768), (1024, 512), (1025, 256), (1027, 768), (1030, 2048),
         (1100, 4096), (1026, 5120), (1031, 8192), (1500, 8448)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", CASES)
def test_forward_and_backward(T, d, dtype):
    import torch
    from paper_2609_08189_amd import hero as H
    from tests import train_ends as E
    print(f"case final_norm T={T} d={d} {dtype}", flush=True)
    h, dx, w = _rows(T, d, dtype, T + d)
    h[T // 2] = 0                      # a row of zeros: eps alone
    dims, u = E.dims(d, dtype, EPS), E.HALF_STEP[dtype]
    f = (d / 64 + 24) * 2.0 ** -24
    x = E.Guarded((T, d), h.dtype)
    H.check(H.hero_final_norm(dims, T, h, w, x.t, E.stream()), "hero_final_norm")
    dh, free, dw = E.Guarded((T, d), h.dtype), E.Guarded((T, d), h.dtype), E.Guarded((d,), torch.float32)
    ws = E.Guarded((H.hero_final_norm_backward_workspace_size(dims, T),), torch.uint8)
    H.check(H.hero_final_norm_backward(dims, T, h, dx, w, dh.t, dw.t, ws.t, ws.n, E.stream()), "hero_final_norm_backward")
    H.check(H.hero_final_norm_backward(dims, T, h, dx, w, free.t, None, None, 0, E.stream()), "hero_final_norm_backward")
    torch.cuda.synchronize()
    assert all(g.whole() for g in (x, dh, free, dw, ws))
    assert torch.equal(dh.t, free.t)   # with and without the gain's gradient
    hh, yy, ww = E.f64(h), E.f64(dx), E.f64(w)
    ref = O.rmsnorm(hh, ww, EPS)
    assert np.all(np.abs(E.f64(x.t) - ref) <= (u + f) * np.abs(ref))
    r = 1.0 / np.sqrt(np.mean(hh * hh, 1, keepdims=True) + EPS)
    ref = O.rmsnorm_backward(hh, ww, EPS, yy)
    terms = r * np.abs(yy * ww) + r ** 3 / d * np.abs(hh) * np.sum(np.abs(hh * yy * ww), 1, keepdims=True)
    assert np.all(np.abs(E.f64(dh.t) - ref) <= 1.01 * u * np.abs(ref) + 4 * f * terms)
    ref = O.rmsnorm_gain_grad(hh, EPS, yy)
    # a sum of T terms in any order, each with r's error
    assert np.all(np.abs(E.f64(dw.t) - ref) <= ((T + 8) * 2.0 ** -24 + f) * np.sum(np.abs(yy * hh * r), 0))


def test_graph_and_repeat():
    import torch
    from paper_2609_08189_amd import hero as H
    from tests import train_ends as E
    T, d = 1500, 1024
    print("case final_norm graph", flush=True)
    h, dx, w = _rows(T, d, "bf16", 0)
    dims = E.dims(d)
    x, dh, dw = torch.empty_like(h), torch.empty_like(h), torch.empty(d, device=E.DEV)
    ws = torch.empty(H.hero_final_norm_backward_workspace_size(dims, T), dtype=torch.uint8, device=E.DEV)

    def run():
        H.check(H.hero_final_norm(dims, T, h, w, x, E.stream()), "hero_final_norm")
        H.check(H.hero_final_norm_backward(dims, T, h, dx, w, dh, dw, ws, ws.numel(), E.stream()), "hero_final_norm_backward")

    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for seed in (1, 2, 3):
        h2, dx2, _ = _rows(T, d, "bf16", seed)
        h.copy_(h2)
        dx.copy_(dx2)
        run()
        torch.cuda.synchronize()
        ref = [t.clone() for t in (x, dh, dw)]
        for t in (x, dh, dw, ws):
            t.view(torch.uint8).fill_(0xFF)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((x, dh, dw), ref))
    del g
