"""hero_grad_norm and hero_grad_clip against numpy in 64 bits: the norm to its rounding to fp32, the scaled gradients to
theirs (the factor's, the product's: half a step of fp32 each, then half a step of the type)."""
import numpy as np
import pytest

from oracle import hero_oracle as O

pytestmark = pytest.mark.gpu
S24 = 2.0 ** -24


class Clip:
    """Tensors of (count, dtype, elements off a 16-byte boundary), in place or beside; values from 10^lo to 10^hi."""

    def __init__(self, specs, max_norm, in_place, seed=0, lo=-6, hi=0):
        import torch
        from paper_2609_08189_amd import hero as H
        from tests import train_ends as E
        rng = np.random.default_rng(seed)
        self.H, self.E, self.max_norm = H, E, max_norm
        self.raw, self.grads, self.outs, self.keep = [], [], [], []
        items = []
        for n, dtype, off in specs:
            v = (rng.standard_normal(n) * 10.0 ** rng.uniform(lo, hi)).astype(np.float32)
            g = E.Guarded((n + off,), E.TORCH[dtype])
            g.t[off:] = torch.from_numpy(v).to(E.DEV).to(E.TORCH[dtype])
            o = g if in_place else E.Guarded((n + 2 * off,), E.TORCH[dtype])
            self.raw += [g, o]
            self.grads.append(g.t[off:])
            self.outs.append(self.grads[-1] if in_place else o.t[2 * off:])
            items.append((self.grads[-1], self.outs[-1], n, H.HERO_BF16 if dtype == "bf16" else H.HERO_F32))
        self.before = [E.f64(g) for g in self.grads]
        self.types = [dtype for _, dtype, _ in specs]
        self.tensors = H.hero_grad_tensors(items)
        self.norm, self.norm_only = E.Guarded((1,), torch.float32), E.Guarded((1,), torch.float32)
        self.ws = E.Guarded((H.hero_grad_norm_workspace_size(self.tensors),), torch.uint8)

    def run(self):
        H, E = self.H, self.E
        H.check(H.hero_grad_norm(self.tensors, self.norm_only.t, self.ws.t, self.ws.n, E.stream()), "hero_grad_norm")
        H.check(H.hero_grad_clip(self.tensors, self.max_norm, self.norm.t, self.ws.t, self.ws.n, E.stream()), "hero_grad_clip")
        return self

    def check(self):
        import torch
        E = self.E
        torch.cuda.synchronize()
        assert all(r.whole() for r in self.raw + [self.norm, self.norm_only, self.ws])
        norm, ref = O.grad_clip(self.before, self.max_norm)
        for n in (self.norm, self.norm_only):
            assert abs(E.f64(n.t)[0] - norm) <= 1.01 * S24 * norm
        for got, r, dtype in zip(self.outs, ref, self.types):
            u = E.HALF_STEP[dtype]
            # below the normal range half a step is absolute
            assert np.all(np.abs(E.f64(got) - r) <= (u + 2.02 * S24) * np.abs(r) + 2.0 ** -149 * (65536 if dtype == "bf16" else 1))


ODD = [(1, "f32", 0), (3, "bf16", 0), (8191, "f32", 0), (8192, "bf16", 0), (8193, "f32", 1), (0, "f32", 0), (70000, "bf16", 3),
       (65537, "f32", 2), (384, "f32", 0), (1000001, "bf16", 0), (5, "f32", 3)]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("max_norm", [1e-3, 1.0, 1e9, 0.0, float("inf")])
def test_mixed_tensors(max_norm, in_place):
    import torch
    print(f"case clip mixed {max_norm} in place {in_place}", flush=True)
    c = Clip(ODD, max_norm, in_place).run()
    c.check()
    if max_norm >= 1e9:   # nothing to scale: the very bits
        for g, b in zip(c.outs, c.before):
            assert torch.equal(g.double().cpu(), torch.from_numpy(b))


@pytest.mark.parametrize("n", [1, 95, 96, 97, 300, 4096])
def test_many_tensors(n):
    print(f"case clip {n} tensors", flush=True)
    rng = np.random.default_rng(n)
    Clip([(int(rng.integers(0, 3000)), ["f32", "bf16"][i % 2], int(rng.integers(0, 4))) for i in range(n)], 0.05, True).run().check()


def test_large_tensors():
    print("case clip large", flush=True)
    Clip([(40_000_003, "f32", 0), (7, "f32", 0), (30_000_001, "bf16", 1), (25_000_000, "f32", 1)], 1.0, False).run().check()


@pytest.mark.parametrize("lo,hi", [(18, 30), (-37, -30)])
def test_squares_outside_the_range_of_fp32(lo, hi):
    print(f"case clip 1e{lo} to 1e{hi}", flush=True)
    Clip([(5000, "f32", 0), (5000, "bf16", 0)], 1e-3 if lo > 0 else 1e-33, False, lo=lo, hi=hi).run().check()


def test_factor_below_the_normal_range():
    """max_norm / norm of about 1e-42, which fp32 holds to three digits."""
    print("case clip, a factor of 1e-42", flush=True)
    Clip([(5000, "f32", 0), (5000, "bf16", 0), (5001, "f32", 1)], 1e-5, False, lo=35, hi=35).run().check()


def test_zeros_and_values_that_are_not_finite():
    import torch
    print("case clip special values", flush=True)
    c = Clip([(5000, "f32", 0), (3000, "bf16", 1)], 1.0, True)
    for g in c.grads:
        g.zero_()
    c.run()
    torch.cuda.synchronize()
    assert float(c.norm.t) == 0 and not any(g.any() for g in c.grads)
    for bad, want in ((float("nan"), "nan"), (float("inf"), "inf")):
        c = Clip([(5000, "f32", 0), (3000, "bf16", 1)], 1.0, True)
        c.grads[1][17] = bad
        c.run()
        torch.cuda.synchronize()
        if want == "nan":
            assert torch.isnan(c.norm.t).all() and all(torch.isnan(g).all() for g in c.grads)
        else:
            assert torch.isinf(c.norm.t).all() and not c.grads[0].any() and torch.isnan(c.grads[1][17])


def test_list_is_not_read_after_the_call_and_a_graph_replays_it():
    import ctypes
    import torch
    from tests import train_ends as E
    print("case clip graph", flush=True)
    c = Clip(ODD + [(100, "f32", 0)] * 120, 0.3, False).run()
    c.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    ctypes.memset(c.tensors, 0, ctypes.sizeof(c.tensors))
    for seed in (1, 2, 3):
        for t in c.grads:
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(seed)).to(E.DEV) * 10.0 ** -seed)
        c.before = [E.f64(t) for t in c.grads]
        for t in c.outs:
            t.fill_(7.0)
        c.norm.t.fill_(-1.0)
        torch.cuda.synchronize()
        g.replay()
        c.check()
    del g
