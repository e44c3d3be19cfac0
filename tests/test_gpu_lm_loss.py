"""hero_lm_loss against the oracle in 64 bits, element by element, within bounds derived from the roundings on the way
(train_ends.loss_bounds)."""
import numpy as np
import pytest

from oracle import hero_oracle as O

pytestmark = pytest.mark.gpu


def _inputs(T, d, V, dtype, seed, keep=0.8, size=1.0, sure=8.0):
    import torch
    from tests import train_ends as E
    rng = np.random.default_rng(seed)
    w = torch.from_numpy(rng.standard_normal((V, d)).astype(np.float32) * (1.5 / d ** 0.5)).to(E.DEV).to(E.TORCH[dtype])
    y = rng.integers(0, V, T)
    x = rng.standard_normal((T, d)).astype(np.float32)
    x += (sure * rng.random((T, 1)) / 1.5).astype(np.float32) * w.float().cpu().numpy()[y]
    y[rng.random(T) >= keep] = -1
    return torch.from_numpy(x * np.float32(size)).to(E.DEV).to(E.TORCH[dtype]), w, y


def _check(c, y):
    from tests import train_ends as E
    x, w = E.f64(c.x), E.f64(c.w)
    worst = E.check_loss(c, O.lm_loss(x, w, y, c.scale, c.mean), E.loss_bounds(x, w, y, c.scale, c.mean, c.dtype))
    print("  share of the bounds:", {k: f"{v:.2f}" for k, v in worst.items()}, flush=True)
    for k in ("token_loss", "dx"):
        if k in c.out:
            lost = (y < 0) | (y >= c.V)
            assert not E.f64(c.out[k].t)[lost].any(), f"{k} of a token that does not count"


SIZES = [(1, 256, 65), (1, 512, 2003), (2, 256, 127), (3, 256, 128), (17, 512, 256), (63, 256, 257), (64, 768, 320),
         (65, 256, 1000), (129, 512, 4001), (257, 256, 2003), (300, 1024, 511), (600, 256, 3001), (1025, 256, 1537),
         (1, 256, 40001), (5, 256, 33000), (300, 256, 20011), (130, 1280, 700), (2000, 256, 8000),
         (16, 256, 9001), (17, 512, 8200), (33, 768, 8191), (64, 1024, 10007), (48, 256, 24577), (100, 1280, 9000), (128, 512, 2000), (127, 256, 40000),
         (3000, 512, 1100), (1300, 256, 600), (40, 256, 140001), (767, 256, 33333)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", SIZES)
def test_loss_and_gradients(T, d, V, dtype):
    from tests import train_ends as E
    print(f"case lm_loss T={T} d={d} V={V} {dtype}", flush=True)
    x, w, y = _inputs(T, d, V, dtype, T + V, keep=1.0 if T < 4 else 0.8)
    _check(E.Loss(x, w, y, mean=T % 2 == 1, scale=1.0 if T % 2 else 0.37).run(), y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dx,dw", [(False, False), (True, False), (False, True)])
def test_outputs_are_optional(dx, dw, dtype):
    import torch
    from tests import train_ends as E
    print(f"case lm_loss outputs dx={dx} dw={dw} {dtype}", flush=True)
    x, w, y = _inputs(150, 512, 1333, dtype, 5)
    c, full = E.Loss(x, w, y, dx=dx, dw=dw).run(), E.Loss(x, w, y).run()
    _check(c, y)
    for k in c.out:
        assert torch.equal(c.out[k].t, full.out[k].t), k


@pytest.mark.parametrize("d,V", [(384, 64), (384, 1000), (128, 5000)])
@pytest.mark.parametrize("T", [1, 40, 400])
def test_fp32_widths_of_half_a_tile(T, d, V):
    """d a multiple of 128 only, vocabularies below 65: fp32 models alone."""
    from tests import train_ends as E
    print(f"case lm_loss f32 T={T} d={d} V={V}", flush=True)
    x, w, y = _inputs(T, d, V, "f32", T + d, keep=1.0 if T < 4 else 0.7)
    _check(E.Loss(x, w, y).run(), y)


@pytest.mark.parametrize("T,d,V,dtype", [(8192 + 9, 256, 16384 + 300, "bf16"), (8192 + 9, 256, 5376 + 200, "f32"),
                                         (8192, 256, 32768 + 77, "bf16"), (5001, 256, 9000, "bf16"), (8193, 256, 3000, "bf16"), (40000, 256, 300, "bf16"), (2000, 384, 33800, "f32"), (1500, 256, 30000, "f32")])
def test_chunks_of_rows_and_pieces_of_the_vocabulary(T, d, V, dtype):
    from tests import train_ends as E
    print(f"case lm_loss pieces T={T} d={d} V={V} {dtype}", flush=True)
    x, w, y = _inputs(T, d, V, dtype, 1, keep=0.97)
    _check(E.Loss(x, w, y).run(), y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,size,V", [(5, 30.0, 1700), (200, 30.0, 1700), (200, 120.0, 1700), (7, 30.0, 9001), (40, 120.0, 20011),
                                      (300, 60.0, 16001)])
def test_logits_far_above_the_target(T, size, V, dtype):
    """References move: differences of several hundred between a row's logits."""
    from tests import train_ends as E
    print(f"case lm_loss far T={T} size={size} V={V} {dtype}", flush=True)
    x, w, y = _inputs(T, 256, V, dtype, 11, keep=0.9, size=size, sure=2.0)
    _check(E.Loss(x, w, y, mean=False).run(), y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_reference_moves_between_pieces(dtype):
    """The target in the first piece, a logit 200 above it in the last, another 150 above it before."""
    import torch
    from tests import train_ends as E
    T, d, V = 8192, 256, 40000
    print(f"case lm_loss far, by pieces {dtype}", flush=True)
    g = torch.Generator().manual_seed(3)
    w = torch.randn(V, d, generator=g) * 0.02
    x = torch.randn(T, d, generator=g)
    w[20000] = x[5] / x[5].norm() * 9.5
    w[39999] = x[5] / x[5].norm() * 13.0
    w[30000] = -x[7] / x[7].norm() * 14.0
    x, w = x.to(E.DEV).to(E.TORCH[dtype]), w.to(E.DEV).to(E.TORCH[dtype])
    y = np.full(T, -1)
    y[[0, 5, 7, 4000, 8191]] = [9, 100, 30000, 39999, 20000]
    _check(E.Loss(x, w, y, dw=False).run(), y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sure_tokens_keep_the_digits_of_their_loss(dtype):
    from tests import train_ends as E
    print(f"case lm_loss sure {dtype}", flush=True)
    x, w, y = _inputs(64, 256, 700, dtype, 4, keep=1.0, sure=30.0)
    c = E.Loss(x, w, y).run()
    _check(c, y)
    ref = O.lm_loss(E.f64(x), E.f64(w), y).token_loss
    small = ref < 1e-3
    assert small.sum() > 10
    # a relative error of the loss: that of exp at arguments of some tens, and the logits' (256 additions of fp32)
    assert np.all(np.abs(E.f64(c.out["token_loss"].t)[small] / ref[small] - 1) < 256 * 2.0 ** -24 * 60)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_that_do_not_count(dtype):
    """None counts; targets at both ends of int32; rows of NaN and infinity without a target."""
    import torch
    from tests import train_ends as E
    print(f"case lm_loss ignored {dtype}", flush=True)
    T, V = 90, 400
    x, w, y = _inputs(T, 256, V, dtype, 9, keep=1.0)
    y[::3], y[1::9], y[5] = -100, V, 2 ** 31 - 1
    y[8] = -2 ** 31
    x[::3] = float("nan")
    x[1::9] = float("inf")
    c = E.Loss(x, w, y).run()
    got = c.results()
    clean = x.clone()
    clean[torch.from_numpy((y < 0) | (y >= V)).to(E.DEV)] = 0
    ref = O.lm_loss(E.f64(clean), E.f64(w), y)
    E.check_loss(c, ref, E.loss_bounds(E.f64(clean), E.f64(w), y, 1.0, True, dtype), got)
    assert not got["dx"][(y < 0) | (y >= V)].any()
    for mean in (True, False):
        none = E.Loss(x, w, np.full(T, -1), mean=mean).run().results()
        assert all(not v.any() for v in none.values())


def test_one_counted_token_anywhere():
    from tests import train_ends as E
    x, w, _ = _inputs(2500, 256, 600, "bf16", 2)
    for t in (0, 1, 7, 1023, 1024, 2049, 2499):
        print(f"case lm_loss one counted token {t}", flush=True)
        y = np.full(2500, -1)
        y[t] = 599
        _check(E.Loss(x, w, y).run(), y)


def test_nan_in_one_token_stays_there():
    import torch
    from tests import train_ends as E
    print("case lm_loss nan", flush=True)
    x, w, y = _inputs(130, 256, 500, "bf16", 6, keep=1.0)
    x[70, 3] = float("nan")
    x[71] = 3e38           # its logits overflow
    c = E.Loss(x, w, y, mean=False, dw=False).run()
    got = c.results()
    assert np.isnan(got["loss"]).all() and np.isnan(got["token_loss"][70:72]).all() and np.isnan(got["dx"][70:72]).all()
    rest = np.r_[0:70, 72:130]
    assert np.isfinite(got["token_loss"][rest]).all() and np.isfinite(got["dx"][rest]).all()
    alone = E.Loss(x[:70], w, y[:70], mean=False, dw=False).run()
    torch.cuda.synchronize()
    assert torch.equal(alone.out["token_loss"].t, c.out["token_loss"].t[:70])


def test_head_copy_is_the_transpose_with_zeros():
    import torch
    from tests import train_ends as E
    for dtype in ("bf16", "f32"):
        for d, V in [(256, 65), (512, 128), (256, 1001), (1280, 70)]:
            print(f"case head copy d={d} V={V} {dtype}", flush=True)
            x, w, y = _inputs(1, d, V, dtype, V)
            c = E.Loss(x, w, y, dw=False)
            torch.cuda.synchronize()
            assert c.w_t.whole() and torch.equal(c.w_t.t[:, :V], w.t()) and not c.w_t.t[:, V:].any()


def test_head_beyond_32_bit_offsets():
    """300000 rows of 8192: 4.9 GB, scored in pieces."""
    import torch
    from tests import train_ends as E
    print("case lm_loss 300000 x 8192", flush=True)
    V, d, T = 300000, 8192, 3
    g = torch.Generator(device=E.DEV).manual_seed(1)
    w = torch.empty(V, d, dtype=torch.bfloat16, device=E.DEV)
    for i in range(0, V, 50000):
        w[i:i + 50000] = torch.randn(50000, d, generator=g, device=E.DEV) * 0.02
    x = torch.randn(T, d, generator=g, device=E.DEV).bfloat16()
    y = np.array([5, 299999, 150000])
    c = E.Loss(x, w, y, dx=False, dw=False).run()
    got = c.results()
    logits = torch.cat([x.double() @ w[i:i + 50000].double().t() for i in range(0, V, 50000)], 1)
    ref = torch.logsumexp(logits, 1) - logits[torch.arange(T), torch.as_tensor(y)]
    # the logits' relative error: 8192 additions of |x W| about 0.8 0.016 each, twice; far above the rest
    assert np.all(np.abs(got["token_loss"] - ref.cpu().numpy()) < 2 * 8192 * 2.0 ** -24 * 8192 * 0.8 * 0.016)
    assert np.all(np.abs(got["token_loss"] - ref.cpu().numpy()) < 1e-4)
    del w, logits
    torch.cuda.empty_cache()


def test_calls_repeat_bit_for_bit_and_leave_inputs_alone():
    import torch
    from tests import train_ends as E
    print("case lm_loss repeat", flush=True)
    x, w, y = _inputs(700, 512, 5000, "bf16", 8)
    c = E.Loss(x, w, y).run()
    torch.cuda.synchronize()
    first, x0, w0 = {k: v.t.clone() for k, v in c.out.items()}, x.clone(), w.clone()
    for v in c.out.values():
        v.poison()
    c.ws.poison()
    c.run()
    torch.cuda.synchronize()
    assert all(torch.equal(first[k], v.t) for k, v in c.out.items())
    assert torch.equal(x, x0) and torch.equal(w, w0)


def test_two_calls_on_two_streams():
    import torch
    from tests import train_ends as E
    print("case lm_loss two streams", flush=True)
    a, b = _inputs(500, 512, 3000, "bf16", 21), _inputs(333, 512, 2500, "f32", 22)
    ca, cb = E.Loss(*a), E.Loss(*b)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(sa):
            ca.run()
        with torch.cuda.stream(sb):
            cb.run()
    _check(ca, a[2])
    _check(cb, b[2])


@pytest.mark.parametrize("T,d,V,size", [(1, 512, 30000, 1.0), (16, 1024, 15001, 1.0), (17, 640, 33003, 1.0), (33, 512, 30001, 1.0),
                                        (64, 1024, 16000, 1.0), (65, 1024, 15000, 1.0), (96, 1024, 14401, 60.0), (97, 1152, 16001, 1.0),
                                        (127, 1024, 15003, 120.0), (128, 1152, 15003, 1.0), (20, 512, 30000, 120.0), (50, 256, 140001, 60.0), (3, 128, 131073, 1.0)])
def test_few_fp32_rows_against_large_heads(T, d, V, size):
    from tests import train_ends as E
    print(f"case lm_loss few fp32 rows T={T} d={d} V={V} size={size}", flush=True)
    x, w, y = _inputs(T, d, V, "f32", T + V, keep=1.0 if T < 4 else 0.9, size=size, sure=2.0)
    _check(E.Loss(x, w, y, mean=False).run(), y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", [(90, 131072), (90, 131073), (90, 131199), (90, 131200), (3, 262150), (8192, 33000)])
def test_last_pieces_that_would_be_narrow(T, V, dtype):
    from tests import train_ends as E
    print(f"case lm_loss narrow rest T={T} V={V} {dtype}", flush=True)
    x, w, y = _inputs(T, 256, V, dtype, T + V, keep=0.9 if T < 1000 else 0.05)
    _check(E.Loss(x, w, y, dw=T < 1000).run(), y)


def _scored(x, w, y, **kw):
    """The loss without gradients, checked."""
    from tests import train_ends as E
    c = E.Loss(x, w, y, dx=False, dw=False, **kw).run()
    _check(c, y)
    return c


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", [(1, 256, 16384), (1, 768, 20011), (2, 256, 14337), (16, 512, 30001), (17, 256, 33000), (32, 256, 14400),
                                   (33, 512, 16001), (64, 1024, 20000), (64, 256, 131071), (5, 256, 131200)])
def test_scoring_few_tokens(T, d, V, dtype):
    import torch
    from tests import train_ends as E
    print(f"case lm_loss score T={T} d={d} V={V} {dtype}", flush=True)
    x, w, y = _inputs(T, d, V, dtype, T + V, keep=1.0 if T < 4 else 0.7)
    y[0] = V - 1
    a, b = _scored(x, w, y, mean=T % 2 == 1, scale=0.7), _scored(x, w, y, mean=T % 2 == 1, scale=0.7)
    assert all(torch.equal(a.out[k].t, b.out[k].t) for k in a.out)      # one order of every sum
    far = x * 40
    _scored(far, w, y)
    sure = E.f64(w)[y] * 30 * (np.arange(T) % 2 == 0)[:, None]
    _scored(x + torch.from_numpy(sure).to(x), w, y, mean=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scoring_tokens_that_do_not_count_and_values_that_are_not_finite(dtype):
    import torch
    from tests import train_ends as E
    print(f"case lm_loss score specials {dtype}", flush=True)
    T, V = 40, 20011
    x, w, y = _inputs(T, 256, V, dtype, 9, keep=1.0)
    y[::3], y[1::9], y[5], y[8] = -100, V, 2 ** 31 - 1, -2 ** 31
    dead = torch.from_numpy((y < 0) | (y >= V)).to(E.DEV)
    clean = _scored(torch.where(dead[:, None], torch.zeros_like(x), x), w, y)
    x[::3], x[1::9] = float("nan"), float("inf")
    c = E.Loss(x, w, y, dx=False, dw=False).run()
    for k, v in c.results().items():
        assert np.array_equal(v, E.f64(clean.out[k].t)), k
    assert not c.out["token_loss"].t[dead].any()
    for mean in (True, False):
        none = E.Loss(x, w, np.full(T, -1), dx=False, dw=False, mean=mean).run().results()
        assert all(not v.any() for v in none.values())
    # one counted row of NaN, one with an infinite element: no finite loss of these, the others as they were
    x, w, y = _inputs(T, 256, V, dtype, 9, keep=1.0)
    good = E.Loss(x, w, y, dx=False, dw=False).run().results()["token_loss"]
    x[3], x[7, 5] = float("nan"), float("inf")
    bad = E.Loss(x, w, y, dx=False, dw=False).run()
    torch.cuda.synchronize()
    token = E.f64(bad.out["token_loss"].t)
    assert not np.isfinite(token[[3, 7]]).any() and not np.isfinite(float(bad.out["loss"].t))
    keep = np.delete(np.arange(T), [3, 7])
    assert np.array_equal(token[keep], good[keep])
    # 128 columns of -infinity (a whole part), and one in each of the others, change nothing but their own share
    x, w, y = _inputs(T, 256, V, dtype, 9, keep=1.0, sure=0.0)
    x.abs_()
    y = y % 128
    gone = np.concatenate([np.arange(1280, 1408), np.arange(200, V, 128)])
    w[torch.from_numpy(gone).to(E.DEV)] = -3e38
    c = E.Loss(x, w, y, dx=False, dw=False).run()
    rest = torch.ones(V, dtype=torch.bool, device=E.DEV)
    rest[torch.from_numpy(gone).to(E.DEV)] = False
    short = w[rest].contiguous()
    E.check_loss(c, O.lm_loss(E.f64(x), E.f64(short), y), E.loss_bounds(E.f64(x), E.f64(short), y, 1.0, True, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scoring_replays(dtype):
    import torch
    from tests import train_ends as E
    print(f"case lm_loss score graph {dtype}", flush=True)
    x, w, y = _inputs(20, 256, 20011, dtype, 3, keep=1.0)
    c = E.Loss(x, w, y, dx=False, dw=False).run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    for keep in (1.0, 0.3, 0.0, 0.8):
        x2, _, y2 = _inputs(20, 256, 20011, dtype, 50 + int(10 * keep), keep=keep)
        c.x.copy_(x2)
        c.y.copy_(torch.as_tensor(y2, dtype=torch.int32))
        eager = E.Loss(x2, w, y2, dx=False, dw=False).run()
        for v in c.out.values():
            v.poison()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for k, v in c.results().items():
            assert np.array_equal(v, E.f64(eager.out[k].t)), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", [(5, 1000), (5, 9001), (200, 1000), (300, 40001)])
def test_logits_of_minus_infinity(T, V, dtype):
    """A head row whose logits are below the range: no share in a loss, zeros in dW, and dx as without it."""
    from tests import train_ends as E
    print(f"case lm_loss -inf T={T} V={V} {dtype}", flush=True)
    x, w, y = _inputs(T, 256, V, dtype, 21, sure=0.0)
    x.abs_()
    y[y == 7] = 8
    w[7] = -3e38
    assert x.double().sum(1).min() > 10          # times 3e38: past the range of fp32
    got = E.Loss(x, w, y).run().results()
    assert not got["dw"][7].any()
    w[7] = -100.0                                 # logits of -1000 and less: exponentials of zero in 64 bits too
    x64, w64 = E.f64(x), E.f64(w)
    c = E.Loss(x, w, y)
    # the row without size: its exp(0) of a sum of V others of about e takes less than 1 in 100 of what they are bounded by
    bounds = E.loss_bounds(x64, np.where(np.arange(V)[:, None] == 7, 0.0, w64), y, 1.0, True, dtype)
    E.check_loss(c, O.lm_loss(x64, w64, y), [1.01 * b for b in bounds], got)


@pytest.mark.parametrize("T,dtype", [(5, "bf16"), (300, "bf16"), (70, "f32"), (1200, "f32"), (1100, "bf16")])
def test_graph_replays_with_new_inputs(T, dtype):
    """Targets, and with them the number of rows, change between the replays; eager work runs in between."""
    import torch
    from tests import train_ends as E
    print(f"case lm_loss graph T={T} {dtype}", flush=True)
    x, w, y = _inputs(T, 512, 2003, dtype, 13, keep=1.0)
    c = E.Loss(x, w, y).run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    torch.cuda.synchronize()
    junk = torch.randn(1 << 20, device=E.DEV)
    rng = np.random.default_rng(0)
    for keep in (1.0, 0.4, 0.0, 0.9):
        x2, _, _ = _inputs(T, 512, 2003, dtype, 100 + int(10 * keep), keep=1.0)
        y2 = np.where(rng.random(T) < keep, rng.integers(0, 2003, T), -1)
        c.x.copy_(x2)
        c.y.copy_(torch.as_tensor(y2, dtype=torch.int32))
        eager = E.Loss(x2, w, y2).run()
        for v in c.out.values():
            v.poison()
        junk.mul_(1.0001)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for k, v in c.out.items():
            assert v.whole() and torch.equal(v.t, eager.out[k].t), f"keep {keep}: {k}"
    del g
