"""One training step through the C ABI as a program runs it: routed layers forwards, final norm, language-model loss, the
norm's backward, the penalty, the blocks' and the routers' backwards, and the clipping of every trained tensor by the
global norm; twice eagerly (the second time on the same buffers).  Compared with the oracle's chain in 64 bits, which
takes the GPU's branch decisions and its stack output: the loss, dL/dh_out, the global norm and the clipped gradients.
The bars are those of the stack's backward: 1e-4 of a tensor's largest element in fp32, 2e-2 in bf16."""
import numpy as np
import pytest

from oracle import hero_oracle as O
from paper_2609_08189_amd import synth
from tests.oracle_inputs import adapter_of, dims_of, ffn_of, router_of

pytestmark = pytest.mark.gpu


def _err(x, ref):
    return float(np.max(np.abs(x - ref)) / max(np.max(np.abs(ref)), 1e-30))


@pytest.mark.parametrize("dtype,max_norm", [("f32", 0.01), ("f32", 1e6), ("bf16", 0.01)])
def test_step(dtype, max_norm):
    import torch
    from paper_2609_08189_amd import hero as H
    from paper_2609_08189_amd.device import DeviceProblem, LayerStats
    from tests.train_ends import f64

    L, batch, seq, V, d_m, alpha = 3, 4, 30, 1009, 64, 0.1
    T = batch * seq
    if dtype == "f32":
        w = synth.Workload("step_f32", "f32", d=256, d_ff=688, d_r=16, L_R=L, d_m=d_m, T=T, mode="budget", budget=0.3)
    else:
        w = synth.Workload("step_bf16", "bf16", d=512, d_ff=1408, d_r=64, L_R=L, d_m=d_m, T=T, mode="budget", budget=0.3)
    tol, wt = (1e-4, torch.float32) if dtype == "f32" else (2e-2, torch.bfloat16)
    print(f"case training step {dtype} max_norm={max_norm}", flush=True)
    prob = synth.make_problem(w, seed=7)
    dp = DeviceProblem(prob, stats=False, for_stack=True)
    dev, dims, s, d = dp.device, dp.dims, dp.stream(), w.d
    f32 = lambda *shape: torch.zeros(*shape, dtype=torch.float32, device=dev)  # noqa: E731
    buf = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device=dev)     # noqa: E731
    rng = np.random.default_rng(1)
    head = torch.from_numpy((rng.standard_normal((V, d)) * 1.5 / d ** 0.5).astype(np.float32)).to(dev).to(wt)
    gain = torch.from_numpy(rng.uniform(0.5, 1.5, d).astype(np.float32)).to(dev).to(wt)
    y = rng.integers(0, V, T)
    y[seq - 1::seq] = -1                      # the last token of a sequence predicts nothing
    y[:10] = -1                               # a prompt
    targets = torch.as_tensor(y, dtype=torch.int32, device=dev)
    head_t = torch.empty(d, (V + 63) // 64 * 64, dtype=wt, device=dev)
    H.check(H.hero_lm_head_weights_make(dims, V, head, head_t, s), "head")
    ffn_t = []
    for j in range(L):
        a, b = torch.empty(w.d_ff, d, dtype=wt, device=dev), torch.empty(d, 2 * w.d_ff, dtype=wt, device=dev)
        H.check(H.hero_ffn_backward_weights_make(dims, dp.ffn_s[j], a, b, s), "ffn_t")
        ffn_t.append((a, b))

    hb = [dp.hbar] + [torch.empty_like(dp.hbar) for _ in range(L)]
    stats = [LayerStats(T, dev) for _ in range(L)]
    x, dx, dh = (torch.empty_like(dp.hbar) for _ in range(3))
    loss, norm, skip = f32(1), f32(1), f32(1)
    outs = H.hero_lm_loss_out(loss.data_ptr(), None, dx.data_ptr(), None)
    gates, dgates = f32(L, T), f32(L, T)
    rgrads = {k: f32(*dp.router[k].shape) for k in H.ROUTER_FIELDS}
    rgrads_s = H.hero_router_grads(**{k: v.data_ptr() for k, v in rgrads.items()})
    deta, dw1, dw2 = f32(L, 4), [f32(w.d_r, d) for _ in range(L)], [f32(d, w.d_r) for _ in range(L)]
    trained = list(rgrads.values()) + dw1 + dw2 + [deta[j, :1] for j in range(L)]
    clipped = H.hero_grad_tensors([(t, t, t.numel(), H.HERO_F32) for t in trained])
    ws = buf(H.hero_workspace_size(dims, T, False))
    lws = buf(H.hero_lm_loss_workspace_size(dims, V, T, True, False))
    bws, rws = buf(H.hero_backward_workspace_size(dims, T)), buf(H.hero_router_backward_workspace_size(dims, T))
    gws = buf(H.hero_grad_norm_workspace_size(clipped))

    def step():
        S, zeta, p, m = f32(T, d_m, d_m), f32(T, d_m), torch.ones(T, device=dev), torch.ones(T, device=dev)
        st = H.hero_state(S.data_ptr(), zeta.data_ptr(), p.data_ptr(), m.data_ptr())
        states = []
        for j in range(1, L + 1):
            states.append([t.clone() for t in (S, zeta, p, m)])
            H.check(H.hero_routed_layer(dims, j, T, hb[j - 1], hb[j - 2] if j >= 2 else None, hb[j - 3] if j >= 3 else None,
                                        hb[j], st, dp.ffn_s[j - 1], dp.router_s, dp.adapter_s[j - 1], dp.eta[j - 1],
                                        dp.routing_s, stats[j - 1].struct, ws, ws.numel(), s), "layer")
            gates[j - 1].copy_(stats[j - 1].gate)
        H.check(H.hero_final_norm(dims, T, hb[L], gain, x, s), "final norm")
        H.check(H.hero_lm_loss(dims, V, T, x, H.hero_lm_head(head.data_ptr(), head_t.data_ptr()), targets,
                               H.HERO_LOSS_MEAN, 1.0, outs, lws, lws.numel(), s), "loss")
        H.check(H.hero_final_norm_backward(dims, T, hb[L], dx, gain, dh, None, None, 0, s), "norm backward")
        H.check(H.hero_skip_penalty(L, batch, seq, gates, alpha, skip, dgates, s), "penalty")
        carry_t = [f32(T, d_m, d_m), f32(T, d_m), f32(T), f32(T)]
        carry = H.hero_router_carry(*[t.data_ptr() for t in carry_t])
        dHB = [f32(T, d) for _ in range(L + 1)] + [dh.float()]
        for t in trained:
            t.zero_()
        tmp, dgate, dlogit = torch.empty_like(dp.hbar), f32(T), f32(T)
        for j in range(L, 0, -1):
            sj = stats[j - 1]
            H.check(H.hero_routed_block_backward(
                dims, T, hb[j - 1], dHB[j + 1].to(wt), sj.gate, sj.idx_ffn, sj.idx_ad, sj.counts, None, dgates[j - 1],
                dp.ffn_s[j - 1], H.hero_ffn_backward_weights(*[t.data_ptr() for t in ffn_t[j - 1]]), dp.adapter_s[j - 1],
                H.hero_block_grads(*[t.data_ptr() for t in (tmp, dgate, dlogit, dw1[j - 1], dw2[j - 1])]), bws, bws.numel(),
                s), "block backward")
            dHB[j] += tmp.float()
            H.check(H.hero_router_backward(
                dims, j, T, hb[j - 1], hb[j - 2] if j >= 2 else None, hb[j - 3] if j >= 3 else None,
                H.hero_state(*[t.data_ptr() for t in states[j - 1]]), dp.router_s, dp.eta[j - 1], dlogit, carry, dHB[j],
                dHB[j - 1] if j >= 2 else None, dHB[j - 2] if j >= 3 else None, rgrads_s, deta[j - 1], rws, rws.numel(), s),
                "router backward")
        H.check(H.hero_grad_clip(clipped, max_norm, norm, gws, gws.numel(), s), "clip")
        torch.cuda.synchronize()
        return [t.clone() for t in trained]

    first = step()
    got = step()
    assert all(torch.equal(a, b) for a, b in zip(first, got))

    h_out, W, g = f64(hb[L]), f64(head), f64(gain)
    ref = O.lm_loss(O.rmsnorm(h_out, g, w.eps_norm), W, y)
    dh_ref = O.rmsnorm_backward(h_out, g, w.eps_norm, ref.dx)
    errs = {"loss": abs(float(loss) / ref.loss - 1), "dh_out": _err(f64(dh), dh_ref)}
    _, dg = O.skip_penalty(f64(gates), batch, seq, alpha)
    sb = O.routed_stack_backward(dims_of(w), prob.hbar.f64, [ffn_of(prob.ffn[i]) for i in range(L)], router_of(prob),
                                 [adapter_of(prob.adapter[i]) for i in range(L)], [float(e) for e in prob.eta],
                                 [t.host()["mask"] for t in stats], dh_ref, list(dg))
    th1 = np.zeros(tuple(dp.router["th1"].shape))
    th1[:, :sb.router.th1.shape[1]] = sb.router.th1
    grads = [th1 if k == "th1" else getattr(sb.router, k) for k in H.ROUTER_FIELDS] + list(sb.dw1) + list(sb.dw2)
    grads += [np.array([e]) for e in sb.deta]
    norm_ref, ref_clipped = O.grad_clip(grads, max_norm)
    errs["norm"] = abs(float(norm) / norm_ref - 1)
    scale_v = np.max(np.abs(ref_clipped[H.ROUTER_FIELDS.index("w_v")]))
    for i, (t, r) in enumerate(zip(got, ref_clipped)):
        name = H.ROUTER_FIELDS[i] if i < len(H.ROUTER_FIELDS) else f"t{i}"
        a = f64(t).reshape(r.shape)
        # dW_q, dW_k of these short stacks are sums of cancelling terms: against their companion's scale
        errs[name] = float(np.max(np.abs(a - r)) / scale_v) if name in ("w_q", "w_k") else _err(a, r)
    print("  errors:", {k: f"{v:.1e}" for k, v in errs.items()}, flush=True)
    assert (norm_ref > max_norm) == (max_norm < 1)
    # An eta's gradient is one number, the sum of the tokens' shares (tokens meet nowhere else in the stack).  With each
    # share held to the bar, |error| <= tol sum |share|: shares of both signs cancel in the sum, their errors need not.
    one = lambda a, t: a[:, t:t + 1]  # noqa: E731
    masks = np.stack([t.host()["mask"] for t in stats])
    shares = sum(np.abs(O.routed_stack_backward(
        dims_of(w), prob.hbar.f64[t:t + 1], [ffn_of(prob.ffn[i]) for i in range(L)], router_of(prob),
        [adapter_of(prob.adapter[i]) for i in range(L)], [float(e) for e in prob.eta], list(one(masks, t)), dh_ref[t:t + 1],
        list(one(dg, t))).deta) for t in range(T))
    clip = min(1.0, max_norm / norm_ref)
    for j in range(L):
        i = len(got) - L + j
        errs[f"t{i}"] = float(np.abs(f64(got[i]) - ref_clipped[i])[0] / max(clip * shares[j], 1e-30))
    for k, v in errs.items():
        assert v <= tol, f"{k}: {v:.3e} > {tol:.0e}"
