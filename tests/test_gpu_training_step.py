"""The losses and the orthogonalised update as a training step uses them: together with the head's log-probabilities, the replayed
gate and the layer's backward; on other streams, at once, from graphs, from odd addresses and past 2^31 elements."""
import numpy as np
import pytest
import torch

from oracle import operators as ref
from paper_2510_11370_amd import r3, synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
f32 = lambda *s: torch.empty(*s, device=DEV)  # noqa: E731


def test_from_the_head_to_the_loss_and_back():
    """token_logprobs -> policy_loss -> token_logprobs_backward against automatic differentiation of the whole in 64 bits."""
    T, V = 700, 1201
    g = torch.Generator(device=DEV).manual_seed(3)
    z = torch.randn(T, V, generator=g, device=DEV) * 2
    starts = torch.tensor([0, 150, 150, 420, 640], dtype=torch.int32, device=DEV)
    target = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    target[::3] = -1
    rollout = torch.randn(T, generator=g, device=DEV) * 0.3
    adv = torch.randn(4, generator=g, device=DEV)
    logp, H, stats = f32(T), f32(T), f32(T, 2)
    r3.token_logprobs(z, target, logp, entropy=H, stats=stats)
    old, ref_lp = logp + rollout, logp - 0.5 * rollout
    for ratio in ("token", "sequence"):
        D = r3.policy_desc(T, 4, ratio=ratio, norm="sequences", adv_seq=True, clip_high=0.25, kl_coef=0.125, entropy_coef=0.0625)
        dl, dh, out, dz = f32(T), f32(T), f32(8), torch.empty_like(z)
        r3.policy_loss(D, logp, adv, out, logp_old=old, logp_ref=ref_lp, entropy=H, target=target, seq_start=starts, dlogp=dl, dentropy=dh)
        r3.token_logprobs_backward(z, target, stats, dz, dlogp=dl, entropy=H, dentropy=dh)

        z64 = z.double().cpu().requires_grad_()
        lp = torch.log_softmax(z64, 1)
        t, o, rf, A = target.long().cpu(), old.double().cpu(), ref_lp.double().cpu(), adv.double().cpu()
        x, ent = lp.gather(1, t.clamp(min=0)[:, None])[:, 0], -(lp.exp() * lp).sum(1)
        loss = 0.0
        for q, (b, e) in enumerate(((0, 150), (150, 150), (150, 420), (420, 640))):
            i = torch.arange(b, e)[t[b:e] >= 0]
            if len(i) == 0:
                continue
            d = x[i] - o[i]
            r = (d.mean().expand(len(i)) if ratio == "sequence" else d).exp()
            k = rf[i] - x[i]
            clip = r.clamp(1 - float(np.float32(0.2)), 1.25)
            loss = loss + (-torch.minimum(r * A[q], clip * A[q]) + 0.125 * (k.exp() - 1 - k) - 0.0625 * ent[i]).mean() / 3
        loss.backward()
        # the log-probabilities' sums pass some 60 roundings, and a token's |d| and |log p| are below 30
        assert abs(out[0].item() - loss.item()) < 60 * 30 * 2.0 ** -24
        assert float((dz.double().cpu() - z64.grad).norm() / z64.grad.norm()) < 60 * 30 * 2.0 ** -24
        assert (dz[640:] == 0).all() and (dz[::3] == 0).all()


def test_a_step_of_the_layer_with_its_balance_loss_and_update():
    """gate -> balance loss, forward -> backward, the logits' gradient to the router, and an orthogonalised update of every weight."""
    sh = synth.LayerShape(T=600, d=256, E=16, K=4, F=128, act="f32", sigma=0.05, seed=5)
    t = {k: synth.draw(sh, k, DEV).float() for k in ("x", "Wr", "Wg", "Wu", "Wd", "dy")}
    D = r3.desc(sh.T, sh.d, sh.E, sh.K, sh.F, "f32")
    idx = torch.zeros(sh.T, sh.K, dtype=torch.uint8, device=DEV)
    r3.record_topk(D, t["x"] @ t["Wr"] + 0.1 * torch.randn(sh.T, sh.E, device=DEV), idx)
    buf, logits = r3.LayerBuffers(D), f32(sh.T, sh.E)
    r3.forward(buf, t["x"], t["Wr"], idx, t["Wg"], t["Wu"], t["Wd"], logits_out=logits)
    counts, probs, stats, ds = torch.empty(1, sh.E, dtype=torch.int32, device=DEV), f32(1, sh.E), f32(3), f32(sh.T, sh.E)
    r3.balance_loss(D, logits, idx, stats, counts=counts, probs=probs, dlogits=ds, balance_coef=0.5, z_coef=0.01, status=buf.status)
    r3.backward(buf, t["dy"], t["x"], t["Wr"], idx, t["Wg"], t["Wu"], t["Wd"])
    assert torch.equal(counts[0], buf.counts) and buf.status.item() == 0
    dWr = buf.dW_r + t["x"].T @ ds
    x, W = t["x"].double(), t["Wr"].double().requires_grad_()
    p = torch.softmax(x @ W, 1)
    load = counts[0].double() * sh.E / (sh.K * sh.T)
    loss = 0.5 * (load * p.mean(0)).sum() + float(np.float32(0.01)) * (torch.logsumexp(x @ W, 1) ** 2).mean()
    loss.backward()
    # sums of 256 products for the logits, of 600 for the gradient
    assert abs(stats[0].item() - loss.item()) < 256 * 2.0 ** -24 * abs(loss.item())
    assert float(((t["x"].T @ ds).double() - W.grad).norm() / W.grad.norm()) < 600 * 2.0 ** -24
    for G in (dWr, buf.dW_gate, buf.dW_up, buf.dW_down):
        for to in (torch.float32, torch.bfloat16):
            out = torch.empty_like(G, dtype=to)
            r3.orthogonalize(G, out, scale=0.2 * max(G.shape[-2:]) ** 0.5)
            o, g = (out, G) if G.dim() == 3 else (out[None], G[None])
            for i in range(0, o.shape[0], 5):
                want, tol = ref.orthogonalize(g[i].double().cpu().numpy(), scale=0.2 * max(G.shape[-2:]) ** 0.5, to="f32" if to is torch.float32 else "bf16")
                assert np.linalg.norm(o[i].double().cpu().numpy() - want) <= tol


def _calls():
    """One call of each kind over several launches and one over a single one: (run, outputs), the workspaces their own."""
    g = torch.Generator(device=DEV).manual_seed(9)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    out = []
    for n, nseq in ((900, 5), (30000, 40), (200000, 3)):
        D = r3.policy_desc(n, nseq, ratio="sequence", norm="sequences", kl_coef=0.1)
        starts = (torch.arange(nseq + 1, device=DEV) * (n // nseq)).int()
        a = dict(logp=-rand(n).abs(), adv=rand(n))
        a.update(old=a["logp"] + 0.1 * rand(n), ref=a["logp"] + 0.1 * rand(n))
        o = dict(stats=f32(8), dlogp=f32(n))
        ws = r3.policy_loss_workspace(D)
        out.append((lambda D=D, a=a, o=o, ws=ws, starts=starts: r3.policy_loss(D, a["logp"], a["adv"], o["stats"], logp_old=a["old"], logp_ref=a["ref"],
                                                                               seq_start=starts, dlogp=o["dlogp"], ws=ws), o))
    for T, E, nseq in ((100, 16, 2), (5000, 128, 7)):
        L = r3.desc(T, 8, E, 2, 8)
        starts = (torch.arange(nseq + 1, device=DEV) * (T // nseq)).int()
        z, idx = rand(T, E), torch.randint(0, E, (T, 2), generator=g, device=DEV).to(torch.uint8)
        o = dict(stats=f32(3), counts=torch.empty(nseq, E, dtype=torch.int32, device=DEV), probs=f32(nseq, E), dlogits=f32(T, E))
        ws = r3.balance_loss_workspace(L, nseq)
        out.append((lambda L=L, z=z, idx=idx, o=o, ws=ws, starts=starts: r3.balance_loss(L, z, idx, seq_start=starts, z_coef=0.01, ws=ws, **o), o))
    for b, r, c, to in ((2, 100, 300, torch.float32), (24, 520, 600, torch.bfloat16), (40, 300, 700, torch.float32), (3, 900, 128, torch.bfloat16),
                        (300, 60, 200, torch.bfloat16), (2, 130, 2000, torch.bfloat16)):
        G, o = rand(b, r, c), dict(O=torch.empty(b, r, c, dtype=to, device=DEV))
        ws = r3.orthogonalize_workspace(G, o["O"])
        out.append((lambda G=G, o=o, ws=ws: r3.orthogonalize(G, o["O"], ws=ws), o))
    return out


def _wipe(o):
    for v in o.values():
        v.fill_(7)


def test_on_other_streams_and_at_once():
    calls = _calls()
    want = []
    for run, o in calls:
        run()
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in o.items()})
        _wipe(o)
    streams = [torch.cuda.Stream() for _ in calls]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for s, (run, o) in zip(streams, calls):
            with torch.cuda.stream(s):
                _wipe(o)
                run()
    torch.cuda.synchronize()
    for (run, o), w in zip(calls, want):
        for k in o:
            assert torch.equal(o[k], w[k]), k


def test_replays_from_a_graph():
    calls = _calls()
    want = []
    for run, o in calls:
        run()
        want.append({k: v.clone() for k, v in o.items()})
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for run, _ in calls:
            run()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            for run, _ in calls:
                run()
    torch.cuda.current_stream().wait_stream(side)
    for replay in range(4):
        for _, o in calls:
            _wipe(o)
        scratch = torch.randn(1 << 20, device=DEV).sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.isfinite(scratch)
        for (_, o), w in zip(calls, want):
            for k in o:
                assert torch.equal(o[k], w[k]), (k, replay)


def test_two_graphs_that_share_a_workspace():
    g = torch.Generator(device=DEV).manual_seed(11)
    Gs = [torch.randn(3, 200, 400, generator=g, device=DEV) for _ in range(2)]
    outs = [torch.empty_like(G) for G in Gs]
    ws = r3.orthogonalize_workspace(Gs[0], outs[0])
    want = []
    for G, o in zip(Gs, outs):
        r3.orthogonalize(G, o, ws=ws)
        want.append(o.clone())
    side, graphs = torch.cuda.Stream(), [torch.cuda.CUDAGraph() for _ in Gs]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for graph, G, o in zip(graphs, Gs, outs):
            r3.orthogonalize(G, o, ws=ws)
            side.synchronize()
            with torch.cuda.graph(graph, stream=side):
                r3.orthogonalize(G, o, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for o in outs:
            o.fill_(7)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


@pytest.mark.parametrize("by", [1, 2, 3])
def test_arrays_that_begin_at_any_element(by):
    g = torch.Generator().manual_seed(by)

    def odd(v):
        big = torch.zeros(v.numel() + 8, dtype=v.dtype, device=DEV)
        big[by:by + v.numel()] = v.reshape(-1).to(DEV)
        return big[by:by + v.numel()].view(v.shape)

    n = 5000
    starts = torch.tensor([0, 1700, 4100], dtype=torch.int32)
    a = [torch.randn(n, generator=g) for _ in range(4)]
    D = r3.policy_desc(n, 2, norm="sequences", kl_coef=0.1)
    got = []
    for place in (lambda v: v.to(DEV), odd):
        s, dl = place(torch.zeros(8)), place(torch.zeros(n))
        r3.policy_loss(D, place(a[0]), place(a[1]), s, logp_old=place(a[2]), logp_ref=place(a[3]), seq_start=place(starts), dlogp=dl)
        got.append((s, dl))
    assert all(torch.equal(x, y) for x, y in zip(*got))
    T, E = 333, 24
    z, idx = torch.randn(T, E, generator=g), torch.randint(0, E, (T, 3), generator=g).to(torch.uint8)
    L, got = r3.desc(T, 8, E, 3, 8), []
    for place in (lambda v: v.to(DEV), odd):
        o = dict(stats=place(torch.zeros(3)), counts=place(torch.zeros(1, E, dtype=torch.int32)), probs=place(torch.zeros(1, E)), dlogits=place(torch.zeros(T, E)))
        r3.balance_loss(L, place(z), place(idx), z_coef=0.1, **o)
        got.append(o)
    assert all(torch.equal(got[0][k], got[1][k]) for k in got[0])
    for shape in ((2, 37, 50), (2, 300, 41), (30, 300, 270)):
        for src in (torch.float32, torch.bfloat16):
            G, got = torch.randn(shape, generator=g).to(src), []
            for place in (lambda v: v.to(DEV), odd):
                out = place(torch.zeros(shape, dtype=src))
                r3.orthogonalize(place(G), out)
                got.append(out)
            assert torch.equal(*got)


def test_past_2_to_31_elements():
    g = torch.Generator(device=DEV).manual_seed(1)
    # rows of logits far apart
    T, E, ld = 70000, 16, 40000
    full = torch.zeros(T * ld, device=DEV)
    z = full.view(T, ld)[:, :E]
    z.copy_(torch.randn(T, E, generator=g, device=DEV))
    idx = torch.randint(0, E, (T, 2), generator=g, device=DEV).to(torch.uint8)
    L = r3.desc(T, 8, E, 2, 8)
    a, b = f32(T, E), f32(3)
    r3.balance_loss(L, z.contiguous(), idx, b, dlogits=a, z_coef=0.1)
    s = f32(3)
    r3.balance_loss(L, z, idx, s, dlogits=z, z_coef=0.1)
    assert torch.equal(s, b) and torch.equal(z, a)
    del full, z
    # a batch of matrices, in bf16 to save room
    n, r, c = 2900, 1024, 768
    assert n * r * c > 1 << 31
    G = torch.randn(29, r, c, generator=g, device=DEV).bfloat16().repeat(100, 1, 1)
    out = torch.empty_like(G)
    r3.orthogonalize(G, out)
    assert torch.equal(out[:29], out[-29:]) and torch.equal(out[:29], out[29 * 50:29 * 51])
    want, tol = ref.orthogonalize(G[-1].double().cpu().numpy(), to="bf16")
    assert np.linalg.norm(out[-1].double().cpu().numpy() - want) <= tol


def test_short_sides_past_2_to_31_elements():
    n, r, c = 17400, 121, 1030
    assert n * r * c > 1 << 31
    g = torch.Generator(device=DEV).manual_seed(2)
    G = torch.randn(29, r, c, generator=g, device=DEV).bfloat16().repeat(600, 1, 1)
    out = torch.empty_like(G)
    r3.orthogonalize(G, out)
    assert torch.equal(out[:29], out[-29:]) and torch.equal(out[:29], out[29 * 300:29 * 301])
    want, tol = ref.orthogonalize(G[-1].double().cpu().numpy(), to="bf16")
    assert np.linalg.norm(out[-1].double().cpu().numpy() - want) <= tol
