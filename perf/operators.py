"""Performance cases of the operators around a training step: log-probabilities of the sampled tokens with entropy and
top alternatives, their gradient, and the gradients of the weighted combination and of the dispatch to experts.

Four operators (``op`` of a case):

``logprobs``      [n, V] logits -> log-probability of each row's token, entropy, the softmax's two statistics and, where
                  ``top`` > 0, the most probable alternatives.  A row whose target is -1 (prompt, padding) is left out.
``logprobs_bwd``  gradients of the log-probabilities (and, with ``ent``, the entropies) -> gradient of the logits.
``combine_bwd``   gradient of y -> gradients of the expert outputs' rows, of the gates and of the selected logits.
``permute_bwd``   gradient of the rows sorted by expert -> gradient of the tokens (``add``: beside the router's own term).

With ``own`` false ``run`` is elementary torch in 32 bits; with ``own`` true it is the framework's call.
"""
import math

import torch

own = False

_STEP = 1 << 27        # elements that are made, or computed in 64 bits, at a time


def _lp(name, n, V, dtype, top=0, scale=1.0, skip=0.0, masked=False, pad=0):
    return {"name": name, "op": "logprobs", "n": n, "V": V, "dtype": dtype, "top": top, "scale": scale, "skip": skip,
            "masked": masked, "pad": pad}


def _lb(name, n, V, dtype, ent=True, scale=1.0, skip=0.0, masked=False, pad=0):
    return {"name": name, "op": "logprobs_bwd", "n": n, "V": V, "dtype": dtype, "ent": ent, "scale": scale, "skip": skip,
            "masked": masked, "pad": pad}


def _cb(name, T, d, E, K, act):
    return {"name": name, "op": "combine_bwd", "T": T, "d": d, "E": E, "K": K, "act": act}


def _pb(name, T, d, E, K, act, add=False):
    return {"name": name, "op": "permute_bwd", "T": T, "d": d, "E": E, "K": K, "act": act, "add": add}


def listed():
    return [
        # one decoded token: its log-probability and the 20 alternatives that a rollout's log keeps; launches are the time
        _lp("lp_decode_1", 1, 151936, "bf16", top=20),
        # one decode step of a batch under a grammar: half of an odd-sized f32 vocabulary is masked with -inf, temperature 0.6
        _lp("lp_decode_64_masked", 64, 50257, "f32", top=8, scale=1.0 / 0.6, masked=True),
        # scoring a rollout with its alternatives, prompts left out
        _lp("lp_score_4k_top20", 4096, 151936, "bf16", top=20, skip=0.25),
        # recompute stage: old-policy log-probabilities and entropies of a whole training batch
        _lp("lp_recompute_16k", 16384, 151936, "bf16"),
        # gradient over a small f32 vocabulary (numerics study), rows padded to a multiple of 64
        _lb("lpb_f32_500", 500, 32000, "f32", pad=40),
        # gradient of an odd-sized vocabulary: no row but the first is aligned; log-probabilities only
        _lb("lpb_odd_3k", 3001, 50257, "bf16", ent=False),
        # update stage: gradient of policy loss and entropy bonus, prompts left out
        _lb("lpb_8k", 8192, 151936, "bf16", skip=0.25),
        # the unit-test layer in f32
        _cb("cb_f32_256", 256, 128, 8, 2, "f32"),
        # the ordinary training batch of the 2048-wide, 128-expert layer
        _cb("cb_64k", 65536, 2048, 128, 8, "bf16"),
        # ragged width, top-6, odd token count
        _pb("pb_ragged_3k", 3001, 1000, 64, 6, "bf16"),
        # the same ordinary batch, added to the router's term
        _pb("pb_64k_add", 65536, 2048, 128, 8, "bf16", add=True),
        # a small batch of the same layer: some of the chip's compute units and a few microseconds
        _cb("cb_512", 512, 2048, 128, 8, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs"] * 4 + ["logprobs_bwd"] * 3 + ["combine_bwd"] * 2 + ["permute_bwd"] * 2)
    if op in ("logprobs", "logprobs_bwd"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        V = _log(rng, 500, 262144)
        if rng.random() < 0.5:
            V = max(8, V // 8 * 8)
        n = _log(rng, 1, 32768)
        most = 16384 * 151936 * 2 // (2 if op == "logprobs_bwd" else 1)      # bytes of logits in the largest listed case
        n = max(1, min(n, most // (V * (2 if dtype == "bf16" else 4))))
        more = dict(scale=rng.choice([1.0, 1.0, 1.0 / 0.6, 0.5]), skip=rng.choice([0.0, 0.0, 0.3]) if n > 8 else 0.0,
                    masked=rng.random() < 0.25, pad=rng.choice([0, 0, 3, 64]))
        if op == "logprobs":
            # alternatives are asked for in decode and scoring, not over the whole of the largest batches
            top = rng.choice([0, 1, 5, 20, 32]) if n * V <= 4096 * 151936 else 0
            c = _lp("", n, V, dtype, top=top, **more)
        else:
            c = _lb("", n, V, dtype, ent=rng.random() < 0.5, **more)
    else:
        act = rng.choice(["bf16", "bf16", "f32"])
        d = rng.choice([128, 512, 768, 1000, 1024, 2048, 2880, 4096, 501])
        E, K = rng.choice([(8, 2), (16, 1), (64, 6), (128, 8), (256, 8), (384, 4), (60, 5)])
        T = _log(rng, 1, 65536)
        T = max(1, min(T, 65536 * 2048 * 8 * 2 // (d * K * (2 if act == "bf16" else 4))))
        c = _cb("", T, d, E, K, act) if op == "combine_bwd" else _pb("", T, d, E, K, act, add=rng.random() < 0.5)
    del c["name"]
    return c


def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _rows(c):
    return max(1, _STEP // c["V"])


def _stats(z, scale):
    """max, sum of exponentials and entropy of each row in 64 bits, some rows at a time"""
    out = []
    for part in z.split(max(1, _STEP // 4 // z.shape[1])):
        x = part.double()
        m = x.amax(1)
        x = (x - m[:, None]) * scale
        e = x.exp()
        S = e.sum(1)
        H = S.log() - torch.where(e > 0, e * x, torch.zeros_like(e)).sum(1) / S
        out.append(torch.stack([m, S, H]))
    m, S, H = torch.cat(out, 1).float()
    return torch.stack([m, S], 1).contiguous(), H.contiguous()


def _logits(c, g):
    """Logits of a trained model's head in kind: a spread of about 2, the sampled token usually well above it."""
    n, V = c["n"], c["V"]
    full = torch.empty(n, V + c["pad"], dtype=_dt(c["dtype"]), device="cuda")
    target = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    lift = 6.0 + 2.0 * torch.randn(n, generator=g, device="cuda")
    mask = torch.rand(V, generator=g, device="cuda") < 0.5 if c["masked"] else None
    for a in range(0, n, _rows(c)):
        b = min(n, a + _rows(c))
        x = torch.randn(b - a, V + c["pad"], generator=g, device="cuda") * 2.0
        t = target[a:b].long()[:, None]
        if mask is not None:
            x[:, :V].masked_fill_(mask, -math.inf)
            x.scatter_(1, t, 0.0)
        x.scatter_add_(1, t, lift[a:b, None])
        full[a:b] = x
    if c["skip"]:
        target[torch.rand(n, generator=g, device="cuda") < c["skip"]] = -1
    return full[:, :V], target


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    f32 = lambda *shape: torch.empty(*shape, dtype=torch.float32, device="cuda")  # noqa: E731
    if c["op"] == "logprobs":
        n, V, top = c["n"], c["V"], c["top"]
        s["logits"], s["target"] = _logits(c, g)
        s["logp"], s["entropy"], s["stats"] = f32(n), f32(n), f32(n, 2)
        s["top_logp"] = f32(n, top) if top else None
        s["top_id"] = torch.empty(n, top, dtype=torch.int32, device="cuda") if top else None
        s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    elif c["op"] == "logprobs_bwd":
        n, V = c["n"], c["V"]
        s["logits"], s["target"] = _logits(c, g)
        s["stats"], s["entropy"] = _stats(s["logits"], c["scale"])
        s["dlogp"] = torch.randn(n, generator=g, device="cuda") / n          # advantages over the batch's mean
        s["dent"] = torch.full((n,), -0.01 / n, device="cuda") * (0.5 + torch.rand(n, generator=g, device="cuda")) if c["ent"] else None
        s["dlogits"] = torch.empty(n, V, dtype=_dt(c["dtype"]), device="cuda")
    else:
        T, d, E, K, act = c["T"], c["d"], c["E"], c["K"], _dt(c["act"])
        idx = torch.rand(T, E, generator=g, device="cuda").topk(K, 1).indices.sort(1).values      # recorded experts
        perm = idx.reshape(-1).argsort(stable=True)
        inv = torch.empty_like(perm)
        inv[perm] = torch.arange(T * K, device="cuda")
        s["inv_perm"] = inv.int()
        rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(act)  # noqa: E731
        if c["op"] == "combine_bwd":
            s["dy"], s["Yp"] = rand(T, d), rand(T * K, d)
            s["gates"] = torch.randn(T, K, generator=g, device="cuda").softmax(1)
            s["dYp"] = torch.empty(T * K, d, dtype=act, device="cuda")
            s["dgates"], s["dz"] = f32(T, K), f32(T, K)
        else:
            s["dXp"] = rand(T * K, d)
            s["add"] = rand(T, d) if c["add"] else None
            s["dx"] = torch.empty(T, d, dtype=act, device="cuda")
    return s


def _workspace(s, make):
    """The workspace and the call's descriptor, kept with the state as a user's program keeps them"""
    if "kept" not in s:
        s["kept"] = make()
    return s["kept"]


def _run_own(s):
    from paper_2510_11370_amd import r3
    c = s["case"]
    if c["op"] == "logprobs":
        ws = _workspace(s, lambda: r3.token_logprobs_workspace(c["n"], c["V"], c["top"]))
        r3.token_logprobs(s["logits"], s["target"], s["logp"], entropy=s["entropy"], stats=s["stats"], top_logp=s["top_logp"],
                          top_id=s["top_id"], scale=c["scale"], status=s["status"], ws=ws)
        return {k: s[k] for k in ("logp", "entropy", "stats", "top_logp", "top_id")}
    if c["op"] == "logprobs_bwd":
        r3.token_logprobs_backward(s["logits"], s["target"], s["stats"], s["dlogits"], dlogp=s["dlogp"], entropy=s["entropy"],
                                   dentropy=s["dent"], scale=c["scale"])
        return {"dlogits": s["dlogits"]}
    D = _workspace(s, lambda: r3.desc(c["T"], c["d"], c["E"], c["K"], 16, _dt(c["act"])))
    if c["op"] == "combine_bwd":
        r3.combine_backward(D, s["dy"], s["Yp"], s["gates"], s["inv_perm"], dYp=s["dYp"], dgates=s["dgates"], dz=s["dz"])
        return {k: s[k] for k in ("dYp", "dgates", "dz")}
    r3.permute_backward(D, s["dXp"], s["inv_perm"], s["dx"], add=s["add"])
    return {"dx": s["dx"]}


def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    if c["op"] == "logprobs":
        target = s["target"].long()
        live = target >= 0
        z = s["logits"].float()
        m = z.amax(1)
        x = (z - m[:, None]) * c["scale"]
        e = x.exp()
        S = e.sum(1)
        logS = S.log()
        H = logS - torch.where(e > 0, e * x, torch.zeros_like(e)).sum(1) / S
        logp = x.gather(1, target.clamp(min=0)[:, None])[:, 0] - logS
        zero = torch.zeros_like(logp)
        out = {"logp": torch.where(live, logp, zero), "entropy": torch.where(live, H, zero),
               "stats": torch.where(live[:, None], torch.stack([m, S], 1), zero[:, None]), "top_logp": None, "top_id": None}
        if c["top"]:
            del e
            k = min(c["top"], c["V"])
            bits = (z + 0.0).view(torch.int32)
            order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()          # the floats' order as whole numbers
            key = (order << 32) | (0xFFFFFFFF - torch.arange(c["V"], device=z.device))  # ties: the lower id is the larger key
            best = key.topk(k, 1).values
            ids = 0xFFFFFFFF - (best & 0xFFFFFFFF)
            lp = x.gather(1, ids) - logS[:, None]
            none = torch.isinf(lp) | ~live[:, None]
            lp = torch.where(none, torch.full_like(lp, -math.inf), lp)
            ids = torch.where(none, torch.full_like(ids, -1), ids).int()
            out["top_logp"] = torch.nn.functional.pad(lp, (0, c["top"] - k), value=-math.inf)
            out["top_id"] = torch.nn.functional.pad(ids, (0, c["top"] - k), value=-1)
        return out
    if c["op"] == "logprobs_bwd":
        target = s["target"].long()
        live = (target >= 0)[:, None]
        m, S = s["stats"][:, :1], s["stats"][:, 1:]
        x = (s["logits"].float() - m) * c["scale"]
        p = x.exp() / S
        w = s["dlogp"][:, None]
        if c["ent"]:
            w = w + torch.where(p > 0, s["dent"][:, None] * (x - S.log() + s["entropy"][:, None]), torch.zeros_like(p))
        dz = -p * w
        dz.scatter_add_(1, target.clamp(min=0)[:, None], s["dlogp"][:, None])
        return {"dlogits": torch.where(live, dz * c["scale"], torch.zeros_like(dz)).to(s["logits"].dtype)}
    T, d, K = c["T"], c["d"], c["K"]
    rows = s["inv_perm"].long()
    if c["op"] == "combine_bwd":
        dy, g = s["dy"].float()[:, None, :], s["gates"]
        dYp = torch.empty_like(s["Yp"])
        dYp[rows] = (g[:, :, None] * dy).to(s["Yp"].dtype).view(T * K, d)
        dg = (s["Yp"].float()[rows].view(T, K, d) * dy).sum(2)
        return {"dYp": dYp, "dgates": dg, "dz": g * (dg - (g * dg).sum(1, keepdim=True))}
    dx = s["dXp"].float()[rows].view(T, K, d).sum(1)
    if c["add"]:
        dx = dx + s["add"].float()
    return {"dx": dx.to(s["dXp"].dtype)}


def work(c):
    if c["op"] in ("logprobs", "logprobs_bwd"):
        n, V, b = c["n"], c["V"], 2 if c["dtype"] == "bf16" else 4
        read = n * (1.0 - c["skip"]) * V * b
        if c["op"] == "logprobs":
            return {"bytes": read + n * (4 + 16 + 8 * c["top"]), "flops": 6.0 * n * (1.0 - c["skip"]) * V}
        return {"bytes": read + n * V * b + n * (24 if c["ent"] else 16), "flops": 6.0 * n * (1.0 - c["skip"]) * V}
    T, d, K, b = c["T"], c["d"], c["K"], 2 if c["act"] == "bf16" else 4
    if c["op"] == "combine_bwd":
        return {"bytes": float(T * d * b + 2 * T * K * d * b + 16 * T * K), "flops": 3.0 * T * K * d}
    return {"bytes": float(T * K * d * b + (2 if c["add"] else 1) * T * d * b + 4 * T * K), "flops": float(T * K * d)}


def exact(c, seed):
    """The outputs from the definitions, in 64 bits, some rows at a time."""
    s = prepare(c, seed)
    if c["op"] in ("logprobs", "logprobs_bwd"):
        z, t, got = s["logits"], s["target"].long(), []
        step = max(1, _STEP // 4 // c["V"])
        for a in range(0, c["n"], step):
            zz, tt = z[a:a + step].double(), t[a:a + step]
            lse = torch.logsumexp(c["scale"] * zz, 1)
            logq = c["scale"] * zz - lse[:, None]
            q = torch.softmax(c["scale"] * zz, 1)
            H = -torch.special.xlogy(q, q).sum(1)
            keep = (tt >= 0).double()
            at = tt.clamp(min=0)[:, None]
            if c["op"] == "logprobs":
                top = zz.max(1).values
                r = [logq.gather(1, at)[:, 0] * keep, H * keep, torch.stack([top * keep, (lse - c["scale"] * top).exp() * keep], 1)]
                if c["top"]:
                    k = min(c["top"], c["V"])
                    v = torch.nn.functional.pad(logq.topk(k, 1).values, (0, c["top"] - k), value=-math.inf)
                    r.append(v.masked_fill(keep[:, None] == 0, -math.inf))
                got.append(r)
            else:
                one = torch.zeros_like(q).scatter_(1, at, 1.0)
                dz = s["dlogp"][a:a + step].double()[:, None] * (one - q)
                if c["ent"]:
                    dz -= s["dent"][a:a + step].double()[:, None] * (torch.special.xlogy(q, q) + q * H[:, None])
                got.append(dz * (c["scale"] * keep)[:, None])
        if c["op"] == "logprobs_bwd":
            return {"dlogits": torch.cat(got)}
        cols = [torch.cat(x) for x in zip(*got)]
        return {"logp": cols[0], "entropy": cols[1], "stats": cols[2], "top_logp": cols[3] if c["top"] else None, "top_id": None}
    T, d, K = c["T"], c["d"], c["K"]
    row = s["inv_perm"].long().view(T, K)
    step = max(1, _STEP // 4 // (K * d))
    if c["op"] == "combine_bwd":
        dYp = torch.empty(T * K, d, dtype=torch.float64, device="cuda")
        dg = torch.empty(T, K, dtype=torch.float64, device="cuda")
        for a in range(0, T, step):
            r, dy, g = row[a:a + step], s["dy"][a:a + step].double(), s["gates"][a:a + step].double()
            for j in range(K):
                dYp[r[:, j]] = dy * g[:, j:j + 1]
                dg[a:a + step, j] = (s["Yp"][r[:, j]].double() * dy).sum(1)
        g = s["gates"].double()
        jac = torch.diag_embed(g) - g[:, :, None] * g[:, None, :]           # of the softmax over the selected logits
        return {"dYp": dYp, "dgates": dg, "dz": (jac * dg[:, :, None]).sum(1)}
    dx = s["add"].double() if c["add"] else torch.zeros(T, d, dtype=torch.float64, device="cuda")
    for j in range(K):
        dx += s["dXp"][row[:, j]].double()
    return {"dx": dx}
