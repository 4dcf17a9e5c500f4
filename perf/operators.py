"""Performance cases of the operators for causal models whose relative bias decays.

With b_t = rate t for t <= 0 and -inf after (every position weighs e^-rate less
than the next), Eq. (10) needs no more of the past than a state of its own size:

  z_i  = [S_i phi(q_i)] / (s_i . phi(q_i)),   [S_i; s_i] = e^-rate [S_{i-1}; s_{i-1}] + [v_i; 1] phi(k_i)^T

The state of a head is [d + 1, M] (M features; its last row the denominators'),
that of a layer a row of a pool [slots, H, d + 1, M], fp32.

A case is a dict of plain values.  `op`:
  "fwd"   krpe.decay_attention_fwd: a prompt in chunks, the pool's rows left as the states behind it
  "bwd"   krpe.decay_attention_bwd: the gradients of a training step
  "step"  krpe.decay_attention_step: one token of every sequence
  "tree"  krpe.decay_attention_tree and krpe.decay_attention_commit: drafted tokens that form a
          tree, looked at from the states, then the accepted path taken into them
  "copy"  krpe.decay_state_copy: states forked, moved and freed within a pool
"""
import math

import numpy as np
import torch

own = False


def _case(name, op, B, H, d, m, dtype="bf16", features="prf", nprf=False, **more):
    return {"name": name, "op": op, "B": B, "H": H, "d": d, "m": m, "dtype": dtype, "features": features,
            "nprf": nprf, **more}


def listed():
    return [
        # a chat turn on a small model: one short prompt, where a call costs its launches
        _case("fwd-short-n128", "fwd", 1, 12, 64, 64, n=128, ragged=False, resume=False),
        # a layer of the benchmark's headline shape, fp32, as it is evaluated over whole documents
        _case("fwd-layer-n4096", "fwd", 8, 12, 64, 128, dtype="f32", n=4096, ragged=False, resume=False),
        # prefill of a 16k prompt (the causal layer of the benchmark, bf16, 256 features)
        _case("fwd-long-n16384", "fwd", 1, 16, 64, 256, n=16384, ragged=False, resume=False),
        # turns of different lengths that go on from kept states, odd sizes, normalised rows
        _case("fwd-ragged-n777", "fwd", 6, 10, 72, 90, nprf=True, n=777, ragged=True, resume=True),
        # training, BERT-base sized layer, bf16
        _case("bwd-short-n512", "bwd", 16, 12, 64, 64, n=512, ragged=False),
        # training, long fp32 sequences
        _case("bwd-long-n4096", "bwd", 2, 12, 64, 128, dtype="f32", n=4096, ragged=False),
        # one user's next token
        _case("step-one", "step", 1, 12, 64, 64, pool=4),
        # a server's next tokens, 256 sequences with 256 features (the largest states)
        _case("step-batch", "step", 256, 16, 64, 256, pool=272),
        # speculative decoding of one sequence, a small tree of drafts
        _case("tree-one-t12", "tree", 1, 16, 64, 128, T=12, pool=4),
        # speculative decoding of a full server, wide trees
        _case("tree-batch-t64", "tree", 64, 16, 64, 256, T=64, pool=72),
        # beams of a few requests reordered
        _case("copy-beams", "copy", 8, 12, 64, 64, dtype="f32", pool=8, kind="reorder"),
        # a shared prefix forked to many sequences, others moved together or freed
        _case("copy-fork", "copy", 96, 16, 64, 256, dtype="f32", pool=256, kind="mixed"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over the listed range (log-uniform, odd ones among them), options as used."""
    op = rng.choice(["fwd", "fwd", "fwd", "bwd", "bwd", "step", "step", "tree", "tree", "copy"])
    most = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        H = rng.choice([1, 2, 4, 8, 12, 16, rng.randint(1, 20)])
        d = rng.choice([64, 64, 64, 32, 128, rng.randint(8, 128)])
        m = rng.choice([32, 64, 128, 128, 256, rng.randint(16, 256)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        nprf = rng.random() < 0.25
        features = "elu" if rng.random() < 0.15 else "prf"
        if features == "elu":
            m = d
        c = _case("", op, 1, H, d, m, dtype, features, nprf)
        if op in ("fwd", "bwd"):
            c["B"] = _logint(rng, 1, 16)
            c["n"] = _logint(rng, 1 if op == "fwd" else 16, 16384 if op == "fwd" else 8192)
            c["ragged"] = rng.random() < 0.4
            if op == "fwd":
                c["resume"] = rng.random() < 0.4
        else:
            c["B"] = _logint(rng, 1, 256 if op == "step" else 96)
            c["pool"] = c["B"] + rng.randint(0, 16)
            if op == "tree":
                c["T"] = rng.choice([1, rng.randint(2, 64), rng.randint(2, 64), 64])
            if op == "copy":
                c.update(dtype="f32", nprf=False, pool=c["B"] + rng.randint(1, 64), kind=rng.choice(["reorder", "mixed"]))
        if _cost(c) > most:
            continue
        del c["name"]
        return c


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


# ------------------------------------------------------------------ inputs --
def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    host = np.random.default_rng([seed, 2106])
    B, H, d, M = c["B"], c["H"], c["d"], c["m"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    s = {"case": c}
    # half-lives from about 20 positions to about 3000, one for each head, jittered
    s["rate"] = 2.0 ** -(5 + 7 * torch.arange(H, device=dev) / max(1, H - 1) + 0.2 * randn(H))
    if c["op"] != "copy":
        s["W"] = None if c["features"] == "elu" else randn(H, M, d)
        rows = () if c["op"] == "step" else (c["T"],) if c["op"] == "tree" else (c["n"],)
        for name in ("q", "k", "v", "dz") if c["op"] == "bwd" else ("q", "k", "v"):
            # the softmax temperature split over queries and keys: N(0, 1) d^(-1/4)
            s[name] = (randn(B, H, *rows, d) * (d ** -0.25 if name in "qk" else 1.0)).to(dt)
    if c["op"] in ("fwd", "bwd"):
        s["lens"] = None
        if c["ragged"]:
            s["lens"] = torch.from_numpy(host.integers(0, c["n"] + 1, B).astype(np.int32)).to(dev)
    if c["op"] == "fwd":
        s["state"] = _states(B, H, d, M, randn) if c["resume"] else torch.zeros((B, H, d + 1, M), device=dev)
    if c["op"] in ("step", "tree", "copy"):
        s["state"] = _states(c["pool"], H, d, M, randn)
    if c["op"] in ("step", "tree"):
        # sequences sit in the pool in the order in which they came
        s["slots"] = torch.from_numpy(host.permutation(c["pool"])[:B].astype(np.int32)).to(dev)
    if c["op"] == "tree":
        parent, path = _tree(host, B, c["T"])
        s["parent"], s["path"] = torch.from_numpy(parent).to(dev), torch.from_numpy(path).to(dev)
    if c["op"] == "copy":
        if c["kind"] == "reorder":  # each beam goes on from one of the beams before
            dst = host.permutation(c["pool"])[:B]
            src = dst[host.integers(0, B, B)]
        else:  # forks of a few, moves, and one in eight freed (-1: cleared)
            order = host.permutation(c["pool"])
            dst = order[:B]
            src = np.where(host.random(B) < 0.5, order[host.integers(0, max(1, c["pool"] // 8), B)],
                           host.integers(0, c["pool"], B))
            src = np.where(host.random(B) < 0.125, -1, src)
        s["src"] = torch.from_numpy(src.astype(np.int32)).to(dev)
        s["dst"] = torch.from_numpy(dst.astype(np.int32)).to(dev)
    return s


def _states(count, H, d, M, randn):
    """States as prompts leave them: positive denominators, numerators of the size of the values' mean."""
    den = (8.0 * (0.7 * randn(count, H, 1, M)).exp()) / math.sqrt(M)
    return torch.cat([den * (0.3 * randn(count, H, d, 1) + 0.2 * randn(count, H, d, M)), den], dim=2).contiguous()


def _tree(host, B, T):
    """Trees of T drafts (parent[t] < t, -1 for the children of the last token) and one path from a root in each."""
    parent = np.full((B, T), -1, dtype=np.int32)
    path = np.full((B, T), -1, dtype=np.int32)
    for b in range(B):
        for t in range(1, T):
            # drafts prefer the likely branch: a node near the one before
            parent[b, t] = max(-1, t - 1 - int(host.geometric(0.5)) + 1)
        end, nodes = int(host.integers(0, T)), []
        while end >= 0:
            nodes.append(end)
            end = int(parent[b, end])
        path[b, :len(nodes)] = nodes[::-1]
    return parent, path


# --------------------------------------------------------------- the calls --
def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if not own:
        return _PLAIN[op](s, c)
    from paper_2106_12566_amd import krpe
    if op == "copy":
        krpe.decay_state_copy(s["state"], s["src"], s["dst"])
        return s["state"]
    more = {"nprf": c["nprf"], "features": c["features"]}
    if op == "fwd":
        z = krpe.decay_attention_fwd(s["q"], s["k"], s["v"], s["rate"], s["W"], state=s["state"], lens=s["lens"],
                                     fresh=not c["resume"], **more)
        return {"z": z, "state": s["state"]}
    if op == "bwd":
        dq, dk, dv = krpe.decay_attention_bwd(s["q"], s["k"], s["v"], s["rate"], s["W"], s["dz"], lens=s["lens"],
                                              **more)
        return {"dq": dq, "dk": dk, "dv": dv}
    if op == "step":
        z = krpe.decay_attention_step(s["q"], s["k"], s["v"], s["rate"], s["W"], s["state"], slots=s["slots"], **more)
        return {"z": z, "state": s["state"]}
    z = krpe.decay_attention_tree(s["q"], s["k"], s["v"], s["parent"], s["rate"], s["W"], s["state"],
                                  slots=s["slots"], **more)
    krpe.decay_attention_commit(s["k"], s["v"], s["path"], s["rate"], s["W"], s["state"], slots=s["slots"], **more)
    return {"z": z, "state": s["state"]}


# ------------------------------------------------------------- plain forms --
_C = 128  # positions of a chunk


def _unit(x, c):
    """x in fp32, its rows divided by their norms with nprf, and 1 / norm (1 without, 0 for a zero row)."""
    x = x.float()
    if not c["nprf"]:
        return x, torch.ones_like(x[..., :1])
    sq = (x * x).sum(-1, keepdim=True)
    inv = torch.where(sq > 0, sq.rsqrt(), torch.zeros_like(sq))
    return x * inv, inv


def _phi(x, W, c):
    """Feature map of x [B, H, rows, d], in fp32."""
    if c["features"] == "elu":
        return torch.where(x > 0, x + 1, x.clamp(max=0).exp())
    return (x @ W.mT - 0.5 * (x * x).sum(-1, keepdim=True) - 0.5 * math.log(c["m"])).exp()


def _phi_grad(df, f, x, inv, W, c):
    """Gradient of the rows from that of their features."""
    if c["features"] == "elu":
        dx = df * torch.where(x > 0, torch.ones_like(f), f)
    else:
        p = df * f
        dx = p @ W - x * p.sum(-1, keepdim=True)
    if c["nprf"]:
        dx = (dx - x * (x * dx).sum(-1, keepdim=True)) * inv
    return dx


def _with_one(v):
    return torch.cat([v, torch.ones_like(v[..., :1])], dim=-1)


def _live(s, c, dev):
    """[B, 1, n, 1]: positions before the sequence's length."""
    n = c["n"]
    lens = torch.full((c["B"],), n, device=dev) if s["lens"] is None else s["lens"]
    return (torch.arange(n, device=dev) < lens[:, None])[:, None, :, None], lens


def _split(x):
    """[B, H, n, w] -> [B, H, chunks, _C, w], zeros behind the end."""
    B, H, n, w = x.shape
    nc = -(-n // _C)
    return torch.nn.functional.pad(x, (0, 0, 0, nc * _C - n)).reshape(B, H, nc, _C, w)


def _decays(rate, nc):
    """Weights within a chunk [H, 1, C, C], from a chunk's start [H, 1, C, 1], to its end, and between chunks' ends."""
    i = torch.arange(_C, device=rate.device)
    dist = i[:, None] - i
    r = rate[:, None, None, None]
    inside = torch.where(dist >= 0, (-r * dist.clamp(min=0)).exp(), torch.zeros_like(r))
    k = torch.arange(nc, device=rate.device)
    gap = k[:, None] - 1 - k
    between = torch.where(gap >= 0, (-r[:, 0] * _C * gap.clamp(min=0)).exp(), torch.zeros_like(r[:, 0]))
    return inside, (-r * (i + 1)[:, None]).exp(), (-r * (_C - 1 - i)[:, None]).exp(), between


def _chunks(fq, fk, vh, rate, first):
    """Sums [B, H, chunks, C, d + 1] over each position's past, and the state before each chunk."""
    B, H, nc, _, M = fq.shape
    inside, since, until, between = _decays(rate, nc)
    part = (vh * until).mT @ fk
    before = (between @ part.flatten(3)).reshape(part.shape)
    if first is not None:
        k = torch.arange(nc, device=rate.device)
        before = before + (-rate[:, None] * _C * k).exp()[:, :, None, None] * first[:, :, None]
    return ((fq @ fk.mT) * inside) @ vh + since * (fq @ before.mT), before


def _plain_fwd(s, c):
    live, lens = _live(s, c, s["q"].device)
    n, d, rate = c["n"], c["d"], s["rate"]
    fq = _phi(_unit(torch.where(live, s["q"], torch.zeros_like(s["q"])), c)[0], s["W"], c)
    fk = _phi(_unit(torch.where(live, s["k"], torch.zeros_like(s["k"])), c)[0], s["W"], c)
    vh = _with_one(s["v"].float()) * live
    first = s["state"] if c["resume"] else None
    sums, _ = _chunks(_split(fq), _split(fk), _split(vh), rate, first)
    sums = sums.flatten(2, 3)[:, :, :n]
    z = torch.where(live, sums[..., :d] / sums[..., d:], torch.zeros_like(sums[..., :d]))
    left = (lens[:, None] - 1 - torch.arange(n, device=lens.device)).clamp(min=0)
    last = (vh * (-rate[:, None] * left[:, None]).exp()[..., None]).mT @ fk
    if c["resume"]:
        last = last + (-rate * lens[:, None]).exp()[:, :, None, None] * s["state"]
    s["state"].copy_(last)
    return {"z": z.to(s["q"].dtype), "state": s["state"]}


def _plain_bwd(s, c):
    live, _ = _live(s, c, s["q"].device)
    n, d, rate, W = c["n"], c["d"], s["rate"], s["W"]
    (q, iq), (k, ik) = (_unit(torch.where(live, s[x], torch.zeros_like(s[x])), c) for x in ("q", "k"))
    fq, fk = _split(_phi(q, W, c)), _split(_phi(k, W, c))
    vh = _split(_with_one(s["v"].float()) * live)
    sums, before = _chunks(fq, fk, vh, rate, None)
    on = _split(live.expand(-1, c["H"], -1, 1).float())
    den = torch.where(on > 0, sums[..., d:], torch.ones_like(on))
    dz = _split(torch.where(live, s["dz"], torch.zeros_like(s["dz"])).float())
    g = torch.cat([dz, -(dz * (sums[..., :d] / den)).sum(-1, keepdim=True)], dim=-1) / den * on
    inside, since, until, between = _decays(rate, fq.shape[2])
    # what the later chunks' queries ask of a chunk's end
    after = (between.mT @ ((g * since).mT @ fq).flatten(3)).reshape(before.shape)
    A = (fq @ fk.mT) * inside
    R = (g @ vh.mT) * inside
    dvh = A.mT @ g + until * (fk @ after.mT)
    dfq = R @ fk + since * (g @ before)
    dfk = R.mT @ fq + until * (vh @ after)
    out = []
    for df, f, x, inv in ((dfq, fq, q, iq), (dfk, fk, k, ik)):
        out.append(_phi_grad(df.flatten(2, 3)[:, :, :n], f.flatten(2, 3)[:, :, :n], x, inv, W, c))
    out.append(dvh.flatten(2, 3)[:, :, :n, :d])
    return {name: torch.where(live, x, torch.zeros_like(x)).to(s["q"].dtype) for name, x in zip(("dq", "dk", "dv"), out)}


def _plain_step(s, c):
    d, at = c["d"], s["slots"].long()
    fq, fk = (_phi(_unit(s[x][:, :, None], c)[0], s["W"], c) for x in ("q", "k"))
    new = (-s["rate"])[:, None, None].exp() * s["state"][at] + _with_one(s["v"].float())[..., None] * fk
    s["state"][at] = new
    sums = (new * fq).sum(-1)
    return {"z": (sums[..., :d] / sums[..., d:]).to(s["q"].dtype), "state": s["state"]}


def _plain_tree(s, c):
    B, T, d, rate, at = c["B"], c["T"], c["d"], s["rate"], s["slots"].long()
    par = (s["parent"][..., None] == torch.arange(T, device=rate.device)).float()
    seen = par + torch.eye(T, device=rate.device)
    for _ in range(6):  # ancestors up to 64 steps away
        seen = (seen @ seen).clamp(max=1)
    depth = seen.sum(-1) - 1
    fq, fk = (_phi(_unit(s[x], c)[0], s["W"], c) for x in ("q", "k"))
    vh = _with_one(s["v"].float())
    r = rate[:, None, None]
    gap = (depth[:, :, None] - depth[:, None, :])[:, None]
    w = torch.where(seen[:, None] > 0, (-r * gap.clamp(min=0)).exp(), torch.zeros_like(r))
    old = s["state"][at]
    sums = ((fq @ fk.mT) * w) @ vh + (-r * (depth[:, None, :, None] + 1)).exp() * (fq @ old.mT)
    # the accepted path, oldest first
    path = s["path"].long()
    there = path >= 0
    count = there.sum(-1)
    pick = path.clamp(min=0)[:, None, :, None]
    fk = fk.gather(2, pick.expand(-1, c["H"], -1, fk.shape[-1]))
    vh = vh.gather(2, pick.expand(-1, c["H"], -1, d + 1))
    left = (count[:, None] - 1 - torch.arange(T, device=rate.device)).clamp(min=0)
    vh = vh * ((-rate[:, None] * left[:, None]).exp() * there[:, None])[..., None]
    s["state"][at] = (-rate * count[:, None]).exp()[:, :, None, None] * old + vh.mT @ fk
    return {"z": (sums[..., :d] / sums[..., d:]).to(s["q"].dtype), "state": s["state"]}


def _plain_copy(s, c):
    src, dst = s["src"].long(), s["dst"].long()
    there = (src >= 0)[:, None, None, None]
    s["state"][dst] = torch.where(there, s["state"][src.clamp(min=0)], torch.zeros_like(s["state"][:1]))
    return s["state"]


_PLAIN = {"fwd": _plain_fwd, "bwd": _plain_bwd, "step": _plain_step, "tree": _plain_tree, "copy": _plain_copy}


# -------------------------------------------------------------------- work --
def work(case):
    c = case
    B, H, d, m = c["B"], c["H"], c["d"], c["m"]
    cells = (d + 1) * m
    if c["op"] == "copy":
        # every target is written once; sources are at most as many slots as there are moves
        return {"bytes": 2 * B * H * cells * 4 + 8 * B, "flops": 0}
    es = 2 if c["dtype"] == "bf16" else 4
    elu = c["features"] == "elu"
    weights = H * 4 + (0 if elu else H * m * d * 4)
    proj = 0 if elu else 2.0 * m * d  # of one row
    # a position's token: the state's update and its product with phi(q), or the pairs of a short sequence
    if c["op"] == "fwd":
        rows = B * H * c["n"]
        states = B * H * cells * 4 * (2 if c["resume"] else 1)
        per = min(4.0 * cells, 2.0 * cells + c["n"] * (m + d + 1.0))
        return {"bytes": 4 * rows * d * es + weights + states, "flops": rows * (2 * proj + per)}
    if c["op"] == "bwd":
        rows = B * H * c["n"]
        per = min(12.0 * cells, c["n"] * (3.0 * m + 3.0 * (d + 1)))
        return {"bytes": 7 * rows * d * es + weights, "flops": rows * (4 * proj + per)}
    states = 2 * B * H * cells * 4
    if c["op"] == "step":
        return {"bytes": 4 * B * H * d * es + weights + states, "flops": B * H * (2 * proj + 4.0 * cells)}
    T = c["T"]
    return {"bytes": 4 * B * H * T * d * es + weights + states + 8 * B * T,
            "flops": B * H * T * (2 * proj + 4.0 * cells + T * (m + d + 1.0))}


# ----------------------------------------------------------------- 64 bits --
def exact(case, seed):
    c, s = case, prepare(case, seed)
    B, H, d = c["B"], c["H"], c["d"]
    f64 = torch.float64
    state = s["state"].to(f64) if "state" in s else None
    if c["op"] == "copy":
        out = state.clone()
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            out[b] = state[a] if a >= 0 else 0.0
        return out
    rate = s["rate"].to(f64)
    if c["op"] in ("fwd", "bwd"):
        lens = [c["n"]] * B if s["lens"] is None else s["lens"].tolist()
        out = {"z": torch.zeros(s["q"].shape, dtype=f64, device=rate.device)} if c["op"] == "fwd" else \
            {x: torch.zeros(s["q"].shape, dtype=f64, device=rate.device) for x in ("dq", "dk", "dv")}
        if c["op"] == "fwd":
            out["state"] = state.clone()
        for h in range(H):
            for b in range(B):
                _exact_sequence(s, c, b, h, lens[b], rate[h], out, state)
        return out
    slots = s["slots"].tolist()
    z = torch.zeros(s["q"].shape, dtype=f64, device=rate.device)
    new = state.clone()
    fade = (-rate).exp()[:, None, None]
    fq, fk = (_phi64(s[x], s["W"], c) for x in ("q", "k"))
    vh = _with_one(s["v"].to(f64))
    if c["op"] == "step":
        for b in range(B):
            new[slots[b]] = fade * state[slots[b]] + vh[b][:, :, None] * fk[b][:, None, :]
            sums = (new[slots[b]] @ fq[b][:, :, None])[..., 0]
            z[b] = sums[:, :d] / sums[:, d:]
        return {"z": z, "state": new}
    parent, path = s["parent"].tolist(), s["path"].tolist()
    for b in range(B):
        behind = []  # the state behind each drafted token
        for t in range(c["T"]):
            past = state[slots[b]] if parent[b][t] < 0 else behind[parent[b][t]]
            behind.append(fade * past + vh[b, :, t][:, :, None] * fk[b, :, t][:, None, :])
            sums = (behind[t] @ fq[b, :, t][:, :, None])[..., 0]
            z[b, :, t] = sums[:, :d] / sums[:, d:]
        taken = [t for t in path[b] if t >= 0]
        if taken:
            new[slots[b]] = behind[taken[-1]]
    return {"z": z, "state": new}


def _phi64(x, W, c):
    """Feature map in 64 bits of x [..., d], W [..., m, d]."""
    x = x.to(torch.float64)
    if c["nprf"]:
        norm = x.norm(dim=-1, keepdim=True)
        x = torch.where(norm > 0, x / norm, torch.zeros_like(x))
    if c["features"] == "elu":
        return torch.where(x > 0, x + 1, x.exp())
    W = W.to(torch.float64)
    # (step's x is one row of each head)
    p = (W @ x[..., None])[..., 0] if c["op"] == "step" else x @ W.mT
    return (p - 0.5 * (x * x).sum(-1, keepdim=True)).exp() / math.sqrt(c["m"])


def _exact_sequence(s, c, b, h, n, rate, out, state):
    """One sequence of one head by its pairs of positions: Eq. (10) with b_t = rate t, and its gradients."""
    d = c["d"]
    f64 = torch.float64
    W = None if s["W"] is None else s["W"][h]
    if n == 0:
        if c["op"] == "fwd" and not c["resume"]:
            out["state"][b, h] = 0.0
        return
    q, k, v = (s[x][b, h, :n].to(f64) for x in ("q", "k", "v"))
    fq, fk, vh = _phi64(q, W, c), _phi64(k, W, c), _with_one(v)
    at = torch.arange(n, device=rate.device, dtype=f64)
    if c["op"] == "bwd":
        dfq, dfk, dv = torch.zeros_like(fq), torch.zeros_like(fk), torch.zeros_like(v)
    rows = max(64, (1 << 25) // n)
    for i0 in range(0, n, rows):
        i1 = min(n, i0 + rows)
        dist = at[i0:i1, None] - at[None, :i1]
        C = torch.where(dist >= 0, (-rate * dist).exp(), torch.zeros_like(dist))
        A = (fq[i0:i1] @ fk[:i1].T) * C
        sums = A @ vh[:i1]
        if c["op"] == "fwd":
            if c["resume"]:
                sums = sums + (-rate * (at[i0:i1, None] + 1)).exp() * (fq[i0:i1] @ state[b, h].T)
            out["z"][b, h, i0:i1] = sums[:, :d] / sums[:, d:]
            continue
        z, den = sums[:, :d] / sums[:, d:], sums[:, d:]
        gz = s["dz"][b, h, i0:i1].to(f64) / den
        R = (gz @ v[:i1].T - (gz * z).sum(-1, keepdim=True)) * C
        dv[:i1] += A.T @ gz
        dfq[i0:i1] = R @ fk[:i1]
        dfk[:i1] += R.T @ fq[i0:i1]
    if c["op"] == "fwd":
        last = (vh * (-rate * (n - 1 - at)).exp()[:, None]).T @ fk
        if c["resume"]:
            last = last + (-rate * n).exp() * state[b, h]
        out["state"][b, h] = last
        return
    out["dv"][b, h, :n] = dv
    for name, x, f, df in (("dq", q, fq, dfq), ("dk", k, fk, dfk)):
        norm = x.norm(dim=-1, keepdim=True) if c["nprf"] else torch.ones_like(x[:, :1])
        u = torch.where(norm > 0, x / norm, torch.zeros_like(x))
        if c["features"] == "elu":
            du = df * torch.where(u > 0, torch.ones_like(u), u.exp())
        else:
            du = (df * f) @ W.to(f64) - u * (df * f).sum(-1, keepdim=True)
        if c["nprf"]:
            du = torch.where(norm > 0, (du - u * (u * du).sum(-1, keepdim=True)) / norm, torch.zeros_like(du))
        out[name][b, h, :n] = du
