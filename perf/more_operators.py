"""More operators of the packed transformer body, with their plain forms and the cases they are timed on.

``perf/operators.py`` holds the attention and the joins of blocks.  Around them the body runs

  embed    rows of the embedding table for the packed tokens, scaled, and the table's gradient
  qknorm   the heads' norms of queries and keys with the position rotation, forward and backward
  experts  matrix products of rows that are grouped by expert, forward and backward

``own`` False: elementary torch operations in 32 bits (angles in 64).  ``own`` True: the library's
entry points.
"""
import math

import numpy as np
import torch

own = False


# ---------------------------------------------------------------------------- cases
def _embed(name, back, dtype, n, V, d, scale=1.0, picked=True, spare=37):
    c = dict(kind="embed", back=back, dtype=dtype, n=n, V=V, d=d, scale=scale, picked=picked, spare=spare)
    return dict(c, name=name) if name else c


def _qknorm(name, back, dtype, B, lo, hi, Hq, Hkv, D, R, len_seed, interleaved=False, norm=True, first=None, median=0):
    c = dict(kind="qknorm", back=back, dtype=dtype, B=B, lo=lo, hi=hi, median=median, Hq=Hq, Hkv=Hkv, D=D, R=R,
             interleaved=interleaved, norm=norm, first=-1 if first is None else first, len_seed=len_seed)
    return dict(c, name=name) if name else c


def _experts(name, what, dtype, E, n, n_in, n_out, skew, load_seed, spare=37):
    c = dict(kind="experts", what=what, dtype=dtype, E=E, n=n, n_in=n_in, n_out=n_out, skew=skew,
             load_seed=load_seed, spare=spare)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the Tiny configuration's tokens: latency of the lookup's gradient, its sort included
        _embed("embed_bwd_tiny_f32", True, "f32", 290, 512, 64),
        # a full Qwen3-8B-shaped batch of selected tokens, looked up through their indices
        _embed("embed_fwd_8b", False, "bf16", 166001, 151936, 4096, scale=1.0),
        # the Qwen3-0.6B-shaped batch: the gradient of a table that is mostly untouched
        _embed("embed_bwd_0p6b", True, "bf16", 74003, 151936, 1024, scale=32.0),
        # a full Qwen3-8B-shaped batch, its gradient
        _embed("embed_bwd_8b", True, "bf16", 166001, 151936, 4096),
        # the Tiny configuration's batch: latency
        _qknorm("qknorm_fwd_tiny_f32", False, "f32", 8, 8, 64, 4, 2, 64, 64, 1),
        # responses of log-normal length up to 8192, the heads of Qwen3-8B
        _qknorm("qknorm_fwd_8b", False, "bf16", 64, 16, 8192, 32, 8, 128, 128, 2, median=2048),
        # the Qwen3-0.6B-shaped batch, backward
        _qknorm("qknorm_bwd_0p6b", True, "bf16", 64, 256, 2048, 16, 8, 128, 128, 3),
        # long chains of thought (8192..32768 tokens), the heads of Qwen3-8B, backward
        _qknorm("qknorm_bwd_long_cot", True, "bf16", 8, 8192, 32768, 32, 8, 128, 128, 4),
        # rows of the Tiny configuration over four experts: latency
        _experts("experts_fwd_tiny_f32", "fwd", "f32", 4, 290, 64, 128, 0.5, 5),
        # a handful of tokens over many experts: each expert's weights are read for a few rows
        _experts("experts_fwd_few", "fwd", "bf16", 32, 200, 4096, 1536, 1.0, 6),
        # a batch of some ten thousand tokens that go to eight experts of 64 each, uneven loads, forward
        _experts("experts_fwd", "fwd", "bf16", 64, 120007, 2048, 1024, 0.7, 7),
        # a full batch, backward: the rows' gradients and the weights'
        _experts("experts_bwd", "bwd", "bf16", 64, 300013, 2048, 1536, 0.5, 8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "qknorm", "experts"])
    seed = rng.randrange(1 << 20)
    if kind == "embed":
        back = rng.random() < 0.6
        d = 8 * _log_int(rng, 1, 1024)
        V = _log_int(rng, 2, min(152000, 6.2e8 / d))
        n = _log_int(rng, 1, max(1, min(170000, 6.8e8 / d)))
        return _embed(None, back, rng.choice(["bf16", "bf16", "f32"]), n, V, d, rng.choice([1.0, 0.5, math.sqrt(d)]),
                      rng.random() < 0.5, rng.randrange(100))
    if kind == "qknorm":
        Hkv = rng.choice([1, 2, 4, 8])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 5, 8])
        D = rng.choice([32, 64, 64, 80, 96, 128, 128, 128])
        R = 16 * rng.randint(1, D // 16) if rng.random() < 0.3 else D
        hi = _log_int(rng, 1, 33000)
        lo = max(0, int(hi * rng.choice([0.0, 0.1, 0.5, 1.0])))
        B = _log_int(rng, 1, max(1, min(128, int(160000 * 5120 / (hi * (Hq + Hkv) * D)))))
        return _qknorm(None, rng.random() < 0.6, rng.choice(["bf16", "bf16", "f32"]), B, lo, hi, Hq, Hkv, D, R, seed,
                       rng.random() < 0.3, rng.random() < 0.8, rng.choice([None, None, 0, 100000]))
    f32 = rng.random() < 0.2
    E = _log_int(rng, 1, 128)
    n_in, n_out = (8 * _log_int(rng, 1, 64 if f32 else 512) for _ in range(2))
    while E * n_in * n_out > 4e8:
        E = max(1, E // 2)
    n = _log_int(rng, 1, max(1, min(300000, int((2e9 if f32 else 9e11) / (n_in * n_out)), int(1.2e9 / max(n_in, n_out)))))
    return _experts(None, rng.choice(["fwd", "bwd"]), "f32" if f32 else "bf16", E, n, n_in, n_out,
                    rng.choice([0.0, 0.5, 1.0, 2.0]), seed, rng.randrange(100))


def _lengths(c):
    r = np.random.Generator(np.random.PCG64([c["len_seed"], 78]))
    if c["median"]:
        T = np.rint(np.exp(r.normal(math.log(c["median"]), 0.75, size=c["B"])))
        return np.clip(T, c["lo"], c["hi"]).astype(np.int64)
    T = r.integers(c["lo"], c["hi"] + 1, size=c["B"])
    T[0] = max(T[0], 1)          # sequences may be empty, a batch is not
    return T


def _loads(c):
    """Rows of each expert: drawn from uneven shares; with few rows some experts have none."""
    r = np.random.Generator(np.random.PCG64([c["load_seed"], 79]))
    share = np.exp(c["skew"] * r.normal(size=c["E"]))
    return r.multinomial(c["n"], share / share.sum()).astype(np.int64)


def _shares(V):
    """How often each rank of the vocabulary occurs: the usual law of words."""
    p = 1.0 / (np.arange(V, dtype=np.float64) + 2.7)
    return p / p.sum()


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "embed":
        n, d, V = c["n"], c["d"], c["V"]
        index = 4 * n * (2 if c["picked"] else 1)
        if c["back"]:
            return {"bytes": n * d * e + 4 * V * d + index, "flops": n * d}
        seen = float((1.0 - (1.0 - _shares(V)) ** n).sum())   # rows of the table that occur
        return {"bytes": int(seen * d * e) + n * d * e + index, "flops": n * d}
    if c["kind"] == "qknorm":
        n = int(_lengths(c).sum())
        row = (c["Hq"] + c["Hkv"]) * c["D"]
        norm = 1 if c["norm"] else 0
        if c["back"]:      # reads q, k and the gradients, writes dq and dk
            return {"bytes": (2 + norm) * n * row * e, "flops": (6 + 10 * norm) * n * row}
        return {"bytes": 2 * n * row * e, "flops": (3 + 4 * norm) * n * row}
    loads = _loads(c)
    used = int((loads > 0).sum())
    x, y, w = c["n"] * c["n_in"], c["n"] * c["n_out"], c["n_in"] * c["n_out"]
    if c["what"] == "fwd":
        return {"bytes": (x + y + used * w) * e, "flops": 2 * c["n"] * w}
    return {"bytes": (2 * x + y + used * w) * e + 4 * c["E"] * w, "flops": 4 * c["n"] * w}


# --------------------------------------------------------------------------- inputs
EPS, THETA = 1e-6, 1e6


def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    c, dt, dev = case, _type(case), "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(1000003 * int(seed) + 12)

    def rand(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)

    if c["kind"] == "embed":
        n, V, d = c["n"], c["V"], c["d"]
        cap = n + c["spare"]
        s = dict(case=c, n=n, cap=cap, n_rows=torch.tensor([n], dtype=torch.int32, device=dev))
        # ids of the packed stream; the rows are a rising choice among them (prefixes of responses)
        n_tot = 2 * cap if c["picked"] else cap
        cdf = torch.from_numpy(np.cumsum(_shares(V))).to(dev)
        u = torch.rand(n_tot, generator=g, device=dev, dtype=torch.float64)
        rank = torch.searchsorted(cdf, u).clamp_(max=V - 1)
        name = torch.randperm(V, generator=g, device=dev)     # frequent words have ids all over the table
        s["ids"] = name[rank].to(torch.int32)
        s["pick"] = None
        if c["picked"]:
            order = torch.rand(n_tot, generator=g, device=dev).argsort()[:cap]
            s["pick"] = order.sort().values.to(torch.int32)
        if c["back"]:
            s.update(dx=rand(cap, d).to(dt), dtable=torch.empty(V, d, device=dev))
        else:
            s.update(table=(0.02 * rand(V, d)).to(dt), x=torch.empty(cap, d, dtype=dt, device=dev))
        return s
    if c["kind"] == "qknorm":
        T = _lengths(c)
        cu = np.zeros(c["B"] + 1, dtype=np.int32)
        np.cumsum(T, out=cu[1:])
        n, Hq, Hkv, D = int(cu[-1]), c["Hq"], c["Hkv"], c["D"]
        pos = np.arange(n) - np.repeat(cu[:-1], T)
        freq = THETA ** (-2.0 * torch.arange(c["R"] // 2, dtype=torch.float64, device=dev) / c["R"])
        s = dict(case=c, n=n, cu=torch.from_numpy(cu).to(dev), inv_freq=freq, positions=None,
                 pos=torch.from_numpy(pos).to(dev), w_q=None, w_k=None)
        if c["first"] >= 0:       # continued sequences: positions of their own
            s["pos"] = s["pos"] + c["first"]
            s["positions"] = s["pos"].to(torch.int32)
        # the projections leave q, k and v side by side in one row; a few heads are louder than others
        qkv = rand(n, Hq + 2 * Hkv, D)
        qkv[:, ::3] *= 4.0
        s["qkv"] = qkv.to(dt)
        s["q"], s["k"], _ = s["qkv"].split([Hq, Hkv, Hkv], dim=1)
        if c["norm"]:
            s["w_q"], s["w_k"] = 1.0 + 0.1 * rand(D), 1.0 + 0.1 * rand(D)
        s["qk"] = torch.empty(n, Hq + Hkv, D, dtype=dt, device=dev)
        s["q_out"], s["k_out"] = s["qk"].split([Hq, Hkv], dim=1)
        if c["back"]:
            dqk = rand(n, Hq + Hkv, D).to(dt)
            s["dq_out"], s["dk_out"] = dqk.split([Hq, Hkv], dim=1)
            s["dqkv"] = torch.empty_like(s["qkv"])
            s["dq"], s["dk"], _ = s["dqkv"].split([Hq, Hkv, Hkv], dim=1)
            if c["norm"]:
                s["dw_q"], s["dw_k"] = torch.empty(D, device=dev), torch.empty(D, device=dev)
        return s
    loads = _loads(c)
    offs = np.zeros(c["E"] + 1, dtype=np.int32)
    np.cumsum(loads, out=offs[1:])
    cap = c["n"] + c["spare"]
    s = dict(case=c, n=c["n"], cap=cap, offs_h=offs.tolist(), offs=torch.from_numpy(offs).to(dev),
             x=rand(cap, c["n_in"]).to(dt), w=(rand(c["E"], c["n_out"], c["n_in"]) / math.sqrt(c["n_in"])).to(dt))
    if c["what"] == "fwd":
        s["y"] = torch.empty(cap, c["n_out"], dtype=dt, device=dev)
    else:
        s["dy"] = rand(cap, c["n_out"]).to(dt)
        s["dx"] = torch.empty(cap, c["n_in"], dtype=dt, device=dev)
        s["dw"] = torch.empty(c["E"], c["n_out"], c["n_in"], device=dev)
    return s


# ------------------------------------------------------------------------ plain forms
def _ids_of_rows(s):
    n = s["n"]
    return (s["ids"][:n] if s["pick"] is None else s["ids"][s["pick"][:n].long()]).long()


def _embed_plain(s):
    c, ids = s["case"], _ids_of_rows(s)
    if not c["back"]:
        return (s["table"][ids].float() * c["scale"]).to(_type(c))
    out = torch.zeros(c["V"], c["d"], device="cuda")
    out.index_add_(0, ids, s["dx"][: s["n"]].float())
    return out.mul_(c["scale"])


def _angles(s):
    turn = s["pos"].double()[:, None] * s["inv_freq"][None, :]
    return turn.cos().float()[:, None, :], turn.sin().float()[:, None, :]


def _halves(c, x):
    """The two members of each rotated pair."""
    R = c["R"]
    return (x[..., 0:R:2], x[..., 1:R:2]) if c["interleaved"] else (x[..., : R // 2], x[..., R // 2: R])


def _rotate_plain(c, x, cos, sin):
    out = x.clone()
    a, b = _halves(c, x)
    to_a, to_b = _halves(c, out)
    to_a.copy_(a * cos - b * sin)
    to_b.copy_(b * cos + a * sin)
    return out


def _qknorm_plain(s):
    c, dt = s["case"], _type(s["case"])
    cos, sin = _angles(s)
    out = {}
    for name in ("q", "k"):
        x, w = s[name].float(), s["w_" + name]
        if w is not None:
            rstd = torch.rsqrt((x * x).mean(dim=2, keepdim=True) + EPS)
        if not c["back"]:
            out[name] = _rotate_plain(c, x if w is None else x * rstd * w, cos, sin).to(dt)
            continue
        dy = _rotate_plain(c, s["d%s_out" % name].float(), cos, -sin)
        if w is not None:
            xhat = x * rstd
            out["dw_" + name] = (dy * xhat).sum(dim=(0, 1))
            u = dy * w
            dy = rstd * (u - xhat * (u * xhat).mean(dim=2, keepdim=True))
        out["d" + name] = dy.to(dt)
    return out


def _experts_plain(s):
    c, dt, n = s["case"], _type(s["case"]), s["n"]
    spans = list(zip(s["offs_h"][:-1], s["offs_h"][1:]))
    if c["what"] == "fwd":
        y = torch.empty(n, c["n_out"], dtype=dt, device="cuda")
        for e, (lo, hi) in enumerate(spans):
            if hi > lo:
                y[lo:hi] = (s["x"][lo:hi].float() @ s["w"][e].float().t()).to(dt)
        return {"y": y}
    dx = torch.empty(n, c["n_in"], dtype=dt, device="cuda")
    dw = torch.zeros(c["E"], c["n_out"], c["n_in"], device="cuda")
    for e, (lo, hi) in enumerate(spans):
        if hi > lo:
            dy = s["dy"][lo:hi].float()
            dx[lo:hi] = (dy @ s["w"][e].float()).to(dt)
            dw[e] = dy.t() @ s["x"][lo:hi].float()
    return {"dx": dx, "dw": dw}


# -------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "embed":
        return {"dtable" if state["case"]["back"] else "x": _embed_plain(state)}
    return _qknorm_plain(state) if kind == "qknorm" else _experts_plain(state)


def _run_own(s):
    from paper_2603_06619_b200 import nat

    c, n = s["case"], s["n"]
    if c["kind"] == "embed":
        if "params" not in s:
            s["params"] = nat.embed_params(c["V"], c["d"], _type(c), scale=c["scale"])
            if c["back"]:
                s["ws"] = nat.alloc_workspace(nat.nat_embed_workspace_bytes(s["params"], s["cap"]), "cuda")
        if c["back"]:
            nat.nat_embed_bwd(s["params"], s["ids"], s["pick"], s["n_rows"], s["cap"], s["dx"], s["dtable"], s["ws"])
            return {"dtable": s["dtable"]}
        nat.nat_embed_fwd(s["params"], s["table"], s["ids"], s["pick"], s["n_rows"], s["cap"], s["x"])
        return {"x": s["x"][:n]}
    if c["kind"] == "qknorm":
        if "params" not in s:
            s["params"] = nat.qknorm_params(c["Hq"], c["Hkv"], c["D"], _type(c), rot_dim=c["R"],
                                            interleaved=c["interleaved"], eps=EPS)
            if c["back"]:
                s["ws"] = nat.alloc_workspace(nat.nat_qknorm_workspace_bytes(s["params"], n), "cuda")
        where = (c["B"], s["cu"], s["positions"], None, n)
        if not c["back"]:
            nat.nat_qknorm_fwd(s["params"], *where, s["q"], s["k"], s["w_q"], s["w_k"], s["inv_freq"], s["q_out"],
                               s["k_out"])
            return {"q": s["q_out"], "k": s["k_out"]}
        nat.nat_qknorm_bwd(s["params"], *where, s["q"], s["k"], s["w_q"], s["w_k"], s["inv_freq"], s["dq_out"],
                           s["dk_out"], s["dq"], s["dk"], s.get("dw_q"), s.get("dw_k"), s["ws"])
        out = {"dq": s["dq"], "dk": s["dk"]}
        if c["norm"]:
            out.update(dw_q=s["dw_q"], dw_k=s["dw_k"])
        return out
    if "params" not in s:
        s["params"] = nat.experts_params(c["E"], c["n_in"], c["n_out"], _type(c))
        s["ws"] = nat.alloc_workspace(nat.nat_experts_workspace_bytes(s["params"], s["cap"]), "cuda")
    if c["what"] == "fwd":
        nat.nat_experts_fwd(s["params"], s["offs"], s["cap"], s["x"], s["w"], s["y"], s["ws"])
        return {"y": s["y"][:n]}
    nat.nat_experts_bwd(s["params"], s["offs"], s["cap"], s["x"], s["w"], s["dy"], s["dx"], s["dw"], s["ws"])
    return {"dx": s["dx"][:n], "dw": s["dw"]}


# ------------------------------------------------------------------- the definitions, in 64 bits
def _exact_embed(s):
    c, n = s["case"], s["n"]
    ids = s["ids"][:n] if s["pick"] is None else torch.index_select(s["ids"], 0, s["pick"][:n])
    if not c["back"]:
        return {"x": torch.index_select(s["table"], 0, ids).double().mul_(c["scale"])}
    # sums of runs of equal ids, column block by column block
    order = ids.long().argsort(stable=True)
    found, count = torch.unique_consecutive(ids[order], return_counts=True)
    end = count.cumsum(0)
    out = torch.zeros(c["V"], c["d"], dtype=torch.float64, device="cuda")
    for a in range(0, c["d"], 512):
        run_sum = s["dx"][:n, a:a + 512][order].double().cumsum(0)
        at_end = run_sum[end - 1]
        out[found.long(), a:a + 512] = c["scale"] * torch.cat([at_end[:1], at_end[1:] - at_end[:-1]])
    return {"dtable": out}


def _exact_qknorm(s):
    c = s["case"]
    turn = torch.einsum("n,r->nr", s["pos"].double(), s["inv_freq"])
    phase = torch.polar(torch.ones_like(turn), turn)[:, None, :]
    R, ans = c["R"], {}

    def turned(x, by):
        pairs = x[..., :R].unflatten(2, (R // 2, 2)) if c["interleaved"] else x[..., :R].unflatten(2, (2, R // 2)).transpose(2, 3)
        z = torch.complex(pairs[..., 0].contiguous(), pairs[..., 1].contiguous()) * by
        z = torch.view_as_real(z)
        z = z.flatten(2) if c["interleaved"] else z.transpose(2, 3).flatten(2)
        return torch.cat([z, x[..., R:]], dim=2)

    for name in ("q", "k"):
        x = s[name].double()
        w = None if s["w_" + name] is None else s["w_" + name].double()
        size = ((x ** 2).sum(dim=2, keepdim=True) / c["D"] + EPS) ** 0.5
        if not c["back"]:
            ans[name] = turned(x if w is None else x / size * w, phase)
            continue
        G = turned(s["d%s_out" % name].double(), phase.conj())
        if w is not None:
            ans["dw_" + name] = torch.einsum("nhd,nhd->d", G, x / size)
            G = (G * w - x * ((G * w * x).sum(dim=2, keepdim=True) / (c["D"] * size ** 2))) / size
        ans["d" + name] = G
    return ans


def _exact_experts(s):
    c, n = s["case"], s["n"]
    wide = {"y": (n, c["n_out"])} if c["what"] == "fwd" else {"dx": (n, c["n_in"]), "dw": (c["E"], c["n_out"], c["n_in"])}
    ans = {k: torch.zeros(*shape, dtype=torch.float64, device="cuda") for k, shape in wide.items()}
    for e in range(c["E"]):
        rows = slice(s["offs_h"][e], s["offs_h"][e + 1])
        X, W = s["x"][rows].double(), s["w"][e].double()
        if c["what"] == "fwd":
            ans["y"][rows] = torch.einsum("ri,oi->ro", X, W)
        else:
            G = s["dy"][rows].double()
            ans["dx"][rows] = torch.einsum("ro,oi->ri", G, W)
            ans["dw"][e] = torch.einsum("ro,ri->oi", G, X)
    return ans


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "embed":
        return _exact_embed(s)
    return _exact_qknorm(s) if c["kind"] == "qknorm" else _exact_experts(s)
