"""The 4-bit projections and the block residual: what is timed, their plain forms and their 64-bit results.

A program that serves a model with 4-bit weights quantises each weight once when the model is loaded
(``fold``) and then calls the projections (``linear``, ``glu``, ``down``): one row per running
sequence while it decodes, tens to hundreds of rows when it batches or cuts prompts into chunks,
thousands in a prefill.  Between two projections the block's output joins the residual stream
(``residual``: post-norm, gate, scales, the next norm), and in training its gradients come back
(``residual_bwd``).  ``listed()`` gives the cases, ``draw()`` more of the same ranges, ``prepare()``
what the program holds before a call; ``run()`` is the call, in its plain form or through the library.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
W4_KINDS = ("linear", "glu", "down")


def listed():
    return [
        # One sequence decoding: the QKV projection of a grouped-query layer (32 + 8 + 8 heads of 128), weights folded.
        {"name": "w4_decode_linear_m1", "kind": "linear", "M": 1, "K": 4096, "N": 6144, "G": 128, "zeros": False, "g": False},
        # A ragged chunk of a prompt through the Llama-7B QKV projection, with a checkpoint's own codes: zero points, g at run time.
        {"name": "w4_chunk_linear_m333", "kind": "linear", "M": 333, "K": 4096, "N": 12288, "G": 64, "zeros": True, "g": True},
        # Sixteen sequences decoding: the FFN input projection of a Llama-7B layer, the largest weight stream of a token.
        {"name": "w4_decode_glu_m16", "kind": "glu", "M": 16, "K": 4096, "N": 11008, "G": 128, "zeros": True, "g": False},
        # A prefill's FFN input projection, the largest share of its arithmetic.
        {"name": "w4_prefill_glu_m2048", "kind": "glu", "M": 2048, "K": 4096, "N": 11008, "G": 128, "zeros": False, "g": False},
        # A few sequences decoding: the FFN down projection, a long K into a narrow output, small groups.
        {"name": "w4_decode_down_m5", "kind": "down", "M": 5, "K": 11008, "N": 4096, "G": 32, "zeros": False, "row_scale": False},
        # Batched serving: 64 sequences through the down projection, the scale deferred from the norm applied here.
        {"name": "w4_batch_down_m64", "kind": "down", "M": 64, "K": 11008, "N": 4096, "G": 128, "zeros": True, "row_scale": True},
        # Loading a small fp32 model (SmolLM2-135M width): one projection, read back for a check.
        {"name": "w4_load_fold_small", "kind": "fold", "dtype": "f32", "K": 576, "N": 1536, "G": 32, "zeros": False, "transposed": False, "glu": False},
        # Loading a large model: the [N, K] gate and up weights of an FFN.
        {"name": "w4_load_fold_glu", "kind": "fold", "dtype": "bf16", "K": 4096, "N": 22016, "G": 128, "zeros": True, "transposed": True, "glu": True},
        # One token: the smallest call, where latency counts.  The next projection takes its norm itself.
        {"name": "residual_token", "kind": "residual", "dtype": "bf16", "M": 1, "K": 4096, "post": True, "gate_rows": 0, "pre": False},
        # A prefill of eight sequences with a gate per sequence, norms on both sides.
        {"name": "residual_prefill_gated", "kind": "residual", "dtype": "bf16", "M": 4096, "K": 4096, "post": True, "gate_rows": 512, "pre": True},
        # Training a small model in fp32: no gate, an odd row count.
        {"name": "residual_bwd_fp32", "kind": "residual_bwd", "dtype": "f32", "M": 1999, "K": 576, "post": True, "gate_rows": 0, "pre": True},
        # Training a large model: norms on both sides and a gate per sequence of 512 tokens.
        {"name": "residual_bwd_gated", "kind": "residual_bwd", "dtype": "bf16", "M": 4096, "K": 4096, "post": True, "gate_rows": 512, "pre": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _depth(rng, lo, hi, unit):
    """A K of the range: mostly a multiple of 128, else of the unit that the dtype needs."""
    u = 128 if rng.random() < 0.6 else unit
    return max(unit, _log(rng, lo, hi) // u * u)


def draw(rng):
    kind = rng.choice(W4_KINDS + W4_KINDS + ("fold", "residual", "residual", "residual_bwd", "residual_bwd"))
    G = rng.choice((32, 64, 128))
    if kind in W4_KINDS:
        M = rng.choice((lambda: _log(rng, 1, 16), lambda: _log(rng, 17, 256), lambda: _log(rng, 257, 2048)))()
        K = _depth(rng, 256, 11008, 8)
        N = _log(rng, 256, min(22016, 9e7 / K))
        if rng.random() < 0.5:
            N = max(64, N // 64 * 64)
        c = {"kind": kind, "M": M, "K": K, "N": N // 2 if kind == "glu" else N, "G": G, "zeros": rng.random() < 0.5}
        c["row_scale" if kind == "down" else "g"] = rng.random() < 0.4
        return c
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind == "fold":
        K = _depth(rng, 256, 8192, 8)
        return {"kind": kind, "dtype": dtype, "K": K, "N": 2 * (_log(rng, 256, min(12288, 4e7 / K)) // 2), "G": G,
                "zeros": rng.random() < 0.5, "transposed": rng.random() < 0.7, "glu": rng.random() < 0.4}
    K = _depth(rng, 128, 16384, 8)
    M = _log(rng, 1, min(4096, 1.6e7 / K))
    return {"kind": kind, "dtype": dtype, "M": M, "K": K, "post": rng.random() < 0.7,
            "gate_rows": rng.choice((0, 1, _log(rng, 1, M), M)), "pre": kind == "residual_bwd" or rng.random() < 0.7}


def _width(c):
    """Columns of the logical weight."""
    return 2 * c["N"] if c["kind"] == "glu" else c["N"]


def _inputs(c, seed):
    """Seeded inputs: activations with 1% outlier rows, weights of variance 1/K, norm weights around 1."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)

    def around_one(*shape):
        return torch.rand(*shape, generator=gen, device="cuda") + 0.5

    def rows(M, K, dt):
        a = normal(M, K)
        a[torch.randperm(M, generator=gen, device="cuda")[: M // 100]] *= 20.0
        return a.to(dt)

    K, x = c["K"], {}
    if c["kind"] in W4_KINDS:
        N, groups = _width(c), -(-K // c["G"])
        x["a"] = rows(c["M"], K, torch.bfloat16)
        # Codes as a quantised Gaussian weight has them (a spread of 2.6 steps), scales of about 1 / (2.6 sqrt K).
        x["codes"] = (normal(K, N) * 2.6 + 8.0).round_().clamp_(0, 15).to(torch.uint8)
        x["scales"] = (around_one(groups, N) * (K ** -0.5 / 2.6)).to(torch.bfloat16).float()
        if c["zeros"]:
            x["zeros"] = torch.randint(5, 12, (groups, N), generator=gen, device="cuda", dtype=torch.uint8)
        if c.get("g"):
            x["g"] = around_one(K)
        if c.get("row_scale"):
            x["row_scale"] = around_one(c["M"])
        return x
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    if c["kind"] == "fold":
        W = normal(c["N"], K) if c["transposed"] else normal(K, c["N"])
        W = (W * K ** -0.5).to(dt)
        return {"W": W.t() if c["transposed"] else W, "g": around_one(K)}
    M = c["M"]
    x["x"], x["h"] = rows(M, K, dt), rows(M, K, dt)
    if c["post"]:
        x["g_post"] = around_one(K)
    if c["gate_rows"]:
        x["gate"] = normal(-(-M // c["gate_rows"]), K).to(dt)
    if c["pre"]:
        x["g_pre"] = around_one(K)
    if c["kind"] == "residual_bwd":
        x["dh_out"], x["dn"] = normal(M, K).to(dt), normal(M, K).to(dt)
    return x


# The residual stream is kept as it is and the block's output joins it scaled, as in deep models.
RES_SCALE, BRANCH_SCALE = 1.0, 0.5


def prepare(case, seed):
    x = _inputs(case, seed)
    if own and case["kind"] in W4_KINDS:
        from paper_2407_09577_amd import flashnorm as fn
        layout = fn.FN_LAYOUT_GLU if case["kind"] == "glu" else fn.FN_LAYOUT_LINEAR
        x["w4"] = fn.pack_weights_w4(x.pop("codes"), x.pop("scales"), x.pop("zeros", None), layout=layout, group=case["G"])
    return case, x


def run(state):
    c, x = state
    return _run_own(c, x) if own else _run_plain(c, x)


def _run_own(c, x):
    from paper_2407_09577_amd import flashnorm as fn
    kind = c["kind"]
    if kind == "linear":
        return fn.flashnorm_linear_w4(x["a"], x["w4"], EPS, g=x.get("g"))
    if kind == "glu":
        return fn.flashnorm_glu_w4(x["a"], x["w4"], EPS, g=x.get("g"))
    if kind == "down":
        return fn.rowscale_linear_w4(x["a"], x["w4"], row_scale=x.get("row_scale"))
    if kind == "fold":
        layout = fn.FN_LAYOUT_GLU if c["glu"] else fn.FN_LAYOUT_LINEAR
        w4 = fn.fold_weights_w4(x["W"], x["g"], layout=layout, group=c["G"], zero_points=c["zeros"])
        return fn.unpack_weights_w4(w4)
    common = dict(g_post=x.get("g_post"), eps_post=EPS, gate=x.get("gate"), rows_per_gate=c["gate_rows"] or 1,
                  res_scale=RES_SCALE, branch_scale=BRANCH_SCALE, g_pre=x.get("g_pre"), eps_pre=EPS)
    if kind == "residual":
        out, normed = fn.flashnorm_block_residual(x["x"], x["h"], **common)
        return {"out": out, "normed": normed} if c["pre"] else {"out": out}
    grads = fn.flashnorm_block_residual_bwd(x["x"], x["h"], x["dh_out"], x["dn"], **common)
    return _named(c, *grads)


def _named(c, dx, dh, dgate, dg_post, dg_pre):
    out = {"dx": dx, "dh": dh}
    if c["gate_rows"]:
        out["dgate"] = dgate
    if c["post"]:
        out["dg_post"] = dg_post
    if c["pre"]:
        out["dg_pre"] = dg_pre
    return out


def _run_plain(c, x):
    kind = c["kind"]
    if kind == "fold":
        return _fold_plain(c, x)
    if kind not in W4_KINDS:
        return _residual_plain(c, x)
    at = torch.arange(c["K"], device="cuda") // c["G"]  # the group of each input
    zeros = x["zeros"].float() if c["zeros"] else 8.0
    W = (x["codes"].float() - (zeros[at] if c["zeros"] else zeros)) * x["scales"][at]
    a = x["a"].float()
    t = (a * x["g"] if c.get("g") else a) @ W
    if kind == "down":
        return (t * x["row_scale"][:, None] if c["row_scale"] else t).to(torch.bfloat16)
    t = t * torch.rsqrt((a * a).mean(1, keepdim=True) + EPS)
    if kind == "glu":
        gate, up = t[:, : c["N"]], t[:, c["N"]:]
        t = gate / (1.0 + torch.exp(-gate)) * up
    return t.to(torch.bfloat16)


def _twelve_bits(s):
    """fp64 rounded to 12 significant bits, ties to even."""
    bits = s.view(torch.int64)
    return ((bits + ((1 << 40) - 1) + ((bits >> 41) & 1)) & -(1 << 41)).view(torch.float64)


def _fold_plain(c, x):
    # In 64 bits: a weight next to the border of two codes goes to the right one.
    W = x["W"].double() * x["g"].double()[:, None]
    out = torch.empty(c["K"], c["N"], dtype=torch.float32, device="cuda")
    for k in range(0, c["K"], c["G"]):
        w = W[k:k + c["G"]]
        if c["zeros"]:
            lo, hi = w.amin(0).clamp(max=0.0), w.amax(0).clamp(min=0.0)
            s = _twelve_bits((hi - lo) / 15.0)
            z = torch.where(s > 0, torch.round(-lo / s).clamp(0, 15), 8.0)
        else:
            s, z = _twelve_bits(w.abs().amax(0) / 7.0), torch.full_like(w[0], 8.0)
        q = torch.where(s > 0, (torch.round(w / s) + z).clamp(0, 15), z)
        out[k:k + c["G"]] = ((q - z) * s).float()
    return out


def _residual_plain(c, x):
    xf, hf = x["x"].float(), x["h"].float()
    M, K = xf.shape
    T = c["gate_rows"]
    gate = x["gate"].float().repeat_interleave(T, 0)[:M] if T else 1.0
    p = torch.rsqrt((xf * xf).mean(1, keepdim=True) + EPS) if c["post"] else 1.0
    z = xf * p * x["g_post"] if c["post"] else xf
    H = RES_SCALE * hf + BRANCH_SCALE * gate * z
    r = torch.rsqrt((H * H).mean(1, keepdim=True) + EPS) if c["pre"] else None
    if c["kind"] == "residual":
        out = {"out": H.to(x["x"].dtype)}
        if c["pre"]:
            out["normed"] = (H * r * x["g_pre"]).to(x["x"].dtype)
        return out
    D, dn = x["dh_out"].float(), x["dn"].float()
    u = dn * x["g_pre"]
    D = D + u * r - H * (r * r * r * ((u * H).sum(1, keepdim=True) / K))
    dg_pre = (dn * H * r).sum(0)
    dz = BRANCH_SCALE * gate * D
    dgate = dg_post = None
    if T:
        B = x["gate"].shape[0]
        part = torch.zeros(B * T, K, device="cuda")
        part[:M] = BRANCH_SCALE * D * z
        dgate = part.view(B, T, K).sum(1).to(x["x"].dtype)
    dx = dz
    if c["post"]:
        dg_post = (dz * xf * p).sum(0)
        v = dz * x["g_post"]
        dx = v * p - xf * (p * p * p * ((v * xf).sum(1, keepdim=True) / K))
    return _named(c, dx.to(x["x"].dtype), (RES_SCALE * D).to(x["x"].dtype), dgate, dg_post, dg_pre)


def work(case):
    K, kind = case["K"], case["kind"]
    if kind in W4_KINDS:
        M, N = case["M"], _width(case)
        groups = -(-K // case["G"])
        weights = K * N // 2 + groups * N * (2 + (0.5 if case["zeros"] else 0))
        return {"bytes": weights + 2 * M * K + 2 * M * case["N"], "flops": 2.0 * M * K * N}
    size = 2 if case["dtype"] == "bf16" else 4
    if kind == "fold":
        N = case["N"]
        return {"bytes": K * N * (size + 0.5 + 0.5 + 4) + 4 * K, "flops": 6.0 * K * N}
    M = case["M"]
    gates = -(-M // case["gate_rows"]) if case["gate_rows"] else 0
    vectors = 4 * K * (case["post"] + case["pre"])
    if kind == "residual":
        return {"bytes": size * K * (M * (3 + case["pre"]) + gates) + vectors, "flops": 10.0 * M * K}
    return {"bytes": size * K * (6 * M + 2 * gates) + 2 * vectors, "flops": 30.0 * M * K}


def exact(case, seed):
    x = _inputs(case, seed)
    if case["kind"] in W4_KINDS:
        return _exact_w4(case, x)
    if case["kind"] == "fold":
        return _exact_fold(case, x)
    return _exact_residual(case, x)


def _exact_w4(c, x):
    K, G = c["K"], c["G"]
    steps = x["codes"].double()
    steps -= x["zeros"].double().repeat_interleave(G, 0)[:K] if c["zeros"] else 8.0
    steps *= x["scales"].double().repeat_interleave(G, 0)[:K]
    a = x["a"].double()
    if c.get("g"):
        steps *= x["g"].double()[:, None]
    y = torch.mm(a, steps)
    if c["kind"] == "down":
        return torch.diag(x["row_scale"].double()) @ y if c["row_scale"] else y
    y /= (EPS + a.pow(2).sum(1, keepdim=True) / K).sqrt()
    if c["kind"] == "linear":
        return y
    gate, up = y.chunk(2, dim=1)
    return gate * torch.sigmoid(gate) * up


def _exact_fold(c, x):
    K, G, N = c["K"], c["G"], c["N"]
    groups = -(-K // G)
    w = torch.zeros(groups * G, N, dtype=torch.float64, device="cuda")
    w[:K] = x["g"].double()[:, None] * x["W"].double()
    w = w.view(groups, G, N)  # the padding's zeros change no largest or smallest value used below
    if c["zeros"]:
        low, high = torch.minimum(w.amin(1), w.new_zeros(())), torch.maximum(w.amax(1), w.new_zeros(()))
        span = (high - low) / 15
    else:
        span = w.abs().amax(1) / 7
    m, e = torch.frexp(span)
    s = torch.ldexp(torch.round(m * 4096), e - 12)
    safe = torch.where(s == 0, 1.0, s)
    z = torch.round(-low / safe).clamp(0, 15) if c["zeros"] else torch.full_like(s, 8.0)
    steps = (torch.round(w / safe[:, None]) + z[:, None]).clamp(0, 15) - z[:, None]
    return (steps * s[:, None]).reshape(groups * G, N)[:K]


def _exact_residual(c, x):
    names = [n for n in ("x", "h", "gate", "g_post", "g_pre") if n in x]
    v = {n: x[n].double() for n in names}
    backward = c["kind"] == "residual_bwd"
    if backward:
        for t in v.values():
            t.requires_grad_(True)
    M, K = v["x"].shape

    def normed(t, g):
        return t / (t.pow(2).sum(1, keepdim=True) / K + EPS).sqrt() * g

    branch = normed(v["x"], v["g_post"]) if c["post"] else v["x"]
    if c["gate_rows"]:
        branch = branch * v["gate"][torch.arange(M, device="cuda") // c["gate_rows"]]
    out = RES_SCALE * v["h"] + BRANCH_SCALE * branch
    n = normed(out, v["g_pre"]) if c["pre"] else None
    if not backward:
        return {"out": out, "normed": n} if c["pre"] else {"out": out}
    total = (out * x["dh_out"].double()).sum() + (n * x["dn"].double()).sum()
    grads = dict(zip(names, torch.autograd.grad(total, [v[k] for k in names])))
    return _named(c, grads["x"], grads["h"], grads.get("gate"), grads.get("g_post"), grads.get("g_pre"))
