"""Cases, plain forms and 64-bit definitions of the operators of a gated recurrent block.

Three operators that are used together around the mixing kernels:

* scan: the gated linear recurrence h_t = a_t h_{t-1} + i_t with a_t = sigma(g_t) and
  i_t = (1 - a_t) x_t ("leak") or i_t = x_t; over a sequence, as one training pass
  (forward and gradients) and as one decode step;
* linear: y = act(x w^T + bias) + residual, forward and gradients;
* adamw: one AdamW step over many tensors, its moments in 32 bits or in 8 bits.

With ``own`` false, ``run`` computes a case with elementary torch operations in 32 bits,
rounded once to the output's type; with ``own`` true it makes the library's calls.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
BLOCK = 256          # values that share one scale of the 8-bit moments
BETA1, BETA2, EPS, LR, WD = 0.9, 0.95, 1e-8, 3e-4, 0.1


def _lib():
    import paper_2607_05583_gb300 as rlm
    return rlm


# ------------------------------------------------------------------- cases
def listed():
    return [
        # One token for each of 8 sequences of the 6M-parameter model's width: a serving step, launch latency.
        {"name": "scan_decode_b8", "op": "scan_decode", "B": 8, "D": 256, "dtype": "bf16", "leak": True},
        # The library's headline field: four long prompts, no gradients.
        {"name": "scan_prefill_b4_32k", "op": "scan_prefill", "B": 4, "L": 32768, "D": 256, "dtype": "bf16",
         "leak": True, "ragged": False, "fused": True},
        # A padded batch in fp32: odd length, odd width, rows of any length down to none, an initial state.
        {"name": "scan_prefill_ragged", "op": "scan_prefill", "B": 9, "L": 2047, "D": 520, "dtype": "f32",
         "leak": False, "ragged": True, "fused": False},
        # One layer's recurrence of the training shape, forward and gradients.
        {"name": "scan_train_b4_32k", "op": "scan_train", "B": 4, "L": 32768, "D": 512, "dtype": "bf16",
         "leak": True, "ragged": False, "fused": True},
        # The same in fp32 on a padded batch of odd sizes.
        {"name": "scan_train_ragged", "op": "scan_train", "B": 5, "L": 4099, "D": 328, "dtype": "f32",
         "leak": False, "ragged": True, "fused": False},
        # One token for each of 8 sequences through a projection: the weights' bytes.
        {"name": "linear_tokens_8", "op": "linear", "R": 8, "K": 2048, "N": 4096, "act": "silu", "bias": True,
         "residual": False},
        # The input projection of the 6M-parameter model over the headline's 131072 tokens: the fields' bytes.
        {"name": "linear_narrow_131k", "op": "linear", "R": 131072, "K": 256, "N": 512, "act": "none", "bias": True,
         "residual": False},
        # A wide feed-forward product: the tensor cores' rate.
        {"name": "linear_wide", "op": "linear", "R": 8192, "K": 4096, "N": 8192, "act": "gelu", "bias": True,
         "residual": True},
        # Gradients of a gated projection over an odd number of tokens.
        {"name": "linear_backward_odd", "op": "linear_backward", "R": 16387, "K": 1024, "N": 2048, "act": "silu",
         "bias": True},
        # Every tensor of the 6M-parameter model (6 layers of resonators, projections, norms), fp32 throughout.
        {"name": "adamw_small", "op": "adamw", "tensors": 66, "total": 6000000, "param": "f32", "grad": "f32",
         "master": False, "bits": 32},
        # bf16 weights and gradients with fp32 masters and moments.
        {"name": "adamw_master", "op": "adamw", "tensors": 150, "total": 120000000, "param": "bf16", "grad": "bf16",
         "master": True, "bits": 32},
        # The same weights with moments in 8 bits and no masters.
        {"name": "adamw_8bit", "op": "adamw", "tensors": 150, "total": 120000000, "param": "bf16", "grad": "bf16",
         "master": False, "bits": 8},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["scan_decode", "scan_prefill", "scan_prefill", "scan_train", "linear", "linear",
                     "linear_backward", "adamw"])
    if op == "scan_decode":
        return {"op": op, "B": _log(rng, 1, 1024), "D": 8 * _log(rng, 1, 512), "dtype": rng.choice(["bf16", "f32"]),
                "leak": rng.random() < 0.5}
    if op in ("scan_prefill", "scan_train"):
        most = 1 << 25 if op == "scan_prefill" else 1 << 26
        while True:
            B, L, D = _log(rng, 1, 64), _log(rng, 1, 65536), 8 * _log(rng, 1, 256)
            if B * L * D <= most:
                break
        return {"op": op, "B": B, "L": L, "D": D, "dtype": rng.choice(["bf16", "f32"]), "leak": rng.random() < 0.5,
                "ragged": rng.random() < 0.5, "fused": rng.random() < 0.5}
    if op in ("linear", "linear_backward"):
        most = 2.7e11 if op == "linear" else 1.3e11
        while True:
            R, K, N = _log(rng, 1, 131072), 8 * _log(rng, 2, 1024), 8 * _log(rng, 2, 1024)
            if R * K * N <= most and R * (K + N) <= 1 << 27:
                break
        case = {"op": op, "R": R, "K": K, "N": N, "act": rng.choice(["none", "silu", "gelu", "sigmoid"]),
                "bias": rng.random() < 0.5}
        if op == "linear":
            case["residual"] = rng.random() < 0.5
        return case
    param = rng.choice(["bf16", "f32"])
    tensors = _log(rng, 1, 400)
    return {"op": op, "tensors": tensors, "total": max(_log(rng, 1000, 120000000), 2 * tensors), "param": param,
            "grad": rng.choice(["bf16", "f32"]), "master": param == "bf16" and rng.random() < 0.5,
            "bits": rng.choice([8, 32])}


# ------------------------------------------------------------------ inputs
def _sizes(case):
    """Element counts of an optimizer's tensors: spread over a factor of 1000 as weights and norms are, odd ones
    among them."""
    n = case["tensors"]
    w = [1000.0 ** (((7 * i + 3) % n) / max(n - 1, 1)) for i in range(n)]
    s = sum(w)
    return [max(1, int(case["total"] * x / s)) for x in w]


def _lengths(case, gen):
    """Token counts of a padded batch: any from none to all, one row empty and one full where there are two."""
    n = torch.randint(0, case["L"] + 1, (case["B"],), generator=gen, device="cuda", dtype=torch.int32)
    n[0] = case["L"]
    if case["B"] > 1:
        n[1] = 0
    return n


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    op = case["op"]
    st = {"case": case}
    if op.startswith("scan"):
        dt, B, D = DT[case["dtype"]], case["B"], case["D"]
        L = case.get("L", 1)
        # Gates as a trained block has them: decays from about 0.3 to 0.999.
        if case.get("fused"):       # the two halves of one projection's output
            f = randn(B, L, 2 * D).to(dt)
            f[..., D:] = (2.5 + 1.5 * f[..., D:].float()).to(dt)
            x, g = f[..., :D], f[..., D:]
        else:
            x, g = randn(B, L, D).to(dt), (2.5 + 1.5 * randn(B, L, D)).to(dt)
        if op == "scan_decode":
            return dict(st, x=x[:, 0].contiguous(), g=g[:, 0].contiguous(), h=randn(B, D),
                        y=torch.empty(B, D, dtype=dt, device="cuda"))
        st.update(x=x, g=g, h0=randn(B, D), lengths=_lengths(case, gen) if case["ragged"] else None)
        if case["ragged"]:          # what padding holds is never to be used
            past = (torch.arange(L, device="cuda")[None, :] >= st["lengths"][:, None])[..., None]
            x.masked_fill_(past, float("nan"))
            g.masked_fill_(past, float("nan"))
        if op == "scan_train":
            st.update(dy=randn(B, L, D).to(dt), dh=randn(B, D))
        return st
    if op.startswith("linear"):
        R, K, N = case["R"], case["K"], case["N"]
        st["x"] = randn(R, K).bfloat16()
        st["w"] = (randn(N, K) * K ** -0.5).bfloat16()
        st["bias"] = 0.5 * randn(N) if case["bias"] else None
        if op == "linear":
            st["residual"] = randn(R, N).bfloat16() if case["residual"] else None
        else:
            st["pre"] = randn(R, N).bfloat16() if case["act"] != "none" else None   # kept by the forward pass
            st["dy"] = randn(R, N).bfloat16()
        return st
    # Optimizer: tensors laid out one after another, each at a multiple of 256 values.
    sizes = _sizes(case)
    offs, at = [], 0
    for n in sizes:
        offs.append(at)
        at += -(-n // BLOCK) * BLOCK
    real = torch.zeros(at, dtype=torch.bool, device="cuda")
    for o, n in zip(offs, sizes):
        real[o:o + n] = True
    cut = lambda t: [t[o:o + n] for o, n in zip(offs, sizes)]  # noqa: E731
    full = torch.where(real, 0.02 * randn(at), 0.0)
    st["param"] = full.to(DT[case["param"]])
    st["master"] = full if case["master"] else None
    # Gradients and moments as in mid-training: scales that vary from block to block.
    scale = torch.exp(2.0 * randn(at // BLOCK, 1)).mul_(1e-3)
    st["grad"] = torch.where(real, (randn(at // BLOCK, BLOCK) * scale).reshape(-1), 0.0).to(DT[case["grad"]])
    m = torch.where(real, (0.3 * randn(at // BLOCK, BLOCK) * scale).reshape(-1), 0.0)
    v = torch.where(real, ((0.1 + randn(at // BLOCK, BLOCK).square()) * scale * scale).reshape(-1), 0.0)
    if case["bits"] == 8:
        st["m"], st["m_scale"] = _quantise(m, False)
        st["v"], st["v_scale"] = _quantise(v.sqrt(), True)
    else:
        st["m"], st["v"] = m, v
    del m, v, full
    st["step"] = 1000
    st["lists"] = {k: cut(st[k]) for k in ("param", "grad", "m", "v")}
    st["lists"]["master"] = cut(st["master"]) if case["master"] else None
    if case["bits"] == 8:
        st["lists"]["scales"] = [(st["m_scale"][o // BLOCK:-(-(o + n) // BLOCK)], st["v_scale"][o // BLOCK:-(-(o + n) // BLOCK)])
                                 for o, n in zip(offs, sizes)]
    if own:                         # the handle a training program builds once over its tensors
        rlm, ls = _lib(), st["lists"]
        sc = ls.get("scales") or [(None, None)] * len(sizes)
        states = [rlm.AdamState(a, b, c, d) for a, b, (c, d) in zip(ls["m"], ls["v"], sc)]
        st["group"] = rlm.AdamGroup(ls["param"], ls["grad"], states, ls["master"])
    return st


def _quantise(x, up):
    """8-bit floats (4 exponent and 3 mantissa bits) of blocks of BLOCK values with a power-of-two scale 2^(e-8),
    2^e the first power of two above the block's largest magnitude; ``up``: what is above zero stays above zero."""
    b = x.reshape(-1, BLOCK)
    top = b.abs().amax(1)
    e = torch.where(top > 0, torch.frexp(top)[1], -100).clamp_(min=-100)
    power = lambda k: ((k + 127) << 23).to(torch.int32).view(torch.float32)  # noqa: E731
    c = b * power(8 - e)[:, None]
    if up:
        c = torch.where(c > 0, c.clamp(min=2.0 ** -9), c)
    return c.to(torch.float8_e4m3fn).reshape(-1), power(e - 8)


# ------------------------------------------------------------- plain forms
def _doubling_scan(a, u):
    """Inclusive scan of h_t = a_t h_{t-1} + u_t along dimension 1, in place, by doubling."""
    n = 1
    while n < a.shape[1]:
        u[:, n:] += a[:, n:] * u[:, :-n]
        a[:, n:] = a[:, n:] * a[:, :-n]
        n *= 2
    return u


def _gate(g):
    return 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))


def _valid(st):
    if st["lengths"] is None:
        return None
    return (torch.arange(st["x"].shape[1], device="cuda")[None, :] < st["lengths"][:, None])[..., None]


def _plain_scan(st):
    leak, ok = st["case"]["leak"], _valid(st)
    x = st["x"].float()
    a, b = _gate(st["g"].float())
    u = b * x if leak else x.clone()
    if ok is not None:
        a, u = torch.where(ok, a, 1.0), torch.where(ok, u, 0.0)
    u[:, 0] += a[:, 0] * st["h0"]
    h = _doubling_scan(a.clone(), u)
    return h, a, b, x, ok


def _plain_scan_prefill(st):
    h, _, _, _, ok = _plain_scan(st)
    y = h if ok is None else torch.where(ok, h, 0.0)
    return {"y": y.to(st["x"].dtype), "state": h[:, -1].clone()}


def _plain_scan_train(st):
    leak, dt = st["case"]["leak"], st["x"].dtype
    h, a, b, x, ok = _plain_scan(st)
    dy = st["dy"].float()
    if ok is not None:
        dy = torch.where(ok, dy, 0.0)
    # G_t = dy_t + a_{t+1} G_{t+1}: the same scan with time reversed.
    d = dy.flip(1)
    d[:, 0] += st["dh"]
    r = torch.cat([torch.ones_like(a[:, :1]), a[:, 1:].flip(1)], 1)
    G = _doubling_scan(r, d).flip(1)
    prev = torch.cat([st["h0"][:, None], h[:, :-1]], 1)
    out = {"state": h[:, -1].clone(), "dh0": a[:, 0] * G[:, 0]}
    y, dx, dg = h, G * b if leak else G, G * (prev - x if leak else prev) * a * b
    if ok is not None:
        y, dx, dg = (torch.where(ok, t, 0.0) for t in (y, dx, dg))
    return dict(out, y=y.to(dt), dx=dx.to(dt), dg=dg.to(dt))


def _plain_scan_decode(st):
    a, b = _gate(st["g"].float())
    x = st["x"].float()
    st["h"] = a * st["h"] + (b * x if st["case"]["leak"] else x)
    return {"y": st["h"].to(st["x"].dtype), "state": st["h"]}


def _act(z, name):
    if name == "none":
        return z
    s = 1 / (1 + torch.exp(-(_bend(z) if name == "gelu" else z)))
    return s if name == "sigmoid" else z * s


def _bend(z):
    """gelu(z) = z sigma(2 sqrt(2 / pi) (z + 0.044715 z^3))."""
    return 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)


def _act_grad(z, name):
    s = 1 / (1 + torch.exp(-(_bend(z) if name == "gelu" else z)))
    if name == "sigmoid":
        return s * (1 - s)
    bend = 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z) if name == "gelu" else 1.0
    return s + z * s * (1 - s) * bend


def _plain_linear(st):
    z = st["x"].float() @ st["w"].float().t()
    if st["bias"] is not None:
        z = z + st["bias"]
    z = _act(z, st["case"]["act"])
    if st["residual"] is not None:
        z = z + st["residual"].float()
    return {"y": z.bfloat16()}


def _plain_linear_backward(st):
    d = st["dy"].float()
    if st["pre"] is not None:
        d = d * _act_grad(st["pre"].float(), st["case"]["act"])
    out = {"dx": (d @ st["w"].float()).bfloat16(), "dw": (d.t() @ st["x"].float()).bfloat16()}
    if st["bias"] is not None:
        out["dbias"] = d.sum(0)
    return out


def _adamw_outputs(st):
    out = {k: st[k] for k in ("param", "m", "v")}
    for k in ("master", "m_scale", "v_scale"):
        if st.get(k) is not None:
            out[k] = st[k]
    return out


def _plain_adamw(st):
    # Over the flat buffers that the tensors lie in: what no tensor holds between them is zero and stays zero.
    st["step"] += 1
    bc1, bc2 = 1 - BETA1 ** st["step"], 1 - BETA2 ** st["step"]
    g = st["grad"].float()
    if st["case"]["bits"] == 8:
        m = (st["m"].float().reshape(-1, BLOCK) * st["m_scale"][:, None]).reshape(-1)
        r = (st["v"].float().reshape(-1, BLOCK) * st["v_scale"][:, None]).reshape(-1)
        v = r * r
    else:
        m, v = st["m"], st["v"]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * (g * g)
    p = st["master"] if st["master"] is not None else st["param"].float()
    p = p * (1 - LR * WD) - (LR / bc1) * (m / (v.sqrt() * (1 / math.sqrt(bc2)) + EPS))
    if st["case"]["bits"] == 8:
        for k, val, up in (("m", m, False), ("v", v.sqrt(), True)):
            code, scale = _quantise(val, up)
            st[k].copy_(code)
            st[k + "_scale"].copy_(scale)
    else:
        st["m"].copy_(m)
        st["v"].copy_(v)
    if st["master"] is not None:
        st["master"].copy_(p)
    st["param"].copy_(p)
    return _adamw_outputs(st)


PLAIN = {"scan_prefill": _plain_scan_prefill, "scan_train": _plain_scan_train, "scan_decode": _plain_scan_decode,
         "linear": _plain_linear, "linear_backward": _plain_linear_backward, "adamw": _plain_adamw}


# ---------------------------------------------------------- library's calls
def _own_scan_prefill(st):
    rlm, x, leak = _lib(), st["x"], st["case"]["leak"]
    y = torch.empty(x.shape, dtype=x.dtype, device="cuda")
    state = torch.empty_like(st["h0"])
    rlm.rlm_scan_prefill(x, st["g"], y, leak=leak, state_in=st["h0"], state_out=state, lengths=st["lengths"])
    return {"y": y, "state": state}


def _own_scan_train(st):
    rlm, x, leak = _lib(), st["x"], st["case"]["leak"]
    y, dx, dg = (torch.empty(x.shape, dtype=x.dtype, device="cuda") for _ in range(3))
    state, dh0 = torch.empty_like(st["h0"]), torch.empty_like(st["h0"])
    saved = rlm.scan_saved(*x.shape, device="cuda")
    rlm.rlm_scan_prefill(x, st["g"], y, leak=leak, state_in=st["h0"], state_out=state, saved=saved,
                         lengths=st["lengths"])
    rlm.rlm_scan_backward(st["dy"], x, st["g"], saved, dx, dg, leak=leak, d_state_out=st["dh"], d_state_in=dh0,
                          lengths=st["lengths"])
    return {"state": state, "dh0": dh0, "y": y, "dx": dx, "dg": dg}


def _own_scan_decode(st):
    _lib().rlm_scan_decode(st["x"], st["g"], st["h"], st["y"], leak=st["case"]["leak"])
    return {"y": st["y"], "state": st["h"]}


def _own_linear(st):
    y = torch.empty(st["x"].shape[0], st["w"].shape[0], dtype=torch.bfloat16, device="cuda")
    _lib().rlm_linear(st["x"], st["w"], y, bias=st["bias"], residual=st["residual"], act=st["case"]["act"])
    return {"y": y}


def _own_linear_backward(st):
    out = {"dx": torch.empty_like(st["x"]), "dw": torch.empty_like(st["w"])}
    if st["bias"] is not None:
        out["dbias"] = torch.empty_like(st["bias"])
    _lib().rlm_linear_backward(st["dy"], st["x"], st["w"], dx=out["dx"], dw=out["dw"], dbias=out.get("dbias"),
                               act=st["case"]["act"], pre=st["pre"])
    return out


def _own_adamw(st):
    st["step"] += 1
    _lib().rlm_adamw_step(st["group"], st["step"], LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=WD)
    return _adamw_outputs(st)


OWN = {"scan_prefill": _own_scan_prefill, "scan_train": _own_scan_train, "scan_decode": _own_scan_decode,
       "linear": _own_linear, "linear_backward": _own_linear_backward, "adamw": _own_adamw}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# -------------------------------------------------------------------- work
def work(case):
    """Bytes: every input once, every output once.  Operations: of the recurrences and of the products."""
    op = case["op"]
    if op.startswith("scan"):
        s, n = BYTES[case["dtype"]], case["B"] * case.get("L", 1) * case["D"]
        state = 4 * case["B"] * case["D"]
        part = 0.5 if case.get("ragged") else 1.0      # tokens that are not padding, on the average
        if op == "scan_train":      # x, g, dy in; y, dx, dg out; the two ends of the state and of its gradient
            return {"bytes": int((3 + 3 * part) * s * n) + 4 * state, "flops": int(20 * n * part)}
        return {"bytes": int((1 + 2 * part) * s * n) + 2 * state, "flops": int(8 * n * part)}
    if op.startswith("linear"):
        R, K, N, act = case["R"], case["K"], case["N"], case["act"]
        if op == "linear":
            return {"bytes": 2 * (R * K + N * K + R * N * (2 if case["residual"] else 1)) + (4 * N if case["bias"] else 0),
                    "flops": 2 * R * K * N}
        return {"bytes": 2 * (2 * R * K + 2 * N * K + R * N * (1 if act == "none" else 2)) + (4 * N if case["bias"] else 0),
                "flops": 4 * R * K * N}
    n = sum(_sizes(case))
    moments = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    # bf16 weights beside masters are only written
    weights = BYTES[case["param"]] + 8 if case["master"] else 2 * BYTES[case["param"]]
    return {"bytes": n * (weights + BYTES[case["grad"]] + moments), "flops": 15 * n}


# ---------------------------------------------------- definitions in 64 bits
def exact(case, seed):
    op, st = case["op"], prepare(case, seed)
    if op.startswith("scan"):
        return _exact_scan(case, st)
    if op.startswith("linear"):
        return _exact_linear(case, st)
    return _exact_adamw(case, st)


def _exact_scan(case, st):
    """The recurrence and the chain rule, token by token."""
    g, x = st["g"].double(), st["x"].double()
    a = torch.sigmoid(g)
    if case["op"] == "scan_decode":
        h = a * st["h"].double() + ((1 - a) * x if case["leak"] else x)
        return {"y": h, "state": h}
    B, L, D = x.shape
    n = st["lengths"] if st["lengths"] is not None else torch.full((B,), L, device="cuda")
    live = (torch.arange(L, device="cuda")[:, None] < n[None, :])[..., None]         # [L][B][1]
    a, x = a.transpose(0, 1).contiguous(), x.transpose(0, 1).contiguous()            # [L][B][D]
    drive = torch.sigmoid(-g.transpose(0, 1)) * x if case["leak"] else x
    a, drive = torch.where(live, a, 1.0), torch.where(live, drive, 0.0)
    h, before = st["h0"].double(), torch.empty_like(a)
    y = torch.empty_like(a)
    for t in range(L):
        before[t] = h
        h = torch.addcmul(drive[t], a[t], h)
        y[t] = h
    field = lambda v: torch.where(live, v, 0.0).transpose(0, 1)  # noqa: E731
    if case["op"] == "scan_prefill":
        return {"y": field(y), "state": h}
    dy = torch.where(live, st["dy"].double().transpose(0, 1), 0.0)
    back, grad = st["dh"].double(), torch.empty_like(a)          # dl/dh_t from later tokens
    for t in range(L - 1, -1, -1):
        torch.add(dy[t], back, out=grad[t])
        back = a[t] * grad[t]
    rest = torch.sigmoid(-g.transpose(0, 1))
    da = grad * (before - x if case["leak"] else before)
    return {"state": h, "dh0": back, "y": field(y), "dx": field(grad * rest if case["leak"] else grad),
            "dg": field(da * a * rest)}


def _exact_linear(case, st):
    f = {"none": lambda z: z, "silu": torch.nn.functional.silu, "sigmoid": torch.sigmoid,
         "gelu": lambda z: torch.nn.functional.gelu(z, approximate="tanh")}[case["act"]]
    x, w = st["x"].double(), st["w"].double()
    if case["op"] == "linear":
        z = x @ w.T
        if st["bias"] is not None:
            z += st["bias"].double()
        y = f(z)
        if st["residual"] is not None:
            y = y + st["residual"].double()
        return {"y": y}
    d = st["dy"].double()
    if st["pre"] is not None:
        z = st["pre"].double().requires_grad_()
        d, = torch.autograd.grad(f(z), z, d)
    out = {"dx": d @ w, "dw": d.T @ x}
    if st["bias"] is not None:
        out["dbias"] = d.sum(0)
    return out


def _exact_adamw(case, st):
    t = st["step"] + 1
    g, eight = st["grad"].double(), case["bits"] == 8
    if eight:
        m = (st["m"].double().view(-1, BLOCK) * st["m_scale"].double()[:, None]).view(-1)
        v = (st["v"].double().view(-1, BLOCK) * st["v_scale"].double()[:, None]).view(-1) ** 2
    else:
        m, v = st["m"].double(), st["v"].double()
    m = m + (1 - BETA1) * (g - m)
    v = v + (1 - BETA2) * (g * g - v)
    p = (st["master"] if case["master"] else st["param"]).double()
    p = p - LR * WD * p - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
    out = {"param": p}
    if case["master"]:
        out["master"] = p
    if not eight:
        return dict(out, m=m, v=v)
    # The 8-bit codes stand for these values before they are rounded to 4 significant bits.
    for k, val in (("m", m), ("v", v.sqrt())):
        b = val.view(-1, BLOCK)
        top = b.abs().amax(1)
        scale = torch.where(top > 0, 2.0 ** (torch.floor(torch.log2(top.clamp(min=2.0 ** -101))) - 7), 2.0 ** -108)
        out[k], out[k + "_scale"] = (b / scale[:, None]).view(-1), scale
    return out
