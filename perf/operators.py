"""Cases of the operators around a mixer: the short causal convolution before it, the selective state space scan beside the
delta-rule mixers, and the norms before and after it.

    own                 False: `run` computes the plain form; True: it calls the framework's entry points
    listed(), draw(rng) the named cases, and one more of the ranges they stand for
    prepare(case, seed) what a program holds on the GPU before the call
    run(state)          one pass; returns every output whole
    work(case)          bytes and operations that one pass cannot do without
    exact(case, seed)   the outputs from the definitions, in 64 bits

A case names an operation and its sizes:
    op      "conv", "conv_bwd", "conv_step"     short causal depthwise convolution and SiLU over C channels, W taps
            "ssm", "ssm_bwd", "ssm_step"        selective state space scan: H heads of dv channels, G groups of keys and queries of dk
            "norm", "norm_bwd"                  RMS norm of `width` channels: "add" (of residual + scale * x) or "gate" (times SiLU of a gate)
    B, T                sequences and tokens of each; or
    n_seq, max_len      packed sequences, lengths drawn uniformly in [1, max_len] (lens_seed)
    dtype               "bf16" or "f32"
    state               whether the call starts from a given state (and, backwards, has a gradient of the final one)

The values are those a layer meets: activations of unit size behind a SiLU, steps dt log-uniform in [0.001, 0.1], decay rates
uniform in [1, 16], norm weights around one.  Values, keys and queries of the scan are slices of one array, as the convolution
before it leaves them.
"""
import math
import random

import torch

own = False

EPS = 1e-6


def listed():
    return [
        # the convolution of a training layer: 2048 channels of values, 128 of keys and 128 of queries
        dict(name="conv B8 T4096", op="conv", B=8, T=4096, C=2304, W=4, dtype="bf16", state=False),
        # its gradient, over packed sequences of all lengths that continue from earlier parts
        dict(name="conv backward packed 16", op="conv_bwd", n_seq=16, max_len=4096, lens_seed=2001, C=2304, W=4, dtype="bf16", state=True),
        # one token for each of 64 users
        dict(name="conv step B64", op="conv_step", B=64, C=2304, W=4, dtype="bf16"),
        # the scan of a training layer, hidden size 1024 expanded twice
        dict(name="scan B8 T4096", op="ssm", B=8, T=4096, H=32, G=1, dk=128, dv=64, dtype="bf16", state=False),
        # a prompt of ragged length, and a context of 65 536 tokens that continues from a state
        dict(name="scan prompt 777", op="ssm", B=1, T=777, H=32, G=1, dk=128, dv=64, dtype="bf16", state=False),
        dict(name="scan long 65536", op="ssm", B=1, T=65536, H=8, G=8, dk=128, dv=128, dtype="bf16", state=True),
        # full precision: packed, small heads
        dict(name="scan fp32 packed 8", op="ssm", n_seq=8, max_len=1024, lens_seed=2002, H=8, G=2, dk=64, dv=64, dtype="f32", state=True),
        # the gradient of a training layer's scan, and of packed sequences
        dict(name="scan backward B8 T4096", op="ssm_bwd", B=8, T=4096, H=32, G=1, dk=128, dv=64, dtype="bf16", state=False),
        dict(name="scan backward packed 16", op="ssm_bwd", n_seq=16, max_len=4096, lens_seed=2003, H=16, G=2, dk=64, dv=64, dtype="bf16", state=True),
        # decoding: a batch whose states live in HBM
        dict(name="scan step B512", op="ssm_step", B=512, H=32, G=1, dk=128, dv=64, dtype="bf16"),
        # before a block: the residual stream in fp32 takes the previous block's output, scaled per channel, and is normed
        dict(name="norm add B8 T4096", op="norm", kind="add", B=8, T=4096, width=1024, group=1024, dtype="bf16", res="f32"),
        # after a mixer: each head's output is normed and gated, backwards
        dict(name="norm gate backward", op="norm_bwd", kind="gate", B=8, T=4096, width=2048, group=128, dtype="bf16", gate_first=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["conv", "conv_bwd", "conv_step", "ssm", "ssm", "ssm", "ssm_bwd", "ssm_bwd", "ssm_step", "norm", "norm_bwd"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    c = dict(op=op, dtype=dtype)
    if op.startswith("conv"):
        c.update(C=rng.choice([_log_int(rng, 64, 2304), 8 * _log_int(rng, 8, 288), 2304]), W=rng.choice([2, 3, 4, 4]))
        most = 32768 * 2304 // c["C"] // (2 if dtype == "f32" else 1)
    elif op.startswith("ssm"):
        H = rng.choice([2, 4, 8, 16, 32])
        dk, dv = rng.choice([64, 128, 128]), rng.choice([64, 64, 128])
        if rng.random() < 0.15:   # sizes that the tensor cores' kernels do not take
            dk, dv = rng.choice([16, 32, 96]), rng.choice([32, 48, 80])
        c.update(H=H, G=rng.choice([g for g in (1, 2, 4, 8) if H % g == 0]), dk=dk, dv=dv)
        most = 32768 * 32 * 64 * 128 // (H * dk * dv) // (2 if op == "ssm_bwd" else 1)
        if dtype == "f32" or dk % 64 or dv % 64:
            most //= 16
    else:
        kind = rng.choice(["add", "gate"])
        width = 8 * _log_int(rng, 8, 512) if rng.random() < 0.7 else _log_int(rng, 64, 4096)
        c.update(kind=kind, width=width, group=width)
        if kind == "gate":
            c.update(gate_first=rng.random() < 0.5)
            if rng.random() < 0.5:
                c.update(width=128 * rng.choice([4, 8, 16, 32]), group=rng.choice([64, 128]))
        else:
            c.update(res=rng.choice(["f32", dtype]))
        most = 32768 * 1024 // c["width"] // (2 if dtype == "f32" else 1)
    if op.endswith("_step"):
        c.update(B=_log_int(rng, 1, min(1024, max(1, most // 64 if op == "ssm_step" else 1024))))
        return c
    most = max(64, min(most, 65536))
    if not op.startswith("norm"):
        c.update(state=rng.random() < 0.5)
        if rng.random() < 0.4:
            n = _log_int(rng, 2, 32)
            c.update(n_seq=n, max_len=_log_int(rng, 2, max(2, min(4096, most // n))), lens_seed=rng.randrange(1 << 20))
            return c
    B = _log_int(rng, 1, 16)
    c.update(B=B, T=_log_int(rng, 1, max(1, most // B)))
    return c


def _lengths(case):
    if "n_seq" not in case:
        return [case["T"]] * case["B"]
    r = random.Random(case["lens_seed"])
    return [r.randint(1, case["max_len"]) for _ in range(case["n_seq"])]


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, dt = case["op"], _dtype(case["dtype"])
    step = op.endswith("_step")
    lens = [1] * case["B"] if step else _lengths(case)
    n_seq, packed = len(lens), "n_seq" in case
    lead = (case["B"],) if step else (1, sum(lens)) if packed else (case["B"], case["T"])

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    s = dict(case=case, op=op)
    s["host"] = s["cu"] = None
    if packed:
        s["host"] = torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32)
        s["cu"] = s["host"].cuda()
    if op.startswith("conv"):
        C, W = case["C"], case["W"]
        s["x"] = randn(*lead, C).to(dt)
        s["weight"] = (2 * rand(C, W) - 1) / W ** 0.5
        s["bias"] = 0.1 * randn(C)
        s["init"] = randn(n_seq, W - 1, C).to(dt) if step or case["state"] else None
        if op == "conv_bwd":
            s["d_out"] = randn(*lead, C).to(dt)
            s["d_final"] = randn(n_seq, W - 1, C).to(dt) if case["state"] else None
        return s
    if op.startswith("ssm"):
        H, G, dk, dv = case["H"], case["G"], case["dk"], case["dv"]
        z = torch.nn.functional.silu(1.5 * randn(*lead, H * dv + 2 * G * dk)).to(dt)
        s["v"] = z[..., :H * dv].unflatten(-1, (H, dv))
        s["k"] = z[..., H * dv:H * dv + G * dk].unflatten(-1, (G, dk))
        s["q"] = z[..., H * dv + G * dk:].unflatten(-1, (G, dk))
        s["dt"] = torch.exp(math.log(1e-3) + math.log(100.0) * rand(*lead, H))
        s["a"] = -(1.0 + 15.0 * rand(H))
        s["skip"] = 1.0 + 0.1 * randn(H)
        s["init"] = 0.5 * randn(n_seq, H, dk, dv) if step or case["state"] else None
        if op == "ssm_bwd":
            s["d_out"] = randn(*lead, H, dv).to(dt)
            s["d_final"] = randn(n_seq, H, dk, dv) if case["state"] else None
        return s
    D = case["width"]
    s["x"] = randn(*lead, D).to(dt)
    s["weight"] = 1.0 + 0.1 * randn(D)
    s["residual"] = s["scale"] = s["gate"] = None
    if case["kind"] == "add":
        s["residual"] = (2.0 * randn(*lead, D)).to(_dtype(case["res"]))
        s["scale"] = 0.5 + rand(D)
    else:
        s["gate"] = randn(*lead, D).to(dt)
    if op == "norm_bwd":
        s["d_out"] = randn(*lead, D).to(dt)
        s["d_residual"] = randn(*lead, D).to(s["residual"].dtype) if case["kind"] == "add" else None
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------------

def _offsets(s):
    """Offsets of the sequences in the rows of the call, on the GPU."""
    if s["cu"] is not None:
        return s["cu"].long()
    B, T = s["x" if "x" in s else "v"].shape[:2]
    return torch.arange(B + 1, device="cuda") * T


def _silu(x):
    return x / (1.0 + torch.exp(-x))


def _conv_taps(x, init, cu, W):
    """[rows, W, C]: the inputs under each tap (the last one is the row's own), from the state before a sequence's first token,
    and the state behind its last [n_seq, W - 1, C]."""
    rows, n = x.shape[0], cu.numel() - 1
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), cu[1:] - cu[:-1], output_size=rows)
    if init is None:
        init = x.new_zeros(n, W - 1, x.shape[1])
    both = torch.cat([x, init.flatten(0, 1)])   # row r < rows: a token; then the states
    at = torch.arange(rows, device="cuda")[:, None] - torch.arange(W - 1, -1, -1, device="cuda")
    before = at < cu[seq][:, None]
    at = torch.where(before, rows + seq[:, None] * (W - 1) + (W - 1) + at - cu[seq][:, None], at)
    last = cu[1:, None] - torch.arange(W - 1, 0, -1, device="cuda")
    empty = last < cu[:-1, None]
    last = torch.where(empty, rows + torch.arange(n, device="cuda")[:, None] * (W - 1) + (W - 1) + last - cu[:-1, None], last)
    return both[at], both[last]


def _plain_conv(x, weight, bias, init, cu):
    taps, final = _conv_taps(x, init, cu, weight.shape[1])
    return _silu((taps * weight.t()).sum(1) + bias), final


def _to_chunks(x, cu, host, Q, shape):
    """Rows of sequences [rows, ...] -> [n_seq, chunks, Q, ...], zeros behind each one's end."""
    if host is None:
        n, T = shape
        x = x.reshape(n, T, *x.shape[1:])
        pad = (-T) % Q
        if pad:
            x = torch.cat([x, x.new_zeros(n, pad, *x.shape[2:])], 1)
    else:
        Tm = max(1, int((host[1:] - host[:-1]).max()))
        Tm += (-Tm) % Q
        at = cu[:-1, None] + torch.arange(Tm, device="cuda")
        inside = (at < cu[1:, None]).reshape(*at.shape, *([1] * (x.dim() - 1)))
        x = torch.where(inside, x[at.clamp(max=x.shape[0] - 1)], x.new_zeros(()))
    return x.reshape(x.shape[0], x.shape[1] // Q, Q, *x.shape[2:])


def _from_chunks(y, cu, host, shape):
    y = y.flatten(1, 2)
    if host is None:
        return y[:, :shape[1]].flatten(0, 1)
    rows = int(host[-1])
    seq = torch.repeat_interleave(torch.arange(cu.numel() - 1, device="cuda"), cu[1:] - cu[:-1], output_size=rows)
    return y[seq, torch.arange(rows, device="cuda") - cu[seq]]


def _plain_scan(q, k, v, dt, a, skip, init, cu, host, shape, Q=64):
    """Rows in, rows out: chunks of Q tokens, sums of log decays in 64 bits, the rest in 32."""
    H, G = v.shape[1], q.shape[1]
    v0 = v
    q, k, v, dt = (_to_chunks(x, cu, host, Q, shape) for x in (q, k, v, dt))   # [n, c, Q, ...]
    l = torch.cumsum(dt.double() * a.double(), 2).transpose(2, 3)               # [n, c, H, Q]
    q, k, v, dt = (x.transpose(2, 3) for x in (q, k, v, dt))                    # [n, c, heads, Q, ...]
    causal = torch.ones(Q, Q, dtype=torch.bool, device="cuda").tril()
    decay = torch.exp(torch.where(causal, l[..., :, None] - l[..., None, :], -math.inf)).float()
    per = H // G
    m = torch.matmul(q, k.transpose(-1, -2)).repeat_interleave(per, 2) * decay * dt[..., None, :]
    y = torch.matmul(m, v)
    w = torch.exp(l[..., -1:] - l).float() * dt
    kh = k.repeat_interleave(per, 2)
    adds = torch.matmul(kh.transpose(-1, -2), w[..., None] * v)                 # [n, c, H, dk, dv]: what each chunk writes
    end = torch.cumsum(l[..., -1], 1)                                           # [n, c, H]: log decay up to each chunk's end
    to = torch.cat([torch.zeros_like(end[:, :1]), end], 1).transpose(1, 2)      # [n, H, c + 1]
    c = end.shape[1]
    later = torch.ones(c + 1, c, dtype=torch.bool, device="cuda").tril(-1)
    carry = torch.exp(torch.where(later, to[..., :, None] - to[..., None, 1:], -math.inf)).float()   # [n, H, c + 1, c]
    states = torch.matmul(carry, adds.transpose(1, 2).flatten(3))               # [n, H, c + 1, dk dv]: before each chunk
    if init is not None:
        states = states + torch.exp(to).float()[..., None] * init.flatten(2)[:, :, None]
    states = states.unflatten(-1, adds.shape[-2:])
    y = y + torch.exp(l).float()[..., None] * torch.matmul(q.repeat_interleave(per, 2), states[:, :, :-1].transpose(1, 2))
    y = _from_chunks(y.transpose(2, 3), cu, host, shape) + skip[:, None] * v0
    return y, states[:, :, -1]


def _plain_norm(x, weight, residual, scale, gate, group, gate_first):
    if residual is not None:
        x = residual + scale * x
    out = x * _silu(gate) if gate is not None and gate_first else x
    u = out.unflatten(-1, (-1, group))
    out = (u / torch.sqrt((u * u).mean(-1, keepdim=True) + EPS)).flatten(-2) * weight
    if gate is not None and not gate_first:
        out = out * _silu(gate)
    return out, x


def _f32(x):
    return None if x is None else x.float()


def _leaves(*ts):
    return [None if t is None else t.detach().float().requires_grad_() for t in ts]


def _grads(outs, d_outs, leaves):
    pairs = [(o, d.float()) for o, d in zip(outs, d_outs) if d is not None]
    got = iter(torch.autograd.grad([o for o, _ in pairs], [l for l in leaves if l is not None], [d for _, d in pairs]))
    return [None if l is None else next(got) for l in leaves]


def _run_plain(s):
    op, case = s["op"], s["case"]
    if op.startswith("conv"):
        x, init, w, b = s["x"], s["init"], s["weight"], s["bias"]
        if op == "conv_step":
            window = torch.cat([init, x[:, None]], 1)
            y = _silu((window.float() * w.t()).sum(1) + b)
            s["init"] = window[:, 1:].contiguous()
            return {"out": y.to(x.dtype), "state": s["init"]}
        cu, rows = _offsets(s), x.flatten(0, 1)
        if op == "conv":
            y, fin = _plain_conv(rows.float(), w, b, _f32(init), cu)
            return {"out": y.to(x.dtype).reshape(x.shape), "final_state": fin.to(x.dtype)}
        with torch.enable_grad():
            leaves = _leaves(rows, w, b, init)
            outs = _plain_conv(*leaves, cu)
            dx, dw, db, di = _grads(outs, (s["d_out"].flatten(0, 1), s["d_final"]), leaves)
        return {"dx": dx.to(x.dtype).reshape(x.shape), "dweight": dw, "dbias": db} | ({} if di is None else {"dinit_state": di.to(x.dtype)})
    if op.startswith("ssm"):
        q, k, v, dt, a, skip, init = (s[n] for n in ("q", "k", "v", "dt", "a", "skip", "init"))
        io = v.dtype
        if op == "ssm_step":
            per = v.shape[1] // q.shape[1]
            kh, qh = k.float().repeat_interleave(per, 1), q.float().repeat_interleave(per, 1)
            st = torch.exp(dt * a)[..., None, None] * init + (dt[..., None] * kh)[..., None] * v.float()[:, :, None]
            y = (qh[..., None] * st).sum(2) + skip[:, None] * v.float()
            s["init"] = st
            return {"out": y.to(io), "state": st}
        cu, shape = _offsets(s), v.shape[:2]
        flat = [x.flatten(0, 1) for x in (q, k, v, dt)]
        if op == "ssm":
            y, fin = _plain_scan(*(x.float() for x in flat), a, skip, init, cu, s["host"], shape)
            return {"out": y.to(io).reshape(v.shape), "final_state": fin}
        with torch.enable_grad():
            leaves = _leaves(*flat, a, skip, init)
            outs = _plain_scan(*leaves, cu, s["host"], shape)
            dq, dk, dv, ddt, da, dd, di = _grads(outs, (s["d_out"].flatten(0, 1), s["d_final"]), leaves)
        return {"dq": dq.to(io).reshape(q.shape), "dk": dk.to(io).reshape(k.shape), "dv": dv.to(io).reshape(v.shape), "ddt": ddt.reshape(dt.shape),
                "da": da, "dd": dd} | ({} if di is None else {"dinit_state": di})
    x, res, gate = s["x"], s["residual"], s["gate"]
    how = (case["group"], case.get("gate_first", False))
    if op == "norm":
        y, r = _plain_norm(x.float(), s["weight"], _f32(res), s["scale"], _f32(gate), *how)
        return {"out": y.to(x.dtype)} | ({} if res is None else {"residual_out": r.to(res.dtype)})
    with torch.enable_grad():
        leaves = _leaves(x, s["weight"], res, s["scale"], gate)
        outs = _plain_norm(*leaves, *how)
        dx, dw, dr, ds, dg = _grads(outs, (s["d_out"], s["d_residual"]), leaves)
    out = {"dx": dx.to(x.dtype), "dweight": dw}
    if res is not None:
        out |= {"dresidual": dr.to(res.dtype), "dscale": ds}
    if gate is not None:
        out |= {"dgate": dg.to(gate.dtype)}
    return out


# ---- the framework's entry points ----------------------------------------------------------------------------------------------

def _run_own(s):
    import paper_2605_08587_b200 as kla
    op, case = s["op"], s["case"]
    packed = dict(cu_seqlens=s["cu"], host_seqlens=s["host"])
    if op == "conv_step":
        out = kla.kla_conv_step(s["x"], s["weight"], s["init"], bias=s["bias"])   # the state moves on in place
        return {"out": out, "state": s["init"]}
    if op == "conv":
        out, fin = kla.kla_conv_fwd(s["x"], s["weight"], bias=s["bias"], init_state=s["init"], **packed)
        return {"out": out, "final_state": fin}
    if op == "conv_bwd":
        g = kla.kla_conv_bwd(s["x"], s["weight"], s["d_out"], bias=s["bias"], init_state=s["init"], d_final_state=s["d_final"],
                             want_dinit_state=s["init"] is not None, **packed)
        return {n: t for n, t in g.items() if t is not None}
    if op.startswith("ssm"):
        a = (s["q"], s["k"], s["v"], s["dt"], s["a"])
        if op == "ssm_step":
            out = kla.kla_ssm_step(*a, s["init"], d_skip=s["skip"])
            return {"out": out, "state": s["init"]}
        if op == "ssm":
            out, fin = kla.kla_ssm_fwd(*a, d_skip=s["skip"], init_state=s["init"], **packed)
            return {"out": out, "final_state": fin}
        g = kla.kla_ssm_bwd(*a, s["d_out"], d_skip=s["skip"], init_state=s["init"], d_final_state=s["d_final"],
                            want_dinit_state=s["init"] is not None, **packed)
        return {n: t for n, t in g.items() if t is not None}
    how = dict(residual=s["residual"], scale=s["scale"], gate=s["gate"], group=case["group"],
               flags=kla.KLA_FLAG_GATE_FIRST if case.get("gate_first") else kla.KLA_FLAG_NONE)
    if op == "norm":
        out, res = kla.kla_norm_fwd(s["x"], s["weight"], EPS, **how)
        return {"out": out} | ({} if res is None else {"residual_out": res})
    g = kla.kla_norm_bwd(s["x"], s["weight"], EPS, s["d_out"], d_residual_out=s["d_residual"], **how)
    return {n: t for n, t in g.items() if t is not None}


def run(s):
    return _run_own(s) if own else _run_plain(s)


def work(case):
    op, io = case["op"], 2 if case["dtype"] == "bf16" else 4
    rows = case["B"] if op.endswith("_step") else sum(_lengths(case))
    n = case["B"] if op.endswith("_step") else len(_lengths(case))
    state = case.get("state", False)
    if op.startswith("conv"):
        C, W = case["C"], case["W"]
        st = n * (W - 1) * C * io
        if op == "conv_step":
            return {"bytes": 2 * rows * C * io + 2 * st + C * (W + 1) * 4, "flops": rows * C * (2 * W + 4)}
        if op == "conv":
            return {"bytes": 2 * rows * C * io + (2 if state else 1) * st + C * (W + 1) * 4, "flops": rows * C * (2 * W + 4)}
        return {"bytes": 3 * rows * C * io + (3 if state else 0) * st + 2 * C * (W + 1) * 4, "flops": rows * C * (6 * W + 8)}
    if op.startswith("ssm"):
        H, G, dk, dv = case["H"], case["G"], case["dk"], case["dv"]
        st = n * H * dk * dv * 4
        tok = rows * (H * dv + 2 * G * dk) * io + rows * H * 4
        if op == "ssm_step":
            return {"bytes": 2 * st + tok + rows * H * dv * io, "flops": rows * H * 5 * dk * dv}
        if op == "ssm":
            return {"bytes": tok + rows * H * dv * io + (2 if state else 1) * st, "flops": rows * H * 4 * dk * dv}
        return {"bytes": 2 * tok + rows * H * dv * io + (3 if state else 0) * st, "flops": rows * H * 12 * dk * dv}
    D = case["width"]
    res = 0 if case["kind"] == "gate" else 2 if case["res"] == "bf16" else 4
    if op == "norm":   # x, out, and the residual twice or the gate
        return {"bytes": rows * D * (2 * io + (2 * res if res else io)) + 8 * D, "flops": rows * D * 8}
    return {"bytes": rows * D * (3 * io + (3 * res if res else 2 * io)) + 16 * D, "flops": rows * D * 20}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------------

def _d(x):
    return None if x is None else x.double()


def _exact_conv(s):
    """Sequence by sequence: the window [state; tokens] and its W shifted slices."""
    W = s["weight"].shape[1]
    w, b = s["weight"].double(), s["bias"].double()
    if s["op"] == "conv_step":
        win = torch.cat([s["init"], s["x"][:, None]], 1).double()
        pre = b + sum(w[:, i] * win[:, i] for i in range(W))
        return {"out": pre * torch.sigmoid(pre), "state": win[:, 1:]}
    bounds = (s["host"].tolist() if s["host"] is not None else [i * s["x"].shape[1] for i in range(s["x"].shape[0] + 1)])
    x = s["x"].flatten(0, 1)
    dy = s["d_out"].flatten(0, 1) if "d_out" in s else None
    outs, fins, dxs, dis = [], [], [], []
    dw, db = torch.zeros_like(w), torch.zeros_like(b)
    for n, (lo, hi) in enumerate(zip(bounds, bounds[1:])):
        before = s["init"][n].double() if s["init"] is not None else w.new_zeros(W - 1, w.shape[0])
        win = torch.cat([before, x[lo:hi].double()])
        T = hi - lo
        pre = b + sum(w[:, i] * win[i:i + T] for i in range(W))
        sig = torch.sigmoid(pre)
        if dy is None:
            outs.append(pre * sig)
            fins.append(win[T:])
            continue
        g = dy[lo:hi].double() * (sig + pre * sig * (1 - sig))
        db += g.sum(0)
        dwin = torch.zeros_like(win)
        for i in range(W):
            dw[:, i] += (g * win[i:i + T]).sum(0)
            dwin[i:i + T] += w[:, i] * g
        if s["d_final"] is not None:
            dwin[T:] += s["d_final"][n].double()
        dxs.append(dwin[W - 1:])
        dis.append(dwin[:W - 1])
    if dy is None:
        return {"out": torch.cat(outs).reshape(s["x"].shape), "final_state": torch.stack(fins)}
    out = {"dx": torch.cat(dxs).reshape(s["x"].shape), "dweight": dw, "dbias": db}
    return out if s["init"] is None else out | {"dinit_state": torch.stack(dis)}


def _exact_scan(s):
    """Token by token over all sequences at once; backwards with the states run again from every 64th."""
    q, k, v, dt = s["q"], s["k"], s["v"], s["dt"]
    a, skip = s["a"].double(), s["skip"].double()
    H, G = v.shape[-2], q.shape[-2]
    if s["op"] == "ssm_step":
        kh, qh = (x.double().repeat_interleave(H // G, 1) for x in (k, q))
        st = torch.exp(dt.double() * a)[..., None, None] * s["init"].double() + torch.einsum("bh,bhk,bhv->bhkv", dt.double(), kh, v.double())
        return {"out": torch.einsum("bhk,bhkv->bhv", qh, st) + skip[:, None] * v.double(), "state": st}
    if s["host"] is not None:
        lens = (s["host"][1:] - s["host"][:-1]).tolist()
        lay = lambda x: torch.nn.utils.rnn.pad_sequence(list(x[0].split(lens)), batch_first=True)  # noqa: E731
    else:
        lens = [v.shape[1]] * v.shape[0]
        lay = lambda x: x  # noqa: E731
    lead = v.shape[:2]
    back = lambda y: torch.cat([y[i, :m] for i, m in enumerate(lens)]).reshape(*lead, *y.shape[2:])  # noqa: E731
    q, k, v, dt = lay(q), lay(k), lay(v), lay(dt)
    n, T = dt.shape[:2]
    alpha = torch.exp(dt.double() * a)   # 1 behind a sequence's end, where nothing is written either
    grouped = (n, G, H // G)

    def write(S, t):
        kt, vt = k[:, t].double(), (dt[:, t, :, None].double() * v[:, t].double()).reshape(*grouped, -1)
        return S.mul(alpha[:, t].reshape(*grouped, 1, 1)).addcmul_(kt[:, :, None, :, None], vt[:, :, :, None])

    dkk, dvv = k.shape[-1], v.shape[-1]
    S = torch.zeros(*grouped, dkk, dvv, dtype=torch.float64, device="cuda") if s["init"] is None else s["init"].double().reshape(*grouped, dkk, dvv)
    if s["op"] == "ssm":
        y = torch.empty(n, T, H, dvv, dtype=torch.float64, device="cuda")
        for t in range(T):
            S = write(S, t)
            y[:, t] = torch.matmul(q[:, t].double()[:, :, None, None], S).reshape(n, H, dvv)
        return {"out": back(y + skip[:, None] * v.double()), "final_state": S.reshape(n, H, dkk, dvv)}
    dy = lay(s["d_out"])
    K, kept = 64, []
    for t in range(T):
        if t % K == 0:
            kept.append(S)
        S = write(S, t)
    Gr = torch.zeros_like(S) if s["d_final"] is None else s["d_final"].double().reshape(S.shape)
    dq, dk, dv, ddt = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (q, k, v, dt))
    da = torch.zeros_like(a)
    for c in reversed(range(len(kept))):
        hi, states = min(T, c * K + K), [kept[c]]
        for t in range(c * K, hi):
            states.append(write(states[-1], t))
        for t in reversed(range(c * K, hi)):
            g, vt, kt, qt = dy[:, t].double().reshape(*grouped, dvv), v[:, t].double().reshape(*grouped, dvv), k[:, t].double(), q[:, t].double()
            dq[:, t] = torch.matmul(states[t - c * K + 1], g[..., None])[..., 0].sum(2)
            Gr = Gr.addcmul(qt[:, :, None, :, None], g[:, :, :, None])
            Gv = torch.matmul(Gr, vt[..., None])[..., 0]                                     # [n, G, per, dk]
            step = dt[:, t].double().reshape(grouped)
            dk[:, t] = (step[..., None] * Gv).sum(2)
            dv[:, t] = (step[..., None] * torch.matmul(kt[:, :, None, None], Gr)[..., 0, :]).reshape(n, H, dvv)
            al = alpha[:, t].reshape(grouped)
            dla = al * (Gr * states[t - c * K]).sum((-1, -2))
            ddt[:, t] = ((Gv * kt[:, :, None]).sum(-1) + dla * a.reshape(G, -1)).reshape(n, H)
            da += (dla * step).sum(0).reshape(H)
            Gr = Gr * al[..., None, None]
    dd = (dy.double() * v.double()).sum((0, 1, 3))
    dv += skip[:, None] * dy.double()
    out = {"dq": back(dq), "dk": back(dk), "dv": back(dv), "ddt": back(ddt), "da": da, "dd": dd}
    return out if s["init"] is None else out | {"dinit_state": Gr.reshape(n, H, dkk, dvv)}


def _exact_norm(s):
    """With r = 1 / sqrt(mean u^2 + eps) and y = r u: du = r (g - y mean(g y)) for a gradient g of y."""
    case, x, w = s["case"], s["x"].double(), s["weight"].double()
    res, sc, z = _d(s["residual"]), _d(s["scale"]), _d(s["gate"])
    first = case.get("gate_first", False)
    act = None if z is None else z * torch.sigmoid(z)
    u = x if res is None else res + sc * x
    if z is not None and first:
        u = x * act
    shape = u.shape
    split = lambda t: t.reshape(-1, shape[-1] // case["group"], case["group"])  # noqa: E731
    r = (split(u).square().mean(-1, keepdim=True) + EPS).rsqrt()
    y = (split(u) * r).reshape(shape)
    if s["op"] == "norm":
        out = y * w if z is None or first else y * w * act
        return {"out": out} | ({} if res is None else {"residual_out": u})
    dy = s["d_out"].double()
    gw = dy if z is None or first else dy * act
    out = {"dweight": (gw * y).flatten(0, -2).sum(0)}
    g = split(gw * w)
    du = (r * (g - split(y) * (g * split(y)).mean(-1, keepdim=True))).reshape(shape)
    dact = None
    if res is not None:
        du = du + s["d_residual"].double()
        out |= {"dresidual": du, "dscale": (du * x).flatten(0, -2).sum(0)}
        du = du * sc
    elif first:
        dact, du = du * x, du * act
    else:
        dact = dy * y * w
    out["dx"] = du
    if dact is not None:
        sig = torch.sigmoid(z)
        out["dgate"] = dact * (sig + z * sig * (1 - sig))
    return out


def exact(case, seed):
    s = prepare(case, seed)
    order = {"conv_bwd": ("dx", "dweight", "dbias", "dinit_state"), "norm_bwd": ("dx", "dweight", "dresidual", "dscale", "dgate")}
    out = (_exact_conv if case["op"].startswith("conv") else _exact_scan if case["op"].startswith("ssm") else _exact_norm)(s)
    return {n: out[n] for n in order.get(case["op"], out) if n in out}
