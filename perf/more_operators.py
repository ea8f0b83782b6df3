"""Measured cases of the operators of a causal block with a matrix state: the
gated delta rule (whole sequences, single tokens, gradients), the norms before
and after a block fused with its gate and residual scale, and the clipping of
the gradients by their global norm.

Features are [batch, tokens, (L+1)^2, channels]; L = 0 is the ordinary layout
of scalar features.  ``op`` names the pass:

  delta_train     cgconv_delta_rule and the gradients of all its inputs
  delta_prompt    SequencePlan.delta_rule of prompts, with the state they leave
  delta_step      SequencePlan.delta_rule_step, one token of every sequence
  residual_train  cgconv_residual_norm and the gradients of all its inputs
  residual_fwd    the forward pass alone
  clip            clip_gradients, the gradients kept and the clipped ones beside them

``run`` computes the plain form in torch where ``own`` is false and calls the
package where it is true; ``exact`` is the definition in float64.
"""

import math
import random

import torch

own = False

EPS = 1e-5        # of the norms by degree
KEY_EPS = 1e-6    # of the keys' and queries' norm
CLIP_EPS = 1e-6
CHUNK = 64        # tokens of one chunk of the plain delta rule


def listed():
    return [
        # one token of one sequence: latency
        dict(name="delta_token", op="delta_step", dtype="bf16", B=1, N=1, L=0, C=2048, H=16, Hk=16, D=128),
        # one token of many sequences, keys and queries shared by two heads
        dict(name="delta_tokens", op="delta_step", dtype="bf16", B=64, N=1, L=0, C=2048, H=16, Hk=8, D=128),
        # a padded batch of prompts
        dict(name="delta_prompts", op="delta_prompt", dtype="bf16", B=4, N=8192, L=0, C=2048, H=16, Hk=16, D=128, ragged=True),
        # one long prompt: few heads, many tokens
        dict(name="delta_long", op="delta_prompt", dtype="bf16", B=1, N=32768, L=0, C=1024, H=8, Hk=8, D=128),
        # training on long rows of scalars
        dict(name="delta_train", op="delta_train", dtype="bf16", B=2, N=4096, L=0, C=1024, H=8, Hk=8, D=128),
        # training on equivariant features, odd token count, a piece of longer sequences with the states between the pieces
        dict(name="delta_train_vectors", op="delta_train", dtype="fp32", B=4, N=1999, L=2, C=32, H=4, Hk=2, D=24,
             ragged=True, carry=True),
        # one small set of vectors for inference, the shortest call: latency
        dict(name="residual_small", op="residual_fwd", dtype="fp32", B=1, N=64, L=2, C=4, gated=True),
        # between two blocks in training at the point-cloud size
        dict(name="residual_pointcloud", op="residual_train", dtype="fp32", B=8, N=16384, L=6, C=32, gated=True),
        # ordinary wide scalar rows in bf16
        dict(name="residual_wide", op="residual_train", dtype="bf16", B=8, N=2048, L=0, C=4096, gated=True),
        # few small parameters: latency
        dict(name="clip_small", op="clip", tensors=12, values=40000, bf16=0, shapes=1, tight=True),
        # the gradients of a large model, most in bf16, the norms' and biases' in fp32
        dict(name="clip_model", op="clip", tensors=290, values=700000000, bf16=70, shapes=2, tight=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["delta_train", "delta_train", "delta_prompt", "delta_prompt", "delta_step", "residual_train",
                     "residual_train", "residual_fwd", "clip"])
    if op == "clip":
        tensors = _log_int(rng, 1, 290)
        return dict(op=op, tensors=tensors, values=max(tensors, _log_int(rng, 1, 300000000)), bf16=rng.choice([0, 30, 70, 100]),
                    shapes=rng.randrange(1 << 20), tight=rng.random() < 0.7)
    case = {"op": op, "dtype": rng.choice(["fp32", "bf16"]), "L": rng.choice([0, 0, 0, 1, 2, 3, 4, 6])}
    K = (case["L"] + 1) ** 2
    case["B"] = _log_int(rng, 1, 16)
    if op.startswith("residual"):
        case["N"] = _log_int(rng, 1, 16384)
        case["C"] = _log_int(rng, 3, 4096 if case["L"] == 0 else 256)
        case["gated"] = rng.random() < 0.7
        while case["B"] * case["N"] * K * case["C"] > 1.5e8:
            case["B" if case["B"] > 1 else "C"] = (case["B" if case["B"] > 1 else "C"] + 1) // 2
        return case
    case["D"] = rng.choice([8, 16, 24, 32, 48, 64, 64, 96, 128, 128])
    case["Hk"] = rng.choice([1, 2, 4, 8])
    case["H"] = case["Hk"] * rng.choice([1, 1, 2, 4])
    if op == "delta_step":
        case["N"] = 1
        case["B"] = _log_int(rng, 1, 128)
    else:
        case["N"] = _log_int(rng, 1, 4096 if op == "delta_train" else 32768)
        case["ragged"] = rng.random() < 0.5
        case["carry"] = rng.random() < 0.4
    per = _log_int(rng, 1, 128 if case["L"] == 0 else 16)  # channels of a head
    # states of all tokens, and tokens' rows
    most = {"delta_train": 1.0e9, "delta_prompt": 8e9, "delta_step": 1.6e7}[op]
    while case["B"] * case["N"] * case["H"] * per * K * case["D"] > most:
        if case["B"] > 1:
            case["B"] = (case["B"] + 1) // 2
        elif per > 1:
            per = (per + 1) // 2
        else:
            case["N"] = (case["N"] + 1) // 2
    case["C"] = case["H"] * per
    return case


# ---- inputs --------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _sizes(case):
    """The tensors' sizes and types of a model's gradients: a few large, most
    small; sizes of every remainder."""
    r = random.Random(case["shapes"])
    share = [math.exp(r.uniform(0, 7)) for _ in range(case["tensors"])]
    total = sum(share)
    sizes = [max(1, int(case["values"] * s / total)) for s in share]
    return [(n, r.randrange(100) < case["bf16"]) for n in sizes]


def _views(sizes, device):
    """Contiguous tensors of these sizes within one buffer a type, each at a
    multiple of 16 bytes, and the buffers."""
    need = {torch.float32: 0, torch.bfloat16: 0}
    at = []
    for n, half in sizes:
        t = torch.bfloat16 if half else torch.float32
        at.append((t, need[t], n))
        need[t] += -(-n // 8) * 8
    flat = {t: torch.zeros(n, dtype=t, device=device) for t, n in need.items() if n}
    return [flat[t][a:a + n] for t, a, n in at], list(flat.values())


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 31))

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    op, s = case["op"], {}
    if op == "clip":
        s["grads"], flat = _views(_sizes(case), "cuda")
        for g in s["grads"]:  # every tensor has a size of its own
            g.normal_(generator=gen)
            g.mul_(float(math.exp(2.0 * math.sin(g.numel()))))
        s["out"], s["flat"] = _views(_sizes(case), "cuda")
        s["max_norm"] = 1.0 if case["tight"] else 1e6
        return s
    B, N, L, C = case["B"], case["N"], case["L"], case["C"]
    K, dt = (L + 1) ** 2, _type(case)
    lead = (B,) if op == "delta_step" else (B, N)
    if op.startswith("residual"):
        # a residual stream and a block's output: channels of unequal size
        s["x"] = (normal(B, N, K, C, dtype=dt).float() * (0.5 + uniform(C)) + normal(C, scale=0.3)).to(dt)
        s["u"] = (normal(B, N, K, C, dtype=dt).float() * (0.2 + uniform(C)) + normal(C, scale=0.1)).to(dt)
        s["gate"] = normal(B, N, C, dtype=dt) if case["gated"] else None
        s["post_weight"] = 1 + normal(L + 1, C, scale=0.1)
        s["scale"] = 0.5 + 0.2 * uniform(C)
        s["weight"] = 1 + normal(L + 1, C, scale=0.1)
        s["bias"] = normal(C, scale=0.1)
        if op == "residual_train":
            s["grad_r"], s["grad_y"] = normal(B, N, K, C, dtype=dt), normal(B, N, K, C, dtype=dt)
        return s
    H, Hk, D = case["H"], case["Hk"], case["D"]
    s["q"], s["k"] = normal(*lead, Hk, D, dtype=dt), normal(*lead, Hk, D, dtype=dt)
    s["v"] = normal(*lead, K, C, dtype=dt)
    # decays as trained models have them: rates of 1 to 16, steps of 1e-3 to 1e-1 that the token changes
    rate = 1 + 15 * uniform(H)
    first = torch.exp(uniform(H) * math.log(100.0) + math.log(1e-3))
    raw = first + torch.log(-torch.expm1(-first)) + normal(*lead, H, scale=0.5)
    s["decay"] = -rate * torch.log1p(torch.exp(raw))
    s["beta"] = 1 / (1 + torch.exp(-normal(*lead, H)))
    if op == "delta_step" or case.get("carry"):
        s["state"] = normal(B, D, K, C, scale=0.2)
    if case.get("ragged"):
        s["lengths"] = torch.randint(N // 2, N + 1, (B,), generator=gen, device="cuda").to(torch.int32)
        s["lengths"][0] = N
    if op == "delta_train":
        s["grad"] = normal(B, N, K, C, dtype=dt)
        if case.get("carry"):
            s["grad_state"] = normal(B, D, K, C, scale=0.2)
    return s


LEAVES = {"delta_train": ("q", "k", "v", "decay", "beta", "state"),
          "residual_train": ("x", "u", "gate", "post_weight", "scale", "weight", "bias")}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2509_24093_amd as P

        s["P"] = P
        sizes = [case.get(n) for n in ("B", "N", "L", "C")]
        if case["op"].startswith("delta"):
            s["plan"] = P.SequencePlan(*sizes, heads=case["H"], key_heads=case["Hk"], key_dim=case["D"],
                                       backward=case["op"] == "delta_train")
        elif case["op"].startswith("residual"):
            s["plan"] = P.SequencePlan(*sizes)
    for name in LEAVES.get(case["op"], ()):
        if s.get(name) is not None:
            s[name].requires_grad_(True)
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    if op == "clip":
        return _plain_clip(s)
    if op == "delta_step":
        return _plain_step(s)
    if op == "delta_prompt":
        with torch.no_grad():
            y, state = _plain_delta(s)
        return {"y": y.to(s["v"].dtype), "state": state}
    if op == "delta_train":
        y, state = _plain_delta(s)
        y = y.to(s["v"].dtype)
        return _with_gradients(s, {"y": y, "state": state} if "state" in s else {"y": y})
    r, y = _plain_residual(s)
    out = {"r": r.to(s["x"].dtype), "y": y.to(s["x"].dtype)}
    return _with_gradients(s, out) if op == "residual_train" else out


def _with_gradients(s, out):
    """The outputs and the gradients of the leaves, given the outputs' own."""
    of = {"y": "grad_y" if "grad_y" in s else "grad", "r": "grad_r", "state": "grad_state"}
    names = [n for n in LEAVES[s["case"]["op"]] if s.get(n) is not None]
    grads = torch.autograd.grad(list(out.values()), [s[n] for n in names], [s[of[n]] for n in out])
    return dict({"grad_" + n: g for n, g in zip(names, grads)}, **{n: t.detach() for n, t in out.items()})


# ---- the package's calls ---------------------------------------------------------

def _own(s, op):
    P, plan = s["P"], s.get("plan")
    if op == "clip":
        norm = P.clip_gradients(s["grads"], s["max_norm"], eps=CLIP_EPS, out=s["out"])
        return {"norm": norm, "clipped": s["flat"]}
    if op.startswith("residual"):
        args = [s[n] for n in ("x", "u", "gate", "post_weight", "scale", "weight", "bias")]
        if op == "residual_fwd":
            r, y = plan.residual_norm(*args, eps=EPS)[:2]
            return {"r": r, "y": y}
        r, y = P.cgconv_residual_norm(*args, plan, eps=EPS)
        return _with_gradients(s, {"r": r, "y": y})
    args = [s[n] for n in ("q", "k", "v", "decay", "beta")]
    if op == "delta_step":
        return {"y": plan.delta_rule_step(*args, s["state"]), "state": s["state"]}
    if op == "delta_prompt":
        y, state = plan.delta_rule(*args, lengths=s.get("lengths"), state=s.get("state"))
        return {"y": y, "state": state}
    if "state" in s:
        y, state = P.cgconv_delta_rule(*args, plan, lengths=s.get("lengths"), state=s["state"], return_state=True)
        return _with_gradients(s, {"y": y, "state": state})
    return _with_gradients(s, {"y": P.cgconv_delta_rule(*args, plan, lengths=s.get("lengths"))})


# ---- the plain forms: delta rule ----------------------------------------------------

def _unit(t):
    return t * torch.rsqrt((t * t).sum(-1, keepdim=True) + KEY_EPS)


def _heads(t, H):
    """[..., Hk, D] with every key head as often as heads share it."""
    return t.repeat_interleave(H // t.shape[-2], -2)


def _split(t, K, H):
    """[..., K, C] as [..., H, K P]: a head's channels of all components."""
    t = t.reshape(*t.shape[:-1], H, -1)
    return t.transpose(-3, -2).reshape(*t.shape[:-3], H, -1)


def _join(t, K):
    """The inverse of _split."""
    t = t.reshape(*t.shape[:-1], K, -1).transpose(-3, -2)
    return t.reshape(*t.shape[:-2], -1)


def _chunked(t):
    """[B, N, H, ...] as [B H, chunks, CHUNK, ...], zeros behind the last token."""
    B, N, H = t.shape[:3]
    n = -(-N // CHUNK)
    t = torch.cat([t, t.new_zeros(B, n * CHUNK - N, *t.shape[2:])], 1) if n * CHUNK > N else t
    t = t.reshape(B, n, CHUNK, H, *t.shape[3:]).permute(0, 3, 1, 2, *range(4, t.ndim + 1))
    return t.reshape(B * H, n, CHUNK, *t.shape[4:])


def _triangle_inverse(A):
    """(1 + A)^-1 of strictly lower triangles, block by block of doubled size."""
    n, T = A.shape[0], A.shape[-1]
    inv = A.new_ones(n, T, 1, 1)
    size = 1
    while size < T:
        two, count = 2 * size, T // (2 * size)
        blocks = A.reshape(n, count, two, count, two).diagonal(dim1=1, dim2=3).permute(0, 3, 1, 2)
        low = blocks[:, :, size:, :size]
        first, second = inv[:, 0::2], inv[:, 1::2]
        corner = -torch.matmul(torch.matmul(second, low), first)
        top = torch.cat([first, torch.zeros_like(first)], -1)
        inv = torch.cat([top, torch.cat([corner, second], -1)], -2)
        size = two
    return inv[:, 0]


def _plain_delta(s):
    """The outputs in fp32 and the state behind every sequence's last token."""
    case = s["case"]
    B, N, H, D, K = case["B"], case["N"], case["H"], case["D"], (case["L"] + 1) ** 2
    there = s["v"].new_ones(B, N, dtype=torch.float32)
    if "lengths" in s:
        there = (torch.arange(N, device=there.device)[None] < s["lengths"][:, None]).float()
    there = there[:, :, None]
    q = _chunked(_heads(_unit(s["q"].float()), H) * there[..., None] / math.sqrt(D))
    k = _chunked(_heads(_unit(s["k"].float()), H) * there[..., None])
    v = _chunked(_split(s["v"].float(), K, H) * there[..., None])
    beta = _chunked(s["beta"] * there)
    total = torch.cumsum(_chunked(s["decay"].double() * there), -1)  # within the chunk
    n = q.shape[1]
    row = torch.arange(CHUNK, device=q.device)
    lower = row[:, None] >= row[None]
    between = torch.where(lower, total[..., :, None] - total[..., None, :], 0.0).exp().float() * lower
    strict = between * (row[:, None] > row[None])
    A = beta[..., None] * strict * torch.matmul(k, k.transpose(-1, -2))
    inverse = _triangle_inverse(A.reshape(-1, CHUNK, CHUNK)).reshape(A.shape)
    inside = between * torch.matmul(q, k.transpose(-1, -2))
    since = total.exp().float()[..., None]
    until = (total[..., -1:] - total).exp().float()[..., None]
    q, late = q * since, (k * until).transpose(-1, -2)
    k, whole = k * since, total[..., -1].exp().float()[..., None, None]
    state = v.new_zeros(B * H, D, v.shape[-1])
    if "state" in s:
        state = _split(s["state"], K, H).transpose(1, 2).reshape(B * H, D, -1)
    out = []
    for c in range(n):
        new = torch.matmul(inverse[:, c], beta[:, c, :, None] * (v[:, c] - torch.matmul(k[:, c], state)))
        out.append(torch.matmul(q[:, c], state) + torch.matmul(inside[:, c], new))
        state = whole[:, c] * state + torch.matmul(late[:, c], new)
    y = torch.stack(out, 1).reshape(B, H, n * CHUNK, -1)[:, :, :N].transpose(1, 2)
    state = _join(state.reshape(B, H, D, -1).transpose(1, 2), K)
    return _join(y, K), state.contiguous()


def _plain_step(s):
    case = s["case"]
    H, D, K = case["H"], case["D"], (case["L"] + 1) ** 2
    q = _heads(_unit(s["q"].float()), H).transpose(1, 2)[..., None] / math.sqrt(D)  # [B, D, H, 1]
    k = _heads(_unit(s["k"].float()), H).transpose(1, 2)[..., None]
    state = _split(s["state"], K, H) * torch.exp(s["decay"])[:, None, :, None]  # [B, D, H, K P]
    new = s["beta"][..., None] * (_split(s["v"].float(), K, H) - (k * state).sum(1))
    state = state + k * new[:, None]
    s["state"].copy_(_join(state, K))
    return {"y": _join((q * state).sum(1), K).to(s["v"].dtype), "state": s["state"]}


# ---- the plain forms: residual norm and clipping ---------------------------------------

def _plain_norm(x, weight, bias, L):
    rows = []
    for l in range(L + 1):  # a degree's components share their statistics
        d = x[:, :, l * l:(l + 1) ** 2]
        if l == 0:
            d = d - d.mean(-1, keepdim=True)
        h = d * torch.rsqrt((d * d).mean((2, 3), keepdim=True) + EPS) * weight[l]
        rows.append(h + bias if l == 0 and bias is not None else h)
    return torch.cat(rows, 2)


def _plain_residual(s):
    L = s["case"]["L"]
    p = _plain_norm(s["u"].float(), s["post_weight"], None, L) * s["scale"]
    if s["gate"] is not None:
        g = s["gate"].float()[:, :, None]
        p = p * (g / (1 + torch.exp(-g)))
    r = s["x"].float() + p
    return r, _plain_norm(r, s["weight"], s["bias"], L)


def _plain_clip(s):
    norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
    factor = torch.clamp(s["max_norm"] / (norm + CLIP_EPS), max=1.0).float()
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * factor)
    return {"norm": norm.float(), "clipped": s["flat"]}


# ---- what a pass cannot do without ------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "clip":
        sizes = _sizes(case)
        return {"bytes": 2 * sum(n * (2 if half else 4) for n, half in sizes), "flops": 3 * sum(n for n, _ in sizes)}
    B, N, L, C = case["B"], case["N"], case["L"], case["C"]
    K, size = (L + 1) ** 2, 2 if case["dtype"] == "bf16" else 4
    n = B * N * K * C * size
    if op.startswith("residual"):
        gate = B * N * C * size if case["gated"] else 0
        par = (2 * (L + 1) + 2) * C * 4
        if op == "residual_fwd":
            return {"bytes": 4 * n + gate + par, "flops": 16 * B * N * K * C}
        return {"bytes": 10 * n + 3 * gate + 3 * par, "flops": 50 * B * N * K * C}
    H, Hk, D = case["H"], case["Hk"], case["D"]
    V = K * C // H
    rows, gates, state = 2 * B * N * Hk * D * size, 2 * B * N * H * 4, B * D * K * C * 4
    if op == "delta_step":
        return {"bytes": rows + gates + 2 * n + 2 * state, "flops": 7 * B * H * D * V}
    flops = 6 * B * N * H * D * V  # read with the key, write, read with the query
    carried = state if case.get("carry") else 0
    if op == "delta_prompt":
        return {"bytes": rows + gates + 2 * n + state + carried, "flops": flops}
    # forward; backward reads the inputs and the outputs' gradient and writes the inputs' gradients
    return {"bytes": 3 * rows + 3 * gates + 5 * n + 5 * carried, "flops": 3 * flops}


# ---- the definitions in float64 ----------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "clip":
        return _exact_clip(s)
    d = {n: t.double() if t is not None and t.is_floating_point() else t for n, t in s.items()}
    if case["op"].startswith("residual"):
        return _exact_residual(case, d)
    return _exact_delta(case, d)


def _exact_delta(case, d):
    """Token by token."""
    op, B, N, H, D = case["op"], case["B"], case["N"], case["H"], case["D"]
    K, P = (case["L"] + 1) ** 2, case["C"] // H
    train = op == "delta_train"
    names = [n for n in LEAVES["delta_train"] if n in d]
    for n in names:
        d[n].requires_grad_(train)
    with torch.set_grad_enabled(train):
        def tokens(t):
            return (t[:, None] if op == "delta_step" else t)

        each = H // case["Hk"]
        q, k = (tokens(d[n]) / (tokens(d[n]).square().sum(-1, keepdim=True) + KEY_EPS).sqrt() for n in ("q", "k"))
        q = q * D ** -0.5
        qs, ks, vs, gs, bs = (t.unbind(1) for t in (q, k, tokens(d["v"]), tokens(d["decay"]), tokens(d["beta"])))
        # states [B, key heads, heads that share them, D, K, P]
        S = d["v"].new_zeros(B, D, K, case["C"])
        if "state" in d:
            S = d["state"]
        S = S.reshape(B, D, K, case["Hk"], each, P).permute(0, 3, 4, 1, 2, 5)
        ends = None if d.get("lengths") is None else d["lengths"].tolist()
        ys = []
        for t in range(N):
            kt, qt = ks[t][:, :, None, :, None, None], qs[t][:, :, None, :, None, None]
            vt = vs[t].reshape(B, K, case["Hk"], each, P).permute(0, 2, 3, 1, 4)
            gt, bt = (x[t].reshape(B, case["Hk"], each, 1, 1) for x in (gs, bs))
            F = gt.exp()[:, :, :, None] * S
            new = F + kt * (bt * (vt - (kt * F).sum(3)))[:, :, :, None]
            y = (qt * new).sum(3)
            if ends is not None and t >= min(ends):
                on = torch.tensor([t < e for e in ends], device=y.device)
                new = torch.where(on[:, None, None, None, None, None], new, S)
                y = torch.where(on[:, None, None, None, None], y, torch.zeros_like(y))
            S = new
            ys.append(y.permute(0, 3, 1, 2, 4).reshape(B, K, -1))
        y = ys[0] if op == "delta_step" else torch.stack(ys, 1)
        S = S.permute(0, 3, 4, 1, 2, 5).reshape(B, D, K, case["C"])
    if not train:
        return {"y": y, "state": S}
    outs = {"y": y, "state": S} if "state" in d else {"y": y}
    given = {"y": d["grad"], "state": d.get("grad_state")}
    grads = torch.autograd.grad(list(outs.values()), [d[n] for n in names], [given[n] for n in outs])
    return dict({"grad_" + n: g for n, g in zip(names, grads)}, **{n: t.detach() for n, t in outs.items()})


def _exact_residual(case, d):
    L, train = case["L"], case["op"] == "residual_train"
    degree = torch.tensor([l for l in range(L + 1) for _ in range(2 * l + 1)], device=d["x"].device)
    count = torch.bincount(degree).double() * case["C"]

    def norm(x, w, b):
        first = torch.zeros_like(x)
        first[:, 0] = x[:, 0].mean(-1, keepdim=True)
        x = x - first
        per = torch.zeros(x.shape[0], L + 1, dtype=x.dtype, device=x.device).index_add(1, degree, x.square().sum(-1))
        x = x / (per / count + EPS).sqrt()[:, degree, None] * w[degree]
        if b is not None:
            x = x + torch.cat([b[None], b.new_zeros(x.shape[1] - 1, x.shape[2])])
        return x

    whole = ("post_weight", "scale", "weight", "bias")
    rows = [n for n in ("x", "u", "gate") if d[n] is not None]
    got = {n: [] for n in ["r", "y"] + (["grad_" + n for n in rows] if train else [])}
    total = {}
    for b in range(case["B"]):  # batch elements on their own: less memory at once
        leaf = {n: d[n][b].clone().requires_grad_(train) for n in rows}
        leaf.update({n: d[n].clone().requires_grad_(train) for n in whole})
        p = norm(leaf["u"], leaf["post_weight"], None) * leaf["scale"]
        if "gate" in leaf:
            p = p * (leaf["gate"] * torch.sigmoid(leaf["gate"]))[:, None]
        r = leaf["x"] + p
        y = norm(r, leaf["weight"], leaf["bias"])
        if train:
            grads = torch.autograd.grad((r, y), list(leaf.values()), (d["grad_r"][b], d["grad_y"][b]))
            for n, g in zip(leaf, grads):
                if n in rows:
                    got["grad_" + n].append(g)
                else:
                    total["grad_" + n] = total.get("grad_" + n, 0) + g
        got["r"].append(r.detach())
        got["y"].append(y.detach())
    return dict({n: torch.stack(t) for n, t in got.items()}, **total)


def _exact_clip(s):
    square = sum(float((g.double() ** 2).sum()) for g in s["grads"])
    norm = math.sqrt(square)
    factor = min(1.0, s["max_norm"] / (norm + CLIP_EPS))
    outs = [torch.zeros(f.shape, dtype=torch.float64, device=f.device) for f in s["flat"]]
    for g, o in zip(s["grads"], s["out"]):
        flat = next(i for i, f in enumerate(s["flat"]) if f.dtype == o.dtype)
        at = o.storage_offset()
        outs[flat][at:at + g.numel()] = g.double() * factor
    return {"norm": torch.tensor(norm, dtype=torch.float64, device=outs[0].device), "clipped": outs}
