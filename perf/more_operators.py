"""Workloads of the operators that train the experts of a block, and serve them: the gated feed-forward block over packed expert
segments, its gradient, and the activation checkpoints in 8 bits that lie between the two.

`run` makes the calls of the public entry points where `own` is true, and computes the same from elementary torch operations in 32
bits where it is false.  A case is a dict of
  op     "ffn"         y of the packed rows (with keep: the pre-activations as well)
         "backward"    dx, dW1 and dW2 from dy, the input rows and the pre-activations, both kept in full or both in 8 bits
         "step"        forward and backward of one training step, whose checkpoints stay between the two
         "checkpoint"  rows packed into 8 bits and restored
  rows   items that the gate has routed (checkpoint: rows); an expert takes 1.25 times an even share of them at most
  d, F   model width, hidden width (checkpoint: d alone)
  E      experts, some of which may have no rows
  dtype  "bf16" or "f32"
  act    "silu", "gelu" (erf) or "gelu_tanh"
  keep   "", "full" or "8bit": the pre-activations (backward, step: the input rows too) stay for the backward pass like this
"""
import math

import torch

own = False

DEV = "cuda:0"
CAPACITY_FACTOR = 1.25
BLOCK = 32                # columns that share a scale
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(op, rows, d, F=0, E=0, dtype="bf16", act="", keep=""):
    return dict(op=op, rows=rows, d=d, F=F, E=E, dtype=dtype, act=act, keep=keep)


def listed():
    cases = [
        # a decode step of one token at the widths of the large layer: latency, and one expert's weights read once
        ("ffn_decode_1", _case("ffn", 1, 2048, 8192, 16, act="silu")),
        # a batch of decode steps: a few rows of every expert, all weights read once
        ("ffn_decode_64", _case("ffn", 64, 2048, 8192, 16, act="silu")),
        # the smallest configuration, fp32: latency and launches
        ("ffn_tiny_f32", _case("ffn", 256, 64, 256, 4, dtype="f32", act="gelu")),
        # an odd number of rows over many experts, widths that fill no tile
        ("ffn_ragged_e32", _case("ffn", 5003, 1000, 2728, 32, act="gelu_tanh")),
        # GPT-style widths: a prompt's rows
        ("ffn_medium", _case("ffn", 16384, 1024, 4096, 8, act="silu")),
        # the vision layer's widths, training with everything kept
        ("backward_small", _case("backward", 8192, 384, 1536, 8, act="gelu", keep="full")),
        # odd sizes in fp32
        ("backward_ragged_f32", _case("backward", 777, 1000, 1360, 5, dtype="f32", act="gelu_tanh", keep="full")),
        # the large layer's gradient
        ("backward_large", _case("backward", 32768, 2048, 8192, 16, act="silu", keep="full")),
        # a step of many experts with a few rows each
        ("step_e64_8bit", _case("step", 2000, 768, 2048, 64, act="silu", keep="8bit")),
        # GPT-style widths: a training step with its checkpoints in 8 bits
        ("step_medium_8bit", _case("step", 16384, 1024, 4096, 8, act="silu", keep="8bit")),
        # a few rows of an odd width in fp32
        ("checkpoint_small_f32", _case("checkpoint", 500, 1000, dtype="f32")),
        # the hidden rows of the large layer
        ("checkpoint_large", _case("checkpoint", 32768, 8192)),
    ]
    return [dict(c, name=n) for n, c in cases]


def draw(rng):
    """One more call of these ranges: 1 to 32768 rows, widths 64 to 2048 (checkpoint: 8192), hidden widths one to four times as wide, 1 to 64 experts."""
    most = [max(work(c)[k] for c in listed()) for k in ("bytes", "flops")]
    while True:
        op = rng.choice(["ffn", "ffn", "backward", "backward", "step", "checkpoint"])
        rows = int(round(math.exp(rng.uniform(0.0, math.log(32768)))))
        dtype = rng.choice(["bf16", "bf16", "f32"])
        act, q8 = rng.choice(["silu", "silu", "gelu", "gelu_tanh"]), rng.random() < 0.5
        if op == "checkpoint":
            case = _case(op, rows, 8 * int(round(math.exp(rng.uniform(math.log(8), math.log(1024))))), dtype=dtype)
        else:
            d = 8 * int(round(math.exp(rng.uniform(math.log(8), math.log(256)))))
            F = min(8192, 8 * int(round(d / 8 * rng.uniform(1.0, 4.0))))
            E = int(round(math.exp(rng.uniform(0.0, math.log(64)))))
            # (fp32: a step's pre-activations next to the middle of two codes take either, which no tolerance of 32 bits has room for)
            keep = ("full" if q8 else "") if op == "ffn" else "8bit" if q8 and (op, dtype) != ("step", "f32") else "full"
            case = _case(op, rows, d, F, E, dtype, act, keep)
        w = work(case)
        if w["bytes"] <= most[0] and w["flops"] * (1 if dtype == "bf16" else 8) <= most[1]:
            return case


# ---- inputs ---------------------------------------------------------------------------------------


def _counts(rows, E, seed):
    """Kept rows of every expert: a gate that prefers some, others for another seed, and a capacity."""
    g = torch.Generator()
    g.manual_seed(rows * 64 + E)
    share = torch.softmax(0.5 * torch.randn(E, generator=g, dtype=torch.float64), 0)
    chosen = torch.multinomial(share, rows, replacement=True, generator=g)
    capacity = max(1, math.ceil(CAPACITY_FACTOR * rows / E))
    counts = torch.bincount(chosen, minlength=E).clamp(max=capacity)
    g.manual_seed(seed)
    return counts[torch.randperm(E, generator=g)], min(rows, E * capacity)


def _ld(width):
    """Bytes of a checkpoint row: a code per column, a scale per block, up to a multiple of 16."""
    return -(-(width + -(-width // BLOCK)) // 16) * 16


def _blocks(x):
    """x [n, w] as [n, blocks, 32], zeros behind the last column."""
    n, w = x.shape
    return torch.nn.functional.pad(x, (0, -w % BLOCK)).reshape(n, -1, BLOCK)


def _codes(x):
    """Codes [n, w] and scales' exponents [n, blocks] of rows in 32 bits."""
    b = _blocks(x)
    m, e = torch.frexp(b.abs().amax(2))
    e = (e - 9 + (m > 0.875).to(e.dtype)).clamp(-126, 127)
    return torch.ldexp(b, -e[:, :, None]).to(torch.float8_e4m3fn).reshape(x.shape[0], -1)[:, :x.shape[1]], e


def _values(codes, e):
    """The values, in 32 bits, that codes and exponents stand for."""
    return torch.ldexp(_blocks(codes.float()), e[:, :, None]).reshape(codes.shape[0], -1)[:, :codes.shape[1]]


def _through_8_bits(x):
    return _values(*_codes(x))


def _packed(x):
    """Checkpoint rows of x as bytes."""
    codes, e = _codes(x)
    out = torch.zeros(x.shape[0], _ld(x.shape[1]), dtype=torch.uint8, device=x.device)
    out[:, :x.shape[1]] = codes.view(torch.uint8)
    out[:, x.shape[1]:x.shape[1] + e.shape[1]] = (e + 127).to(torch.uint8)
    return out


def _restored(q, w):
    """The values, in 32 bits, of checkpoint rows."""
    blocks = -(-w // BLOCK)
    return _values(q[:, :w].contiguous().view(torch.float8_e4m3fn), q[:, w:w + blocks].to(torch.int32) - 127)


def prepare(case, seed):
    """Rows as the dispatch packs them, weights, and the buffers and the workspace that a program keeps.  Hidden states have a few
    outlier channels; gradients have the size that a mean over the rows gives."""
    c, g = case, torch.Generator(device=DEV)
    g.manual_seed(seed)
    d, F, E, tt = c["d"], c["F"], c["E"], TYPES[c["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device=DEV) * scale

    def states(n):
        channel = 0.3 * normal(d)
        channel[::61] *= 10.0
        return (normal(n, d) + channel).to(tt)

    if c["op"] == "checkpoint":
        x = states(c["rows"])
        return dict(case=c, x=x, q=torch.empty(x.shape[0], _ld(d), dtype=torch.uint8, device=DEV), restored=torch.empty_like(x))
    counts, most = _counts(c["rows"], E, seed)
    s = dict(case=c, rows=most, K=int(counts.sum()), E=E)
    s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).to(torch.int32).to(DEV)
    used = counts.nonzero()[:, 0]
    s["used"], s["most_of_one"] = used.to(DEV), int(counts.max())
    s["place"] = torch.cat([j * s["most_of_one"] + torch.arange(int(counts[e])) for j, e in enumerate(used)]).to(DEV)
    s["x"] = states(most)
    s["W1"], s["W2"] = normal(E, 2 * F, d, scale=d ** -0.5).to(tt), normal(E, d, F, scale=F ** -0.5).to(tt)
    new = lambda *shape, dtype=tt: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    if c["op"] != "backward":
        s["hidden"], s["y"] = new(most, F), new(most, d)
        s["pre"] = {"": None, "full": new(most, 2 * F), "8bit": new(2 * most, _ld(F), dtype=torch.uint8)}[c["keep"]]
    if c["op"] == "step" and c["keep"] == "8bit":
        s["x_kept"] = new(most, _ld(d), dtype=torch.uint8)
    if c["op"] == "backward":
        # pre-activations as wide as those of such rows, correlated with nothing
        pre = normal(most, 2 * F, scale=1.2)
        s["pre"] = pre.to(tt) if c["keep"] == "full" else _packed(pre.reshape(2 * most, F))
        s["x_kept"] = s["x"] if c["keep"] == "full" else _packed(s["x"].float())
    if c["op"] != "ffn":
        s["dy"] = normal(most, d, scale=1.0 / c["rows"]).to(tt)
        s["dx"], s["dW1"], s["dW2"] = new(most, d), torch.empty_like(s["W1"]), torch.empty_like(s["W2"])
    return s


# ---- plain form -----------------------------------------------------------------------------------


def _spread(s, rows):
    """Packed rows as one matrix of equal height for every expert that has any, in 32 bits."""
    out = torch.zeros(s["used"].shape[0] * s["most_of_one"], rows.shape[1], device=DEV)
    out[s["place"]] = rows[:s["K"]].float()
    return out.reshape(s["used"].shape[0], s["most_of_one"], -1)


def _gather(s, batch):
    return batch.reshape(-1, batch.shape[2])[s["place"]]


def _act(g, act):
    """The activation and its derivative."""
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (0.5 / math.pi) ** 0.5
    a, b = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(a * (g + b * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * a * (1 + 3 * b * g * g)


def _plain_forward(s, c):
    """y and the pre-activations of the packed rows, in 32 bits."""
    W1, W2 = s["W1"][s["used"]].float(), s["W2"][s["used"]].float()
    pre = torch.bmm(_spread(s, s["x"]), W1.transpose(1, 2))
    g, u = pre.chunk(2, 2)
    return _gather(s, torch.bmm(_act(g, c["act"])[0] * u, W2.transpose(1, 2))), _gather(s, pre)


def _plain_backward(s, c, x, pre):
    """dx of the packed rows, dW1 and dW2, in 32 bits."""
    W1, W2 = s["W1"][s["used"]].float(), s["W2"][s["used"]].float()
    x, dy = _spread(s, x), _spread(s, s["dy"])
    g, u = _spread(s, pre).chunk(2, 2)
    a, slope = _act(g, c["act"])
    dh = torch.bmm(dy, W2)
    dpre = torch.cat([dh * u * slope, dh * a], 2)
    dW1, dW2 = torch.zeros_like(s["W1"], dtype=torch.float32), torch.zeros_like(s["W2"], dtype=torch.float32)
    dW1[s["used"]] = torch.bmm(dpre.transpose(1, 2), x)
    dW2[s["used"]] = torch.bmm(dy.transpose(1, 2), a * u)
    return _gather(s, torch.bmm(dpre, W1)), dW1, dW2


def _plain(s):
    c = s["case"]
    tt, K, F = TYPES[c["dtype"]], s.get("K"), c["F"]
    if c["op"] == "checkpoint":
        return {"restored": _through_8_bits(s["x"].float()).to(tt)}
    out = {}
    if c["op"] != "backward":
        y, pre = _plain_forward(s, c)
        out["y"] = y.to(tt)
        if c["op"] == "ffn":
            return dict(out, pre=pre.to(tt)) if c["keep"] else out
        x = s["x"][:K].float()
        if c["keep"] == "8bit":
            x, pre = _through_8_bits(x), _through_8_bits(pre.reshape(2 * K, F)).reshape(K, 2 * F)
        else:
            pre = pre.to(tt)
    elif c["keep"] == "8bit":
        x, pre = _restored(s["x_kept"][:K], c["d"]), _restored(s["pre"][:2 * K], F).reshape(K, 2 * F)
    else:
        x, pre = s["x_kept"], s["pre"]
    dx, dW1, dW2 = _plain_backward(s, c, x, pre)
    return dict(out, dx=dx.to(tt), dW1=dW1.to(tt), dW2=dW2.to(tt))


# ---- the framework's calls ------------------------------------------------------------------------


def _own(s):
    from paper_2404_05019_amd import binding as B
    c = s["case"]
    if c["op"] == "checkpoint":
        B.scmoe_checkpoint_pack(s["x"], s["q"])
        B.scmoe_checkpoint_unpack(s["q"], s["restored"])
        return {"restored": s["restored"]}
    act = {"silu": B.SILU, "gelu": B.GELU_ERF, "gelu_tanh": B.GELU_TANH}[c["act"]]
    if "workspace" not in s:                  # kept from here on, as a program does
        code = B.dtype_code(s["x"])
        need = B.scmoe_gated_ffn_workspace_bytes(code, c["d"], c["F"])
        if c["op"] != "ffn":
            need = max(need, B.scmoe_gated_ffn_backward_workspace_bytes(code, s["rows"], s["E"], c["d"], c["F"]))
        s["workspace"] = torch.empty(max(16, need), dtype=torch.uint8, device=DEV)
    out, x, K = {}, s.get("x_kept", s["x"]), s["K"]
    if c["op"] != "backward":
        B.scmoe_gated_ffn(s["x"], s["offsets"], s["rows"], s["W1"], s["W2"], s["hidden"], s["y"], act, pre=s["pre"], workspace=s["workspace"])
        out["y"] = s["y"][:K]
        if c["op"] == "ffn":
            return dict(out, pre=s["pre"][:K]) if c["keep"] else out
        if c["keep"] == "8bit":
            B.scmoe_checkpoint_pack(s["x"], x, n_rows=s["offsets"][-1:])
    B.scmoe_gated_ffn_backward(s["dy"], x, s["pre"], s["offsets"], s["rows"], s["W1"], s["W2"], act, s["dx"], s["dW1"], s["dW2"],
                               workspace=s["workspace"])
    return dict(out, dx=s["dx"][:K], dW1=s["dW1"], dW2=s["dW2"])


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ----------------------------------------------------------------


def work(case):
    c = case
    b = 2 if c["dtype"] == "bf16" else 4
    n, d, F = c["rows"], c["d"], c["F"]
    if c["op"] == "checkpoint":
        return {"bytes": n * d * 2 * (b + 33 / 32), "flops": 4 * n * d}
    used = min(n, c["E"])
    weights, kept = 3 * used * d * F * b, {"": 0, "full": b, "8bit": 33 / 32}[c["keep"]]
    forward = {"bytes": 2 * n * d * b + weights + 2 * n * F * kept, "flops": 6 * n * d * F}
    if c["op"] == "ffn":
        return forward
    backward = {"bytes": 2 * n * d * b + n * d * kept + 2 * n * F * kept + weights + 3 * c["E"] * d * F * b, "flops": 12 * n * d * F}
    if c["op"] == "backward":
        return backward
    return {"bytes": forward["bytes"] + backward["bytes"] + (n * d * kept if kept < 2 else 0), "flops": forward["flops"] + backward["flops"]}


# ---- the definition in 64 bits --------------------------------------------------------------------


def _exact_8_bits(x):
    """Rows of 64-bit values as the checkpoint's rounding leaves them, from its definition: the least power of two s of at least 2^-126
    with max |x| <= 448 s for every 32 columns; x / s to three bits behind the leading one, or to multiples of 2^-9, ties to even."""
    out = torch.empty_like(x)
    for at in range(0, x.shape[1], BLOCK):
        v = x[:, at:at + BLOCK]
        top = v.abs().amax(1, keepdim=True)
        s = torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0)).clamp(-126, 127))
        s = torch.where(448.0 * s < top, 2 * s, s)
        s = torch.where((224.0 * s >= top) & (s > 2.0 ** -126), s / 2, s)
        z = v / s
        step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
        out[:, at:at + BLOCK] = torch.round(z / step) * step * s
    return out


def _exact_kept(q, w):
    """64-bit values of checkpoint rows, byte by byte from the format: sign, four bits of exponent (bias 7), three of mantissa."""
    b = q[:, :w].to(torch.int64)
    exponent, mantissa = b >> 3 & 15, (b & 7).double()
    v = torch.where(exponent == 0, mantissa * 2.0 ** -9, (8 + mantissa) * torch.exp2(exponent.double() - 10)) * (1 - 2 * (b >> 7)).double()
    scale = torch.exp2(q[:, w:w + -(-w // BLOCK)].double() - 127).repeat_interleave(BLOCK, 1)[:, :w]
    return v * scale


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "checkpoint":
        return {"restored": _exact_8_bits(s["x"].double())}
    F, K, tt = c["F"], s["K"], TYPES[c["dtype"]]
    ends = s["offsets"].tolist()
    forward, backward = c["op"] != "backward", c["op"] != "ffn"
    out = {}
    if forward:
        out["y"] = torch.empty(K, c["d"], dtype=torch.float64, device=DEV)
        if c["op"] == "ffn" and c["keep"]:
            out["pre"] = torch.empty(K, 2 * F, dtype=torch.float64, device=DEV)
    if backward:
        out["dx"] = torch.empty(K, c["d"], dtype=torch.float64, device=DEV)
        out["dW1"], out["dW2"] = torch.zeros_like(s["W1"], dtype=torch.float64), torch.zeros_like(s["W2"], dtype=torch.float64)
    for e in range(c["E"]):
        lo, hi = ends[e], ends[e + 1]
        if lo == hi:
            continue
        W1, W2 = s["W1"][e].double(), s["W2"][e].double()
        if forward:
            x = s["x"][lo:hi].double()
            pre = x @ W1.t()
        elif c["keep"] == "8bit":
            x, pre = _exact_kept(s["x_kept"][lo:hi], c["d"]), _exact_kept(s["pre"][2 * lo:2 * hi], F).reshape(hi - lo, 2 * F)
        else:
            x, pre = s["x_kept"][lo:hi].double(), s["pre"][lo:hi].double()
        if forward:
            g, u = pre[:, :F], pre[:, F:]
            a = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[c["act"]](g)
            out["y"][lo:hi] = (a * u) @ W2.t()
            if "pre" in out:
                out["pre"][lo:hi] = pre
            if c["keep"] == "8bit":
                x, pre = _exact_8_bits(x), _exact_8_bits(pre.reshape(-1, F)).reshape(hi - lo, 2 * F)
            elif c["keep"]:
                pre = pre.to(tt).double()
        if backward:
            # the gradient by the chain rule, the activation's slope by torch's own derivative in 64 bits
            g = pre[:, :F].clone().requires_grad_(True)
            u = pre[:, F:]
            a = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[c["act"]](g)
            dy = s["dy"][lo:hi].double()
            dh = dy @ W2
            dg = torch.autograd.grad(a, g, dh * u)[0]
            a = a.detach()
            out["dW2"][e] = dy.t() @ (a * u)
            both = torch.cat([dg, dh * a], 1)
            out["dW1"][e] = both.t() @ x
            out["dx"][lo:hi] = both @ W1
    return out
