"""4-bit products with block scales and mixture-of-experts layers of few tokens, as measurable cases.

A case is a plain dict.  Five kinds:

    rows      rows into 4 bits and back, quantize_mx4 and dequantize_mx4
    linear    a projection with its weight in 4 bits: rows quantised per block, then the product, base_gemm_mx4;
              train = True: its gradient with respect to the rows as well, base_gemm_mx4_backward
    product   the product alone on rows that are sorted and quantised already, one matrix per group, gemm_mx4
    moe       gate, gated MLPs of the selected experts and their weighted sum for a few tokens, moe_forward;
              weights in 4 bits or bf16
    experts   the same with the routing given, onto a residual stream, experts_forward

The 4-bit format: values 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives (E2M1), a power of two for every 32 consecutive
inputs of a row (E8M0: the byte E stands for 2^(E - 127)).  Sizes are those of the repository's configurations (Llama3-8B and
Llama2-13B layers, 28 adapters, top-2) and of its tests, or generic.  Activations are Gaussian with a few columns ten times as
large, as the inputs of transformer layers are; weights are Gaussian; routing is uniform or Zipf-like.
"""
import math

import torch

own = False   # True: the framework's operators instead of their plain forms

SCALE = 2.0
D, FFN = 4096, 14336


def _rows(name, T, d, dtype="bf16"):
    return {"name": name, "kind": "rows", "T": T, "d": d, "dtype": dtype}


def _linear(name, T, d_in, d_out, dtype="bf16", train=False):
    return {"name": name, "kind": "linear", "T": T, "d_in": d_in, "d_out": d_out, "dtype": dtype, "train": train}


def _product(name, T, N, d_in, d_out, routing="uniform", dtype="bf16"):
    return {"name": name, "kind": "product", "T": T, "N": N, "d_in": d_in, "d_out": d_out, "routing": routing, "dtype": dtype}


def _moe(name, T, N, k, d, f, weights, routing="uniform", kind="moe"):
    return {"name": name, "kind": kind, "T": T, "N": N, "k": k, "d": d, "f": f, "weights": weights, "routing": routing,
            "padded": False, "dtype": "bf16"}


def listed():
    return [
        # activations of 4 prompts kept in 4 bits between a forward and a backward pass
        _rows("rows_4096", 4096, D),
        # one sequence generating: the q projection of one new token
        _linear("linear_1_q", 1, D, D),
        # 64 sequences generating: a 13B-sized MLP projection
        _linear("linear_64_up", 64, 5120, 13824),
        # a short prompt or a chunk of one, ragged
        _linear("linear_300_q", 300, D, D),
        # the widest MLP layer on 8 prompts of 1024 tokens
        _linear("linear_8192_up", 8192, D, FFN),
        # adapters trained on a frozen 4-bit projection: forward, and the gradient that the layers in front need
        _linear("train_4096_q", 4096, D, D, train=True),
        # full-rank adapters on sorted rows of odd number, skewed load
        _product("product_8_2001", 2001, 8, D, D, routing="zipf"),
        # one sequence generating through experts of the size of the widest MLP
        _moe("moe_1", 1, 8, 2, D, FFN, "mx4"),
        # and through many small ones, where launches count
        _moe("moe_1_small_bf16", 1, 28, 4, 1024, 512, "bf16"),
        # 64 sequences generating, every expert in use
        _moe("moe_64", 64, 8, 2, D, FFN, "mx4"),
        # an odd number of sequences, bf16 experts
        _moe("moe_13_bf16", 13, 8, 2, D, 3584, "bf16", routing="zipf"),
        # drafted tokens of a few sequences, routing known, onto the residual stream; odd widths
        _moe("experts_33", 33, 28, 4, 2080, 1376, "mx4", kind="experts"),
    ]


_SHAPES = [(D, D), (D, 1024), (D, FFN), (FFN, D), (5120, 5120), (5120, 13824)]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _widths(rng):
    if rng.random() < 0.6:
        return rng.choice(_SHAPES)
    return 32 * _log_int(rng, 2, 448), 8 * _log_int(rng, 4, 1792)   # ragged


def draw(rng):
    kind = rng.choice(["rows"] + ["linear"] * 5 + ["product"] * 2 + ["moe"] * 4 + ["experts"] * 2)
    routing = rng.choice(["uniform", "zipf"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if kind == "rows":
        d = rng.choice([D, 5120, 32 * _log_int(rng, 1, 448)])
        return {"kind": kind, "T": _log_int(rng, 1, min(32768, int(1e8 / d))), "d": d, "dtype": dtype}
    if kind == "linear":
        d_in, d_out = _widths(rng)
        train = rng.random() < 0.25
        most = int((1.5e11 if train else 4.8e11) / (d_in * d_out) * (0.1 if train and dtype == "f32" else 1.0))
        return {"kind": kind, "T": _log_int(rng, 1, max(1, min(8192, most))), "d_in": d_in, "d_out": d_out, "dtype": dtype,
                "train": train}
    if kind == "product":
        N = rng.choice([1, 4, 7, 28, 64])
        d_in, d_out = _widths(rng)
        side = rng.choice(["shrink", "expand", "full", "full"])
        if side == "shrink":
            d_out = rng.choice([8, 16, 32, 64])
        elif side == "expand":
            d_in = rng.choice([32, 64])
        elif N > 8:
            d_in, d_out = 32 * _log_int(rng, 2, 64), 8 * _log_int(rng, 4, 256)
        most = int(min(4.8e11 / (d_in * d_out), 1.2e8 / max(d_in, d_out)))
        return {"kind": kind, "T": _log_int(rng, 1, min(16384, most)), "N": N, "d_in": d_in, "d_out": d_out,
                "routing": routing, "dtype": dtype}
    N = rng.choice([4, 7, 8, 8, 16, 28, 64])
    k = rng.choice([1, 2, 2, 4, 8] if N >= 8 else [1, 2, 2, 4])
    weights = rng.choice(["mx4", "mx4", "bf16"])
    unit = 32 if weights == "mx4" else 8
    most = int((1.2e9 if weights == "mx4" else 3e8) / (3 * N))   # d * f
    d = rng.choice([1024, D, unit * _log_int(rng, 512 // unit, 5120 // unit)])
    f = unit * _log_int(rng, 256 // unit, max(512, min(FFN, most // d)) // unit)
    return {"kind": kind, "T": rng.choice([1, 1, _log_int(rng, 1, 64), rng.randint(2, 64)]), "N": N, "k": k, "d": d, "f": f,
            "weights": weights, "routing": routing, "padded": kind == "experts" and rng.random() < 0.3, "dtype": "bf16"}


# ---- the 4-bit format -------------------------------------------------------------------------------------------------------

_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
# |t| up to which the values in front of each one are nearer: halfway, and a value with an odd code loses a tie
_ABOVE = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))


def _quantize(x):
    """(codes 0..15, bytes E) of rows: E = floor(log2(max |x|)) - 2 + 127 of every 32, at least 0; the quotient rounded to the nearest
    value, ties to the even code, at most 6.  x * 2^-e is exact in 32 bits."""
    blocks = x.float().unflatten(-1, (-1, 32))
    top = blocks.abs().amax(-1)
    _, e = torch.frexp(top)   # top = m 2^e, 0.5 <= m < 1
    E = torch.where(top > 0, (e.to(torch.int32) - 1 - 2 + 127).clamp_min(0), torch.zeros_like(e, dtype=torch.int32))
    t = blocks * torch.exp2((127 - E).float())[..., None]
    code = torch.zeros_like(t, dtype=torch.uint8)
    for border, reaches in _ABOVE:
        code += (t.abs() >= border) if reaches else (t.abs() > border)
    code += 8 * (t < 0).to(torch.uint8) * (code > 0)
    return code.flatten(-2), E.to(torch.uint8)


def _pack(code, E):
    """As the operators take them: two codes a byte, the first one low; scales[ceil(d / 512)][rows][16], that of block b in
    [b / 16][row][(b % 4) * 4 + b % 16 / 4]; zeros behind the last."""
    q = code[..., 0::2] | (code[..., 1::2] << 4)
    rows, blocks = E.shape[-2:]
    chunks = (blocks + 15) // 16
    s = torch.zeros((rows, chunks * 16), dtype=torch.uint8, device=E.device)
    s[:, :blocks] = E
    s = s.view(rows, chunks, 4, 4).transpose(-1, -2).reshape(rows, chunks, 16).transpose(0, 1)
    return q.contiguous(), s.contiguous()


def _unpack(q, scale):
    """[rows, d] in 32 bits."""
    table = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device=q.device)
    v = torch.stack([table[(q & 15).long()], table[(q >> 4).long()]], -1).flatten(-2)
    chunks, rows, _ = scale.shape
    E = scale.view(chunks, rows, 4, 4).transpose(-1, -2).reshape(chunks, rows, 16).transpose(0, 1).reshape(rows, chunks * 16)
    E = E[:, :v.shape[-1] // 32]
    return (v.unflatten(-1, (-1, 32)) * torch.exp2(E.float() - 127)[..., None]).flatten(-2)


# ---- inputs -----------------------------------------------------------------------------------------------------------------

class _Inputs:
    def __init__(self, case, seed):
        self.case = case
        self.dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        self.gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(self, shape, std=1.0, dtype=None):
        v = torch.randn(shape, generator=self.gen, device="cuda", dtype=torch.float32)
        return v.mul_(std).to(dtype or self.dtype)

    def activations(self, T, d):
        x = torch.randn((T, d), generator=self.gen, device="cuda", dtype=torch.float32)
        wide = torch.rand(d, generator=self.gen, device="cuda") < 0.004
        return x.mul_(torch.where(wide, 10.0, 1.0)).to(self.dtype)

    def weights(self, N, n, d, mx4=True):
        """(W, scales) of N matrices with n rows of d inputs; bf16 ones have no scales."""
        if not mx4:
            W = torch.empty((N, n, d), dtype=torch.bfloat16, device="cuda")
            for e in range(N):
                W[e] = self.randn((n, d), d ** -0.5, torch.bfloat16)
            return W, None
        W = torch.empty((N, n, d // 2), dtype=torch.uint8, device="cuda")
        s = torch.empty((N, (d + 511) // 512, n, 16), dtype=torch.uint8, device="cuda")
        for e in range(N):
            W[e], s[e] = _pack(*_quantize(self.randn((n, d), d ** -0.5, torch.float32)))
        return W, s

    def load(self, N):
        p = torch.ones(N, device="cuda")
        if self.case["routing"] == "zipf":
            p = 1.0 / torch.arange(1, N + 1, device="cuda", dtype=torch.float32) ** 2
        return torch.log(p)


def prepare(case, seed):
    make = _Inputs(case, seed)
    kind, T, dt = case["kind"], case["T"], make.dtype
    state = {"case": case, "dtype": dt}
    if kind == "rows":
        state["x"] = make.activations(T, case["d"])
        state["out"] = torch.empty_like(state["x"])
    elif kind == "linear":
        state["x"] = make.activations(T, case["d_in"])
        W, s = make.weights(1, case["d_out"], case["d_in"])
        state["W"], state["w_scale"] = W[0], s[0]
        state["out"] = torch.empty((T, case["d_out"]), dtype=dt, device="cuda")
        if case["train"]:
            state["dy"] = make.randn((T, case["d_out"]))
            state["dx"] = torch.empty_like(state["x"])
    elif kind == "product":
        N = case["N"]
        state["q"], state["q_scale"] = _pack(*_quantize(make.activations(T, case["d_in"])))
        state["W"], state["w_scale"] = make.weights(N, case["d_out"], case["d_in"])
        group = torch.multinomial(make.load(N).exp(), T, replacement=True, generator=make.gen)
        ends = torch.cumsum(torch.bincount(group, minlength=N), 0)
        state["offsets"] = torch.cat([ends.new_zeros(1), ends]).to(torch.int32)
        state["bounds"] = state["offsets"].tolist()
        state["out"] = torch.empty((T, case["d_out"]), dtype=dt, device="cuda")
    else:
        N, k, d, f, mx4 = case["N"], case["k"], case["d"], case["f"], case["weights"] == "mx4"
        state["x"] = make.activations(T, d)
        state["W1"], state["s1"] = make.weights(N, 2 * f, d, mx4)
        state["W2"], state["s2"] = make.weights(N, d, f, mx4)
        state["out"] = torch.empty((T, d), dtype=dt, device="cuda")
        if kind == "moe":
            state["W_gate"] = make.randn((d, N), d ** -0.5, torch.float32)
            state["bias"] = make.load(N)
        else:
            u = torch.rand((T, N), generator=make.gen, device="cuda").clamp_(1e-9, 1 - 1e-7)
            idx = torch.topk(make.load(N) - torch.log(-torch.log(u)), k, dim=1).indices.to(torch.int32)
            if case["padded"]:   # sequences that have ended keep their place in the batch
                idx[torch.rand(T, generator=make.gen, device="cuda") < 0.3] = -1
            state["idx"] = idx.contiguous()
            state["w"] = torch.softmax(make.randn((T, k), 1.0, torch.float32), 1).contiguous()
            state["base"] = make.randn((T, d))
    if own:
        import paper_2405_13053_amd as m
        if kind == "linear":
            n = m.base_gemm_mx4_workspace_bytes(T, case["d_in"])
            state["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
            if case["train"]:
                n = m.base_gemm_mx4_backward_workspace_bytes(case["d_in"], case["d_out"], dt)
                state["ws_back"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        elif kind in ("moe", "experts"):
            n = m.experts_workspace_bytes(T, case["d"], case["f"], case["N"], case["k"])
            state["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return state


# ---- plain forms ------------------------------------------------------------------------------------------------------------

def _rounded(x):
    return _unpack(*_pack(*_quantize(x)))


def _weight(state, name, e):
    s = state["s" + name]
    return state["W" + name][e].float() if s is None else _unpack(state["W" + name][e], s[e])


def _routing(state):
    """(ids, weights): the k largest logits, equal ones by their index, and their softmax."""
    case = state["case"]
    if case["kind"] == "experts":
        return state["idx"].long(), state["w"]
    logits = state["x"].float() @ state["W_gate"] + state["bias"]
    top, idx = torch.sort(logits, dim=1, descending=True, stable=True)
    top, idx = top[:, :case["k"]], idx[:, :case["k"]]
    w = torch.exp(top - top[:, :1])
    return idx, w / w.sum(1, keepdim=True)


def _run_plain(state):
    case, dt = state["case"], state["dtype"]
    kind = case["kind"]
    if kind == "rows":
        return _rounded(state["x"]).to(dt)
    if kind == "linear":
        V = _unpack(state["W"], state["w_scale"])
        y = (_rounded(state["x"]) @ V.t()).to(dt)
        return {"y": y, "dx": (state["dy"].float() @ V).to(dt)} if case["train"] else y
    if kind == "product":
        rows = _unpack(state["q"], state["q_scale"])
        out = torch.empty_like(state["out"])
        for e, (a, b) in enumerate(zip(state["bounds"], state["bounds"][1:])):
            if b > a:
                out[a:b] = (rows[a:b] @ _unpack(state["W"][e], state["w_scale"][e]).t()).to(dt)
        return out
    idx, w = _routing(state)
    f = case["f"]
    total = torch.zeros((case["T"], case["d"]), device="cuda")
    for e in range(case["N"]):
        share = (w * (idx == e)).sum(1)
        rows = (idx == e).any(1).nonzero().flatten()
        if rows.numel() == 0:
            continue
        both = state["x"][rows].float() @ _weight(state, "1", e).t()
        g, u = both[:, :f], both[:, f:]
        h = g / (1 + torch.exp(-g)) * u
        total[rows] += share[rows, None] * (h @ _weight(state, "2", e).t())
    if kind == "experts":
        total = state["base"].float() + SCALE * total
    return total.to(dt)


def _run_own(state):
    import paper_2405_13053_amd as m
    case = state["case"]
    kind = case["kind"]
    if kind == "rows":
        q, scale = m.quantize_mx4(state["x"])
        return m.dequantize_mx4(q, scale, out=state["out"])
    if kind == "linear":
        y = m.base_gemm_mx4(state["x"], state["W"], state["w_scale"], out=state["out"], ws=state["ws"])
        if not case["train"]:
            return y
        dx = m.base_gemm_mx4_backward(state["dy"], state["W"], state["w_scale"], out=state["dx"], ws=state["ws_back"])
        return {"y": y, "dx": dx}
    if kind == "product":
        return m.gemm_mx4(state["q"], state["q_scale"], state["W"], state["w_scale"], offsets=state["offsets"], out=state["out"])
    if kind == "moe":
        return m.moe_forward(state["x"], state["W_gate"], state["bias"], state["W1"], state["W2"], case["k"],
                             w1_scale=state["s1"], w2_scale=state["s2"], out=state["out"], ws=state["ws"])
    return m.experts_forward(state["x"], state["idx"], state["w"], state["W1"], state["W2"], w1_scale=state["s1"],
                             w2_scale=state["s2"], scale=SCALE, base=state["base"], out=state["out"], ws=state["ws"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    """Each input read once and each output written once; of the experts and groups those that can have rows."""
    e = 4 if case["dtype"] == "f32" else 2
    four = 0.5 + 1 / 32   # bytes of a 4-bit value and its share of a scale
    kind, T = case["kind"], case["T"]
    if kind == "rows":
        return {"bytes": T * case["d"] * (2 * e + 2 * four), "flops": 4.0 * T * case["d"]}
    if kind == "linear":
        K, n = case["d_in"], case["d_out"]
        both = 2 if case["train"] else 1
        return {"bytes": both * float(T * K * e + T * n * e) + n * K * four, "flops": both * 2.0 * T * K * n}
    if kind == "product":
        K, n, used = case["d_in"], case["d_out"], min(case["N"], T)
        return {"bytes": T * K * four + used * n * K * four + float(T * n * e), "flops": 2.0 * T * K * n}
    N, k, d, f = case["N"], case["k"], case["d"], case["f"]
    # experts that T tokens can be expected to reach, at equal chances
    used = N * (1 - (1 - k / N) ** T)
    size = four if case["weights"] == "mx4" else 2
    extra = 4.0 * d * N if kind == "moe" else 2.0 * T * d + 8.0 * T * k
    return {"bytes": used * 3 * d * f * size + 4.0 * T * d + extra, "flops": 6.0 * T * k * d * f}


# ---- the same from the definitions, in 64 bits --------------------------------------------------------------------------------

def _exact_rows(x):
    """The nearest of the 15 values to the quotient, by distance; of two as near the one whose code is even."""
    b = x.double().unflatten(-1, (-1, 32))
    top = b.abs().max(-1, keepdim=True).values
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(top.clamp_min(1e-300))) - 2, min=-127))
    t = (b / step).clamp(-6, 6)
    best, value = torch.full_like(t, math.inf), torch.zeros_like(t)
    for v in (0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0):   # the even codes first: a tie stays with them
        away = (t.abs() - v).abs()
        value = torch.where(away < best, torch.full_like(t, v), value)
        best = torch.minimum(away, best)
    return (value * torch.sign(t) * step).flatten(-2)


def _exact_values(q, scale):
    d = q.shape[1] * 2
    out = torch.empty((q.shape[0], d), dtype=torch.float64, device=q.device)
    code = torch.empty((q.shape[0], d), dtype=torch.int64, device=q.device)
    code[:, 0::2], code[:, 1::2] = (q % 16).long(), torch.div(q, 16, rounding_mode="floor").long()
    m = code % 8
    size = torch.where(m < 2, 0.5 * m, (1 + 0.5 * (m % 2)) * torch.exp2((m // 2 - 1).double()))
    signed = torch.where(code >= 8, -size, size)
    for b in range(d // 32):
        E = scale[b // 16, :, (b % 4) * 4 + (b % 16) // 4].double()
        out[:, b * 32:(b + 1) * 32] = signed[:, b * 32:(b + 1) * 32] * torch.exp2(E - 127)[:, None]
    return out


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "rows":
        return _exact_rows(state["x"])
    if kind == "linear":
        V = _exact_values(state["W"], state["w_scale"])
        y = torch.matmul(_exact_rows(state["x"]), V.t())
        return {"y": y, "dx": torch.matmul(state["dy"].double(), V)} if case["train"] else y
    if kind == "product":
        rows = _exact_values(state["q"], state["q_scale"])
        out = torch.zeros((case["T"], case["d_out"]), dtype=torch.float64, device="cuda")
        for e in range(case["N"]):
            a, b = state["bounds"][e], state["bounds"][e + 1]
            out[a:b] = torch.matmul(rows[a:b], _exact_values(state["W"][e], state["w_scale"][e]).t())
        return out
    T, N, k, f = case["T"], case["N"], case["k"], case["f"]
    x = state["x"].double()
    share = torch.zeros((T, N), dtype=torch.float64, device="cuda")
    if kind == "moe":
        logits = torch.matmul(x, state["W_gate"].double()) + state["bias"].double()
        left = logits.clone()
        for _ in range(k):
            best = left.argmax(1)   # no two logits are equal
            share[torch.arange(T, device="cuda"), best] = 1.0
            left[torch.arange(T, device="cuda"), best] = -math.inf
        share = torch.softmax(torch.where(share > 0, logits, torch.full_like(logits, -math.inf)), 1)
    else:
        for j in range(k):
            there = state["idx"][:, j] >= 0
            share[there, state["idx"][there, j].long()] += state["w"][there, j].double()
    out = torch.zeros((T, case["d"]), dtype=torch.float64, device="cuda")
    for e in range(N):
        rows = torch.nonzero(share[:, e]).flatten()
        if rows.numel() == 0:
            continue
        W1 = state["W1"][e].double() if state["s1"] is None else _exact_values(state["W1"][e], state["s1"][e])
        both = torch.matmul(x[rows], W1.t())
        h = torch.sigmoid(both[:, :f]) * both[:, :f] * both[:, f:]
        W2 = state["W2"][e].double() if state["s2"] is None else _exact_values(state["W2"][e], state["s2"][e])
        out[rows] += share[rows, e, None] * torch.matmul(h, W2.t())
    return state["base"].double() + SCALE * out if kind == "experts" else out
