"""8-bit products and the sorting of rows by adapter, as measurable cases.

A case is a plain dict.  Five kinds:

    linear    a projection with its weight in 8 bits: rows quantised per token, then the integer product, base_gemm_i8
    product   the integer product alone on rows that are sorted and quantised already, one matrix per group, gemm_i8
    experts   sort_tokens (quantised), gemm_i8 over the adapters' matrices, unsort_tokens with the gate's weights
    sort      sort_tokens: rows next to each other by adapter, and their positions
    unsort    unsort_tokens onto a base projection's output; train = True: the gradients of both directions instead,
              unsort_backward and unsort_tokens without weights (the gradient of sort_tokens)

Sizes are those of the repository's configurations (Llama3-8B and Llama2-13B layers, 28 adapters, top-2) and of its tests.
Activations are Gaussian with a few columns ten times as large, as the inputs of transformer layers are; weights are Gaussian,
quantised per output channel; routing is uniform or Zipf-like, with padding tokens (no adapter) where a batch is padded.
"""
import math

import torch

own = False   # True: the framework's operators instead of their plain forms

SCALE = 2.0
D, FFN = 4096, 14336


def _linear(name, T, d_in, d_out, dtype="bf16"):
    return {"name": name, "kind": "linear", "T": T, "d_in": d_in, "d_out": d_out, "dtype": dtype}


def _product(name, T, N, d_in, d_out, routing="uniform", dtype="bf16"):
    return {"name": name, "kind": "product", "T": T, "N": N, "d_in": d_in, "d_out": d_out, "routing": routing, "dtype": dtype}


def _experts(name, T, N, k, d_in, d_out, routing="uniform", padded=False):
    return {"name": name, "kind": "experts", "T": T, "N": N, "k": k, "d_in": d_in, "d_out": d_out, "routing": routing,
            "padded": padded, "dtype": "bf16"}


def _rows(name, kind, T, N, k, d, dtype="bf16", routing="uniform", padded=False, train=False):
    return {"name": name, "kind": kind, "T": T, "N": N, "k": k, "d": d, "dtype": dtype, "routing": routing, "padded": padded,
            "train": train}


def listed():
    return [
        # one sequence generating: the q projection of one new token, the weight streamed once
        _linear("linear_1_q", 1, D, D),
        # 64 sequences generating: a 13B-sized MLP projection
        _linear("linear_64_up", 64, 5120, 13824),
        # a short prompt or a chunk of one, ragged
        _linear("linear_300_q", 300, D, D),
        # 4 prompts of 1024 tokens
        _linear("linear_4096_q", 4096, D, D),
        # the widest MLP layer
        _linear("linear_8192_up", 8192, D, FFN),
        # the shrink of 28 adapters of rank 64 on 8192 sorted rows, skewed load, kept in fp32 for what follows
        _product("product_28_shrink", 8192, 28, D, 64, routing="zipf", dtype="f32"),
        # and their expand
        _product("product_28_expand", 8192, 28, 64, D, routing="zipf"),
        # full-rank adapters while 64 sequences generate: 16 rows each
        _experts("experts_64", 64, 8, 2, D, D),
        # and in a padded prompt batch of odd size
        _experts("experts_2001", 2001, 8, 2, D, D, routing="zipf", padded=True),
        # rows of 4 prompts by adapter
        _rows("sort_4096", "sort", 4096, 28, 2, D),
        # and back onto the base projection's output, a small fp32 batch as in configuration 1 but wider
        _rows("unsort_777_f32", "unsort", 777, 28, 2, 1024, dtype="f32", routing="zipf"),
        # gradients of both directions in training
        _rows("train_4096", "unsort", 4096, 28, 2, D, train=True),
    ]


_SHAPES = [(D, D), (D, 1024), (D, FFN), (FFN, D), (5120, 5120), (5120, 13824)]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _widths(rng):
    if rng.random() < 0.6:
        return rng.choice(_SHAPES)
    return 16 * _log_int(rng, 4, 896), 8 * _log_int(rng, 4, 1792)   # ragged


def draw(rng):
    kind = rng.choice(["linear"] * 4 + ["product"] * 2 + ["experts"] * 2 + ["sort"] * 2 + ["unsort"] * 2)
    routing = rng.choice(["uniform", "zipf"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind == "linear":
        d_in, d_out = _widths(rng)
        most = int(4.8e11 / (d_in * d_out))
        return {"kind": kind, "T": _log_int(rng, 1, min(8192, most)), "d_in": d_in, "d_out": d_out, "dtype": dtype}
    if kind == "product":
        N = rng.choice([1, 4, 7, 28, 64])
        d_in, d_out = _widths(rng)
        side = rng.choice(["shrink", "expand", "full"])
        if side == "shrink":
            d_out = rng.choice([8, 16, 32, 64])
        elif side == "expand":
            d_in = rng.choice([16, 32, 64])
        elif N > 8:
            d_in, d_out = 16 * _log_int(rng, 4, 128), 8 * _log_int(rng, 4, 256)
        most = int(min(4.8e11 / (d_in * d_out), 1.2e8 / max(d_in, d_out)))
        return {"kind": kind, "T": _log_int(rng, 1, min(16384, most)), "N": N, "d_in": d_in, "d_out": d_out,
                "routing": routing, "dtype": dtype}
    N = rng.choice([4, 7, 8]) if kind == "experts" else rng.choice([4, 7, 28, 64])
    k = rng.choice([1, 2, 2, 4, 8] if N >= 8 else [1, 2, 2, 4])
    padded = rng.random() < 0.3
    if kind == "experts":
        d_in, d_out = rng.choice([(D, D), (D, 1024), (5120, 5120), (16 * _log_int(rng, 4, 320), 8 * _log_int(rng, 4, 640))])
        return {"kind": kind, "T": _log_int(rng, 1, 4096), "N": N, "k": k, "d_in": d_in, "d_out": d_out, "routing": routing,
                "padded": padded, "dtype": "bf16"}
    d = rng.choice([D, 5120, 8 * _log_int(rng, 4, 1792)])
    return {"kind": kind, "T": _log_int(rng, 1, min(32768, int(1e8 / (d * k)))), "N": N, "k": k, "d": d, "dtype": dtype,
            "routing": routing, "padded": padded, "train": kind == "unsort" and rng.random() < 0.5}


# ---- inputs ---------------------------------------------------------------------------------------------------------------

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


class _Inputs:
    def __init__(self, case, seed):
        self.case = case
        self.dtype = _dtype(case)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(self, shape, std=1.0, dtype=None):
        v = torch.randn(shape, generator=self.gen, device="cuda", dtype=torch.float32)
        return v.mul_(std).to(dtype or self.dtype)

    def activations(self, T, d):
        x = torch.randn((T, d), generator=self.gen, device="cuda", dtype=torch.float32)
        wide = torch.rand(d, generator=self.gen, device="cuda") < 0.004
        return x.mul_(torch.where(wide, 10.0, 1.0)).to(self.dtype)

    def int8_rows(self, x):
        """8-bit rows and their scales, as a program has them in hand that loads quantised weights."""
        top = x.abs().amax(-1, keepdim=True)
        return torch.round(x * (127.0 / top)).to(torch.int8), (top[..., 0] / 127.0).contiguous()

    def weights(self, N, d_out, d_in):
        q = torch.empty((N, d_out, d_in), dtype=torch.int8, device="cuda")
        s = torch.empty((N, d_out), dtype=torch.float32, device="cuda")
        for e in range(N):
            q[e], s[e] = self.int8_rows(self.randn((d_out, d_in), d_in ** -0.5, torch.float32))
        return q, s

    def load(self, N):
        p = torch.ones(N, device="cuda")
        if self.case["routing"] == "zipf":
            p = 1.0 / torch.arange(1, N + 1, device="cuda", dtype=torch.float32) ** 2
        return torch.log(p)

    def routing(self, T, N, k):
        """k distinct adapters per token and weights that add up to one; padding tokens have the id -1."""
        u = torch.rand((T, N), generator=self.gen, device="cuda").clamp_(1e-9, 1 - 1e-7)
        score = self.load(N) - torch.log(-torch.log(u))
        idx = torch.topk(score, k, dim=1).indices.to(torch.int32)
        w = torch.softmax(self.randn((T, k), 1.0, torch.float32), 1)
        if self.case["padded"]:   # sequences of 128 tokens, the last ones of each are padding
            length = torch.randint(64, 129, ((T + 127) // 128,), generator=self.gen, device="cuda")
            at = torch.arange(T, device="cuda")
            idx[at % 128 >= length[at // 128]] = -1
        return idx.contiguous(), w.contiguous()


def prepare(case, seed):
    make = _Inputs(case, seed)
    kind, T, dt = case["kind"], case["T"], make.dtype
    state = {"case": case, "dtype": dt}
    if kind == "linear":
        state["x"] = make.activations(T, case["d_in"])
        q, s = make.weights(1, case["d_out"], case["d_in"])
        state["W"], state["w_scale"] = q[0], s[0]
        state["out"] = torch.empty((T, case["d_out"]), dtype=dt, device="cuda")
    elif kind == "product":
        N = case["N"]
        state["q"], state["q_scale"] = make.int8_rows(make.activations(T, case["d_in"]).float())
        state["W"], state["w_scale"] = make.weights(N, case["d_out"], case["d_in"])
        group = torch.multinomial(make.load(N).exp(), T, replacement=True, generator=make.gen)
        ends = torch.cumsum(torch.bincount(group, minlength=N), 0)
        state["offsets"] = torch.cat([ends.new_zeros(1), ends]).to(torch.int32)
        state["bounds"] = state["offsets"].tolist()
        state["out"] = torch.empty((T, case["d_out"]), dtype=dt, device="cuda")
    else:
        N, k = case["N"], case["k"]
        state["idx"], state["w"] = make.routing(T, N, k)
        if kind == "experts":
            state["x"] = make.activations(T, case["d_in"])
            state["W"], state["w_scale"] = make.weights(N, case["d_out"], case["d_in"])
            ends = torch.cumsum(torch.bincount(state["idx"][state["idx"] >= 0].flatten(), minlength=N), 0)
            state["bounds"] = [0] + ends.tolist()
            state["ys"] = torch.zeros((T * k, case["d_out"]), dtype=dt, device="cuda")
        elif kind == "sort":
            state["x"] = make.activations(T, case["d"])
            state["xs"] = torch.zeros((T * k, case["d"]), dtype=dt, device="cuda")   # rows behind the last one stay zero
        else:
            state["pos"] = _positions(state["idx"], N)[0]
            state["ys"] = make.randn((T * k, case["d"]))
            state["base"] = make.randn((T, case["d"]))   # the base projection's output, or the gradient of the sum
            state["out"] = torch.empty_like(state["base"])
            state["dys"] = torch.zeros_like(state["ys"])
    if own:
        import paper_2405_13053_amd as m
        if kind == "linear":
            state["ws"] = torch.empty(m.base_gemm_i8_workspace_bytes(T, case["d_in"]), dtype=torch.uint8, device="cuda")
        elif kind in ("experts", "sort"):
            state["ws"] = torch.empty(m.sort_workspace_bytes(T, case["k"], case["N"]), dtype=torch.uint8, device="cuda")
    return state


# ---- plain forms ----------------------------------------------------------------------------------------------------------

def _quantize(x):
    """Rows as whole numbers of -127 to 127 and their scales; the quotient in 64 bits, since halves are to be seen as such."""
    top = x.float().abs().amax(-1, keepdim=True)
    q = torch.round(x.double() * 127.0 / top.clamp_min(1e-45).double()).float()
    return q, top / 127.0


def _int_product(q, W):
    """q[T,K] * W[n,K]^T of whole numbers up to 127: 1024 products add up exactly in fp32, the rest in whole numbers."""
    total = torch.zeros((q.shape[0], W.shape[0]), dtype=torch.int32, device=q.device)
    for at in range(0, q.shape[1], 1024):
        total += (q[:, at:at + 1024].float() @ W[:, at:at + 1024].float().t()).to(torch.int32)
    return total


def _scaled_product(q, q_scale, W, w_scale, dtype):
    return (_int_product(q, W).float() * q_scale * w_scale).to(dtype)


def _positions(idx, N):
    """pos[T,k]: the place of every (token, slot) among all of them in order of adapter, then token, then slot; -1: none."""
    flat = idx.flatten().long()
    key = torch.where((flat >= 0) & (flat < N), flat, N)
    order = torch.argsort(key, stable=True)
    pos = torch.empty_like(order)
    pos[order] = torch.arange(order.numel(), device=idx.device)
    pos = torch.where(key < N, pos, -1).to(torch.int32).view_as(idx)
    counts = (key[:, None] == torch.arange(N, device=idx.device)).sum(0)
    offsets = torch.cat([counts.new_zeros(1), torch.cumsum(counts, 0)]).to(torch.int32)
    return pos, offsets


def _scatter_rows(rows, pos, k, total):
    """Row pos[t,j] of `total` zero rows = rows[t]; what goes nowhere is written behind the last one and cut off."""
    to = torch.where(pos < 0, total, pos).flatten().long()
    out = rows.new_zeros((total + 1, rows.shape[1]))
    out[to] = rows.repeat_interleave(k, 0)
    return out[:total]


def _gather_rows(rows, pos):
    """[T,k,d] in 32 bits, zeros where pos is -1."""
    return rows[pos.clamp_min(0).long()].float() * (pos >= 0)[..., None]


def _run_plain(state):
    case, dt = state["case"], state["dtype"]
    kind = case["kind"]
    if kind == "linear":
        q, s = _quantize(state["x"])
        return _scaled_product(q, s, state["W"], state["w_scale"], dt)
    if kind == "product":
        out = torch.empty_like(state["out"])
        for e, (a, b) in enumerate(zip(state["bounds"], state["bounds"][1:])):
            if b > a:
                out[a:b] = _scaled_product(state["q"][a:b], state["q_scale"][a:b, None], state["W"][e], state["w_scale"][e], dt)
        return out
    k = case["k"]
    if kind == "experts":
        pos, _ = _positions(state["idx"], case["N"])
        q, s = _quantize(state["x"])
        total = pos.numel()
        q, s = _scatter_rows(q, pos, k, total), _scatter_rows(s, pos, k, total)
        ys = torch.zeros_like(state["ys"])
        for e, (a, b) in enumerate(zip(state["bounds"], state["bounds"][1:])):
            if b > a:
                ys[a:b] = _scaled_product(q[a:b], s[a:b], state["W"][e], state["w_scale"][e], dt)
        return (SCALE * (_gather_rows(ys, pos) * state["w"][..., None]).sum(1)).to(dt)
    if kind == "sort":
        pos, offsets = _positions(state["idx"], case["N"])
        return {"xs": _scatter_rows(state["x"], pos, k, pos.numel()), "pos": pos, "offsets": offsets}
    pos, w, ys, base = state["pos"], state["w"], state["ys"], state["base"]
    if not case["train"]:
        return (base.float() + SCALE * (_gather_rows(ys, pos) * w[..., None]).sum(1)).to(dt)
    dy = base.float()
    dw = SCALE * (_gather_rows(ys, pos) * dy[:, None, :]).sum(-1)
    each = (SCALE * w[..., None] * dy[:, None, :]).to(dt).flatten(0, 1)
    to = torch.where(pos < 0, pos.numel(), pos).flatten().long()
    dys = each.new_zeros((pos.numel() + 1, each.shape[1]))
    dys[to] = each
    return {"dys": dys[:pos.numel()], "dw": dw, "dx": _gather_rows(ys, pos).sum(1).to(dt)}


def _run_own(state):
    import paper_2405_13053_amd as m
    case = state["case"]
    kind = case["kind"]
    if kind == "linear":
        return m.base_gemm_i8(state["x"], state["W"], state["w_scale"], out=state["out"], ws=state["ws"])
    if kind == "product":
        return m.gemm_i8(state["q"], state["q_scale"], state["W"], state["w_scale"], offsets=state["offsets"], out=state["out"])
    if kind == "experts":
        xs, xs_scale, pos, offsets = m.sort_tokens(state["x"], state["idx"], case["N"], quantize=True, ws=state["ws"])
        ys = m.gemm_i8(xs, xs_scale, state["W"], state["w_scale"], offsets=offsets, out=state["ys"])
        return m.unsort_tokens(ys, pos, state["w"], SCALE)
    if kind == "sort":
        xs, pos, offsets = m.sort_tokens(state["x"], state["idx"], case["N"], out=state["xs"], ws=state["ws"])
        return {"xs": xs, "pos": pos, "offsets": offsets}
    if not case["train"]:
        return m.unsort_tokens(state["ys"], state["pos"], state["w"], SCALE, base=state["base"], out=state["out"])
    dys, dw = m.unsort_backward(state["base"], state["ys"], state["pos"], state["w"], SCALE, out=state["dys"])
    # the rows' own gradient, here the same rows again
    return {"dys": dys, "dw": dw, "dx": m.unsort_tokens(state["ys"], state["pos"])}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    """Each input read once and each output written once; 8-bit weights of the groups that have rows, at most."""
    e = 4 if case["dtype"] == "f32" else 2
    kind, T = case["kind"], case["T"]
    if kind == "linear":
        K, n = case["d_in"], case["d_out"]
        return {"bytes": float(T * K * e + n * K + 4 * n + T * n * e), "flops": 2.0 * T * K * n}
    if kind == "product":
        K, n, used = case["d_in"], case["d_out"], min(case["N"], T)
        return {"bytes": float(T * K + 4 * T + used * n * (K + 4) + T * n * e), "flops": 2.0 * T * K * n}
    k = case["k"]
    if kind == "experts":
        K, n, used = case["d_in"], case["d_out"], min(case["N"], T * k)
        return {"bytes": float(T * K * e + 8 * T * k + used * n * (K + 4) + T * n * e), "flops": 2.0 * T * k * K * n}
    d = case["d"]
    if kind == "sort":
        return {"bytes": float(T * d * e * (1 + k) + 8 * T * k), "flops": float(T * k)}
    if case["train"]:   # dy, ys and w, pos in, dys and dw out; the rows' gradient in, dx out
        return {"bytes": float(T * d * e * (2 + 3 * k) + 16 * T * k), "flops": 4.0 * T * k * d}
    return {"bytes": float(T * d * e * (2 + k) + 8 * T * k), "flops": 2.0 * T * k * d}


# ---- the same from the definitions, in 64 bits ------------------------------------------------------------------------------

def _exact_rows(x):
    x = x.double()
    top = x.abs().max(1, keepdim=True).values
    step = torch.where(top > 0, top, torch.ones_like(top))
    q = (x * 127 / step)
    low = torch.floor(q)
    half = q - low
    up = (half > 0.5) | ((half == 0.5) & (torch.remainder(low, 2) == 1))
    return low + up.double(), top / 127


def _exact_order(idx, N):
    """[(token, slot)] of every adapter, one after the other, found by counting."""
    flat = idx.flatten().long()
    pos = torch.full_like(flat, -1)
    offsets, at = [0], 0
    for e in range(N):
        pairs = torch.nonzero(flat == e).flatten()
        pos[pairs] = at + torch.arange(pairs.numel(), device=idx.device)
        at += pairs.numel()
        offsets.append(at)
    return pos.view_as(idx), torch.tensor(offsets, device=idx.device)


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "linear":
        q, s = _exact_rows(state["x"])
        return torch.matmul(q, state["W"].double().t()) * s * state["w_scale"].double()
    if kind == "product":
        out = torch.zeros((case["T"], case["d_out"]), dtype=torch.float64, device="cuda")
        for e in range(case["N"]):
            a, b = state["bounds"][e], state["bounds"][e + 1]
            rows = state["q"][a:b].double() * state["q_scale"][a:b].double()[:, None]
            out[a:b] = torch.matmul(rows, (state["W"][e].double() * state["w_scale"][e].double()[:, None]).t())
        return out
    if kind == "experts":
        q, s = _exact_rows(state["x"])
        out = torch.zeros((case["T"], case["d_out"]), dtype=torch.float64, device="cuda")
        for e in range(case["N"]):
            share = (state["w"].double() * (state["idx"] == e)).sum(1)
            rows = torch.nonzero((state["idx"] == e).any(1)).flatten()
            y = torch.matmul(q[rows], state["W"][e].double().t()) * s[rows] * state["w_scale"][e].double()
            out[rows] += SCALE * share[rows, None] * y
        return out
    if kind == "sort":
        pos, offsets = _exact_order(state["idx"], case["N"])
        xs = torch.zeros(state["xs"].shape, dtype=torch.float64, device="cuda")
        for j in range(case["k"]):
            there = pos[:, j] >= 0
            xs[pos[there, j]] = state["x"][there].double()
        return {"xs": xs, "pos": pos.to(torch.int32), "offsets": offsets.to(torch.int32)}
    pos, w, ys, base = state["pos"].long(), state["w"].double(), state["ys"].double(), state["base"].double()
    total = torch.zeros_like(base) if case["train"] else base.clone()
    dys, dw = torch.zeros_like(ys), torch.zeros_like(w)
    for j in range(case["k"]):
        there = pos[:, j] >= 0
        at = pos[there, j]
        if case["train"]:
            total[there] += ys[at]
            dys[at] = SCALE * w[there, j, None] * base[there]
            dw[there, j] = SCALE * (base[there] * ys[at]).sum(1)
        else:
            total[there] += SCALE * w[there, j, None] * ys[at]
    return {"dys": dys, "dw": dw, "dx": total} if case["train"] else total
