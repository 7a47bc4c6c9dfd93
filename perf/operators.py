"""Timed cases of the operators around a ternary projection in a transformer: layer norm, forward and
backward, layer norm straight to int8 codes, and the projection with low-rank adapters of many requests.

Each case is one call.  ``run`` computes it either from elementary torch operations (``own`` false) or
through the library (``own`` true).  Sizes are token counts from a single decoded one to a prefill of
thousands, widths of the repository's own layers (96 to 1280 channels) and the usual powers of two up
to the library's limit of 4096 channels, and odd ones.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
#: channel counts of the repository's layers and generic ones
WIDTHS = (96, 144, 160, 192, 320, 384, 576, 768, 960, 1024, 1280, 1536, 2048, 2560, 4096)
MOST_VALUES = 16384 * 4096          # of a normed matrix
MOST_PRODUCTS = 8192 * 4096 * 4096  # of a projection


def listed():
    return [
        # Forward pass in training, statistics kept for the backward pass.
        {"name": "norm_16384x4096_bf16", "kind": "norm", "m": 16384, "n": 4096, "pitch": 4096, "type": "bf16", "params": "f32"},
        # Channels-last norm of a feature map (batch 32 at 28 x 28, 192 channels), float activations.
        {"name": "norm_25088x192_f32", "kind": "norm", "m": 25088, "n": 192, "pitch": 192, "type": "f32", "params": "f32"},
        # One decoded token on its way to a projection: what a call costs.
        {"name": "norm_i8_1x2048_bf16", "kind": "norm_i8", "m": 1, "n": 2048, "pitch": 2048, "type": "bf16", "params": "bf16"},
        # A prefill's tokens to codes; the rows are a slice of a wider buffer.
        {"name": "norm_i8_8192x4096_bf16", "kind": "norm_i8", "m": 8192, "n": 4096, "pitch": 4224, "type": "bf16", "params": "f32"},
        # Backward pass of the large training step.
        {"name": "norm_backward_16384x4096_bf16", "kind": "norm_backward", "m": 16384, "n": 4096, "pitch": 4096, "type": "bf16", "params": "f32"},
        # Float gradients over 960 channels (batch 128 at 14 x 14).
        {"name": "norm_backward_25088x960_f32", "kind": "norm_backward", "m": 25088, "n": 960, "pitch": 960, "type": "f32", "params": "f32"},
        # A ragged batch and an odd width: no row but the first starts on a 16-byte boundary.
        {"name": "norm_backward_777x1283_f16", "kind": "norm_backward", "m": 777, "n": 1283, "pitch": 1283, "type": "f16", "params": "f16"},
        # One decoded token of one request.
        {"name": "adapters_1_2048x2048", "kind": "adapters", "batch": 1, "rows": 1, "cin": 2048, "cout": 2048, "pitch": 2048,
         "adapters": 8, "rank": 16, "type": "bf16", "out": "bf16", "own_share": 1.0},
        # A decoding step of 32 requests, nearly each with an adapter of its own.
        {"name": "adapters_32_4096x4096", "kind": "adapters", "batch": 32, "rows": 1, "cin": 4096, "cout": 4096, "pitch": 4096,
         "adapters": 64, "rank": 16, "type": "bf16", "out": "bf16", "own_share": 0.9},
        # A short mixed batch on one of the network's layers, half of the rows without an adapter.
        {"name": "adapters_205_960x1280", "kind": "adapters", "batch": 205, "rows": 1, "cin": 960, "cout": 1280, "pitch": 1280,
         "adapters": 5, "rank": 8, "type": "f16", "out": "f16", "own_share": 0.5},
        # Images of 14 x 14 positions, each with its adapter, float outputs.
        {"name": "adapters_64x196_384x576_f32", "kind": "adapters", "batch": 64, "rows": 196, "cin": 384, "cout": 576, "pitch": 576,
         "adapters": 12, "rank": 4, "type": "bf16", "out": "f32", "own_share": 0.8},
        # Prefill of several requests, into a slice of a wider output (a fused projection's).
        {"name": "adapters_8192_4096x4096", "kind": "adapters", "batch": 8192, "rows": 1, "cin": 4096, "cout": 4096, "pitch": 6144,
         "adapters": 16, "rank": 64, "type": "bf16", "out": "bf16", "own_share": 0.9},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "norm_i8", "norm_backward", "adapters", "adapters", "adapters"))
    if kind != "adapters":
        n = rng.choice(WIDTHS) if rng.random() < 0.5 else _log_int(rng, 32, 8192)
        m = _log_int(rng, 1, min(100352, MOST_VALUES // n))
        pitch = n + (rng.choice((1, 8, 24, 128)) if rng.random() < 0.25 else 0)
        kept = rng.choice(("f32", "bf16", "f16"))
        return {"kind": kind, "m": m, "n": n, "pitch": pitch, "type": kept, "params": rng.choice(("f32", kept))}
    cin = rng.choice([w for w in WIDTHS if w % 16 == 0]) if rng.random() < 0.6 else 16 * _log_int(rng, 1, 256)
    cout = rng.choice(WIDTHS) if rng.random() < 0.6 else 8 * _log_int(rng, 1, 512)
    rows = rng.choice((1, 1, 1, 49, 196))
    batch = _log_int(rng, 1, max(1, min(16384, MOST_PRODUCTS // (cin * cout)) // rows))
    kept = rng.choice(("bf16", "f16"))
    return {"kind": "adapters", "batch": batch, "rows": rows, "cin": cin, "cout": cout,
            "pitch": cout + (rng.choice((8, 64, 128)) if rng.random() < 0.25 else 0),
            "adapters": _log_int(rng, 1, 48), "rank": rng.choice((1, 4, 8, 12, 16, 24, 32, 64)), "type": kept,
            "out": rng.choice(("f32", kept)), "own_share": rng.choice((0.0, 0.5, 0.9, 1.0))}


_BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def work(case):
    if case["kind"] == "adapters":
        m, k, n, r = case["batch"] * case["rows"], case["cin"], case["cout"], case["rank"]
        used = min(case["adapters"], case["batch"]) if case["own_share"] > 0 else 0
        with_one = m * case["own_share"]
        return {"bytes": m * k + k * n // 4 + 4 * n + 8 * case["batch"] + 2 * used * r * (k + n) + _BYTES[case["out"]] * m * n,
                "flops": 2 * m * k * n + 2 * with_one * r * (k + n)}
    m, n, e, p = case["m"], case["n"], _BYTES[case["type"]], _BYTES[case["params"]]
    if case["kind"] == "norm":
        return {"bytes": 2 * m * n * e + 2 * n * p + 8 * m, "flops": 8 * m * n}
    if case["kind"] == "norm_i8":
        return {"bytes": m * n * (e + 1) + 2 * n * p + 8 * m, "flops": 12 * m * n}
    return {"bytes": 3 * m * n * e + 3 * n * p + 8 * m, "flops": 14 * m * n}


# ---- inputs -------------------------------------------------------------------------------------

class _Source:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda")

    def ints(self, lo, hi, shape, dtype):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda", dtype=dtype)


def _matrix(values, pitch, dtype):
    """`values` in `dtype`, as the first columns of a buffer whose rows are `pitch` values apart."""
    m, n = values.shape
    if pitch == n:
        return values.to(dtype)
    buf = torch.zeros((m, pitch), dtype=dtype, device="cuda")
    buf[:, :n] = values
    return buf[:, :n]


def _prepare_norm(case, src):
    m, n, kept, params = case["m"], case["n"], TYPES[case["type"]], TYPES[case["params"]]
    # rows of a residual stream: each with a scale and an offset of its own
    x = src.normal(m, n).mul_(src.normal(m, 1).exp_()).add_(src.normal(m, 1).mul_(0.3))
    s = dict(x=_matrix(x, case["pitch"], kept), weight=src.normal(n).mul_(0.1).add_(1.0).to(params),
             bias=src.normal(n).mul_(0.1).to(params))
    if case["kind"] == "norm_backward":
        s["dy"] = _matrix(src.normal(m, n).mul_(0.1), case["pitch"], kept)
        xf = s["x"].double()
        s["mean"] = xf.mean(1).float()
        s["rstd"] = (xf.var(1, unbiased=False) + EPS).rsqrt().float()
        s["out"] = (torch.empty((m, n), dtype=kept, device="cuda"), torch.empty(n, dtype=params, device="cuda"),
                    torch.empty(n, dtype=params, device="cuda"))
    elif case["kind"] == "norm":
        s["out"] = (torch.empty((m, n), dtype=kept, device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, device="cuda"))
    else:
        s["out"] = (torch.empty((m, n), dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, device="cuda"))
    return s


def _prepare_adapters(case, src):
    b, m, k, n, r, na = case["batch"], case["batch"] * case["rows"], case["cin"], case["cout"], case["rank"], case["adapters"]
    kept = TYPES[case["type"]]
    codes = src.ints(0, 2, (n, k), torch.int8) - src.ints(0, 2, (n, k), torch.int8)      # half of them zero
    c = (codes & 3).view(n, k // 4, 4).to(torch.uint8)
    packed = c[..., 0] | (c[..., 1] << 2) | (c[..., 2] << 4) | (c[..., 3] << 6)
    # requests stand one after the other: short runs of samples with the same adapter, some without one
    runs = src.ints(0, na, (b,), torch.int32)
    runs = runs[torch.arange(b, device="cuda") // max(1, b // (2 * na))]
    runs = torch.where(torch.rand(b, generator=src.g, device="cuda") < case["own_share"], runs, torch.full_like(runs, -1))
    return dict(x=src.normal(m, k).mul_(36.0).round_().clamp_(-127, 127).to(torch.int8), packed=packed.contiguous(),
                alpha=src.normal(n).mul_(0.004).add_(0.03).abs_().add_(0.001), gamma=src.normal(b).abs_().add_(2.0),
                a=src.normal(na, r, k).mul_(1.0 / math.sqrt(k)).to(kept), b=src.normal(na, n, r).mul_(0.3 / math.sqrt(r)).to(kept),
                scale=src.normal(na).abs_().add_(0.5), adapter=runs,
                y=torch.empty((m, case["pitch"]), dtype=TYPES[case["out"]], device="cuda")[:, :n])


def prepare(case, seed):
    src = _Source(seed)
    state = _prepare_adapters(case, src) if case["kind"] == "adapters" else _prepare_norm(case, src)
    state["case"] = case
    return state


# ---- plain forms --------------------------------------------------------------------------------

def _norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    y = d * rstd * s["weight"].float() + s["bias"].float()
    return y.to(s["x"].dtype), mean[:, 0], rstd[:, 0]


def _norm_i8(s):
    # Statistics in 64 bits, each further step one 32-bit operation: the codes have one right value.
    x = s["x"].double()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = (1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)).float()
    y = (s["x"].float() - mean.float()) * rstd
    y = y * s["weight"].float()
    y = y + s["bias"].float()
    gamma = y.abs().amax(1)
    scale = torch.full_like(gamma, 127.0) / gamma.clamp(min=1e-5)
    q = torch.round(y * scale[:, None]).clamp(-128, 127).to(torch.int8)
    return q, gamma, scale


def _norm_backward(s):
    x, dy = s["x"].float(), s["dy"].float()
    rstd = s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * rstd
    g = dy * s["weight"].float()
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    kept = s["weight"].dtype
    return dx.to(s["x"].dtype), (dy * xh).sum(0).to(kept), dy.sum(0).to(kept)


def _weights(packed):
    """The values of 2-bit codes (0, 1, and 3 for -1), four to a byte."""
    shifts = torch.tensor([0, 2, 4, 6], dtype=torch.uint8, device=packed.device)
    codes = (packed[..., None] >> shifts) & 3
    w = torch.where(codes == 3, -1.0, codes.float())
    return w.view(packed.shape[0], -1)


def _adapters(s):
    rows, (na, rank, k) = s["case"]["rows"], s["a"].shape
    f = (s["gamma"].clamp(min=1e-5) / 127.0).repeat_interleave(rows)
    adapter = s["adapter"].repeat_interleave(rows).long()
    x = s["x"].float()
    y = (x @ _weights(s["packed"]).t()) * s["alpha"] * f[:, None]
    # all adapters' inner products, those of other requests' adapters set to zero
    t = (x @ s["a"].float().view(na * rank, k).t()).view(-1, na, rank)
    mine = adapter[:, None] == torch.arange(na, device=x.device)
    t = torch.where(mine[..., None], t * s["scale"][:, None], torch.zeros_like(t)) * f[:, None, None]
    y = y + t.view(-1, na * rank) @ s["b"].float().permute(0, 2, 1).reshape(na * rank, -1)
    return y.to(s["y"].dtype)


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"norm": _norm, "norm_i8": _norm_i8, "norm_backward": _norm_backward, "adapters": _adapters}[kind](state)
    from paper_2505_03254_b200 import binding
    if kind == "norm":
        return binding.layer_norm(state["x"], state["weight"], state["bias"], EPS, out=state["out"])
    if kind == "norm_i8":
        return binding.layer_norm_i8(state["x"], state["weight"], state["bias"], EPS, out=state["out"])
    if kind == "norm_backward":
        return binding.layer_norm_backward(state["dy"], state["x"], state["weight"], state["mean"], state["rstd"], out=state["out"])
    return binding.pw_proj_adapters(state["x"], state["case"]["batch"], state["packed"], state["case"]["cout"], state["alpha"],
                                    state["gamma"], state["a"], state["b"], state["scale"], state["adapter"], y=state["y"])


# ---- definitions in 64 bits ---------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adapters":
        codes = s["packed"].to(torch.int16)
        w = torch.stack([(codes // 4 ** j) % 4 for j in range(4)], dim=2).reshape(case["cout"], case["cin"]).double()
        w[w == 3] = -1
        x = s["x"].double()
        factor = (torch.clamp(s["gamma"].double(), min=float(torch.tensor(1e-5))) / 127).repeat_interleave(case["rows"])
        which = s["adapter"].repeat_interleave(case["rows"])
        y = torch.einsum("rk,ok->ro", x, w) * s["alpha"].double()
        for i in range(case["adapters"]):
            at = torch.nonzero(which == i)[:, 0]
            y[at] += (x[at] @ s["a"][i].double().T) @ s["b"][i].double().T * s["scale"][i].double()
        return y * factor[:, None]
    x, w, b = s["x"].double(), s["weight"].double(), s["bias"].double()
    if case["kind"] == "norm_backward":
        mean, rstd, dy = s["mean"].double(), s["rstd"].double(), s["dy"].double()
        xh = torch.einsum("rk,r->rk", x - mean[:, None], rstd)
        g = dy * w
        dx = (g - (g.sum(1) / case["n"])[:, None] - xh * ((g * xh).sum(1) / case["n"])[:, None]) * rstd[:, None]
        return dx, (dy * xh).sum(0), dy.sum(0)
    mean = x.sum(1) / case["n"]
    rstd = 1 / torch.sqrt(torch.square(x - mean[:, None]).sum(1) / case["n"] + EPS)
    y = (x - mean[:, None]) * rstd[:, None] * w + b
    if case["kind"] == "norm":
        return y, mean, rstd
    gamma = y.abs().max(1).values
    return None, gamma, 127 / torch.clamp(gamma, min=float(torch.tensor(1e-5)))
