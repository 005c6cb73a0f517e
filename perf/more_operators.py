"""Linear layers on 8-bit integers, as cases that can be timed.

A Linear on 8-bit operands takes rows of int8 codes with one fp32 scale for
each token, and weights with one for each output channel.  Its operand is made
from the block's activations by a row operator: the modulated LayerNorm before
the QKV projection and the MLP ("modulate"), a root-mean-square norm that first
adds a residual ("rms"), or the quantiser of rows alone, for the attention's
output, the MLP's hidden rows and the weights ("rows").  "linear" is the
product with dit_linear's epilogues.  The listed cases take the shapes of the
repository's own workloads (``synth``): widths 5,120 and 13,824 with 32,760 and
75,600 tokens, a packed batch of four requests, prompts of 77 and 512 tokens,
and the small fp32 block of width 384.

A row y is held as codes c and a scale s with y ~ c s: s is the larger of
max|y| / 127 and 2^-100, c is y / s rounded to nearest, ties to even.

A case is a dict of plain values; the rows of a packed batch's requests are
written as text, joined by ``,``.  Codes are returned in bfloat16, which holds
every whole number up to 256.
"""
import math

import torch

own = False   # False: elementary torch operations; True: the library's kernels

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
FLOOR = 2.0 ** -100   # the smallest scale
EPS = 1e-6
MOST = 75600 * 15360 * 5120   # products of the largest case


def listed():
    return [
        # the adaLN projection of one request (six vectors of 5,120): one row, bound by the weights
        {"name": "linear_one_row", "kind": "linear", "rows": "1", "n": 30720, "k": 5120, "epi": "none", "dtype": "bf16"},
        # the down projection of the small exact fp32 block (the smallest product)
        {"name": "linear_tiny_fp32", "kind": "linear", "rows": "64", "n": 384, "k": 1536, "epi": "gated", "dtype": "fp32"},
        # text keys and values of two prompts
        {"name": "linear_text", "kind": "linear", "rows": "512,77", "n": 10240, "k": 5120, "epi": "none", "dtype": "bf16"},
        # the down projection of a packed batch, with its gates and residual
        {"name": "linear_packed_down", "kind": "linear", "rows": "512,1152,4095,9450", "n": 5120, "k": 13824, "epi": "gated",
         "dtype": "bf16"},
        # the MLP's up projection of a 480p video
        {"name": "linear_480p_up", "kind": "linear", "rows": "32760", "n": 13824, "k": 5120, "epi": "gelu", "dtype": "bf16"},
        # the QKV projection of a 720p video (the largest product)
        {"name": "linear_720p_qkv", "kind": "linear", "rows": "75600", "n": 15360, "k": 5120, "epi": "none", "dtype": "bf16"},
        # the norm before the QKV projection: a packed batch, and a 720p video
        {"name": "modulate_packed", "kind": "modulate", "rows": "512,1152,4095,9450", "width": 5120, "dtype": "bf16"},
        {"name": "modulate_720p", "kind": "modulate", "rows": "75600", "width": 5120, "dtype": "bf16"},
        # a norm with its residual: one token, where latency counts, and a 480p video
        {"name": "rms_one_token", "kind": "rms", "rows": "1", "width": 5120, "add": True, "out": "codes", "dtype": "bf16"},
        {"name": "rms_480p", "kind": "rms", "rows": "32760", "width": 5120, "add": True, "out": "codes", "dtype": "bf16"},
        # the text rows of one prompt, and the MLP's hidden rows of a 480p video
        {"name": "rows_prompt", "kind": "rows", "rows": "77", "width": 5120, "dtype": "bf16"},
        {"name": "rows_480p_mlp", "kind": "rows", "rows": "32760", "width": 13824, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi, step=1):
    x = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi // step * step, max(-(-lo // step) * step, int(round(x / step)) * step))


def _split(rng, rows):
    """Up to six requests that have `rows` rows together, empty ones among them."""
    cuts = sorted(rng.randint(0, rows) for _ in range(rng.choice([0, 0, 1, 2, 3, 5])))
    return ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [rows]))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "modulate", "rms", "rows"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if kind == "linear":
        few = rng.random() < 0.4
        rows = _log_int(rng, 1, 64) if few else _log_int(rng, 65, 40000 if dtype == "bf16" else 8000)
        n, k = _log_int(rng, 64, 30720 if few else 16384, 8), _log_int(rng, 128, 14336, 16)
        while rows * n * k > MOST // 4:
            rows //= 2
        return {"kind": kind, "rows": _split(rng, rows), "n": n, "k": k,
                "epi": rng.choice(["none", "gelu", "residual", "gated"]), "dtype": dtype}
    widest = 16384 if kind == "rows" else 8192 if dtype == "bf16" else 4096
    width = _log_int(rng, 64, widest, 16)
    rows = _log_int(rng, 1, min(75600, 32760 * 13824 // (width * (1 if dtype == "bf16" else 2))))
    case = {"kind": kind, "rows": _split(rng, rows), "width": width, "dtype": dtype}
    if kind == "rms":
        case |= {"add": rng.random() < 0.8, "out": rng.choice(["codes", "codes", "values", "both"])}
    return case


# ------------------------------------------------------------------- shapes


def _rows(case):
    return [int(x) for x in case["rows"].split(",")]


def _cu(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    lens = _rows(case)
    m, r = sum(lens), sum(n > 0 for n in lens)
    if case["kind"] == "linear":
        n, k, epi = case["n"], case["k"], case["epi"]
        read = m * k + 4 * m + n * k + 4 * n + es * n
        read += es * m * n if epi in ("residual", "gated") else 0
        read += 4 * r * n if epi == "gated" else 0
        return {"bytes": read + es * m * n, "flops": 2 * m * n * k}
    w = case["width"]
    codes = m * w + 4 * m
    if case["kind"] == "modulate":
        return {"bytes": es * m * w + 8 * r * w + codes, "flops": 9 * m * w}
    if case["kind"] == "rms":
        out = (codes if case["out"] != "values" else 0) + (es * m * w if case["out"] != "codes" else 0)
        return {"bytes": es * m * w * (3 if case["add"] else 1) + es * w + out, "flops": 7 * m * w}
    return {"bytes": es * m * w + codes, "flops": 3 * m * w}


# ------------------------------------------------------------------- inputs


def _inputs(case, seed):
    """The tensors of a case, the same for prepare() and exact()."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 2606)
    normal = lambda std, *shape: torch.empty(shape, device="cuda").normal_(0, std, generator=g)
    dtype, lens = DTYPES[case["dtype"]], _rows(case)
    m = sum(lens)
    s = {"kind": case["kind"], "cu": _cu(lens)}

    def activations(std, rows, width):
        """Values of one scale but for a few channels that are larger, as activations have them."""
        x = normal(std, rows, width)
        loud = torch.randint(0, width, (max(1, width // 256),), generator=g, device="cuda")
        x[:, loud] *= 6.0
        return x

    if case["kind"] == "linear":
        n, k = case["n"], case["k"]
        # row by row, so that no tensor in 32 bits is as large as the largest operand
        def codes(rows, make):
            c, scale = torch.empty(rows, k, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
            for a in range(0, rows, 16384):
                x = make(min(16384, rows - a))
                top = x.abs().amax(1)
                scale[a:a + 16384] = top / 127
                c[a:a + 16384] = torch.round(x * (127 / top)[:, None]).to(torch.int8)
            return c, scale
        s["a"], s["a_scales"] = codes(m, lambda rows: activations(1.0, rows, k))
        s["w"], s["w_scales"] = codes(n, lambda rows: normal(0.02, rows, k))
        s["epi"], s["bias"] = case["epi"], normal(0.1, n).to(dtype)
        if case["epi"] in ("residual", "gated"):
            s["res"] = normal(1.0, m, n).to(dtype)
        if case["epi"] == "gated":
            s["gate"] = normal(0.5, len(lens), n)
        return s
    w = case["width"]
    s["x"] = activations(1.5, m, w).to(dtype)
    if case["kind"] == "modulate":   # two of the six vectors of each request
        s["mod"] = normal(0.3, len(lens), 6, w)
    if case["kind"] == "rms":
        s["gain"], s["what"] = (1 + normal(0.2, w)).to(dtype), case["out"]
        s["z"] = normal(0.5, m, w).to(dtype) if case["add"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if s["kind"] == "linear":
        s["out"] = torch.empty(s["a"].shape[0], case["n"], dtype=s["bias"].dtype, device="cuda")
    else:
        rows, w = s["x"].shape
        if s.get("what") != "values":
            s["codes"] = torch.empty(rows, w, dtype=torch.int8, device="cuda")
            s["scales"] = torch.empty(rows, device="cuda")
        if s["kind"] == "rms":
            s["sum"] = torch.empty_like(s["x"]) if s["z"] is not None else None
            s["out"] = torch.empty_like(s["x"]) if s["what"] != "codes" else None
    if own:
        from paper_2606_13501_amd import binding as B
        s["lib"] = B
        s["epilogue"] = {"none": B.EPI_NONE, "gelu": B.EPI_GELU_TANH, "residual": B.EPI_RESIDUAL,
                         "gated": B.EPI_GATED_RESIDUAL}[s.get("epi", "none")]
    else:   # the request of each row
        lens = torch.tensor(_rows(case), device="cuda")
        s["request"] = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), lens)
    return s


# -------------------------------------------------------------- the operators


def run(s):
    if s["kind"] == "linear":
        if own:
            gate = s.get("gate")
            s["lib"].linear_i8(s["a"], s["a_scales"], s["w"], s["w_scales"], s["bias"], s["out"], s["epilogue"], s.get("res"),
                               gate, 0 if gate is None else gate.stride(0), None if gate is None else s["cu"])
        else:
            _plain_linear(s)
        return s["out"]
    if own:
        if s["kind"] == "modulate":
            mod = s["mod"]
            s["lib"].adaln_modulate_i8(s["x"], mod[:, 0], mod[:, 1], mod.stride(0), s["cu"], EPS, s["codes"], s["scales"])
        elif s["kind"] == "rms":
            s["lib"].add_rms_norm(s["x"], s["z"], s["gain"], EPS, s["sum"], s["out"], s.get("codes"), s.get("scales"))
        else:
            s["lib"].quantize_rows(s["x"], s["codes"], s["scales"])
    else:
        {"modulate": _plain_modulate, "rms": _plain_rms, "rows": _plain_rows}[s["kind"]](s)
    found = {}
    if s["kind"] == "rms":
        found = {name: s[name] for name in ("sum", "out") if s[name] is not None}
    if "codes" in s:
        found |= {"codes": s["codes"].to(torch.bfloat16), "scales": s["scales"]}
    return found


def _plain_linear(s):
    # a sum of products of codes may pass 2^24, so they are summed in 64 bits, exactly
    z = torch.matmul(s["a"].double(), s["w"].double().T).float()
    z = z * s["a_scales"][:, None] * s["w_scales"] + s["bias"].float()
    if s["epi"] == "gelu":
        z = 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    elif s["epi"] == "residual":
        z = s["res"].float() + z
    elif s["epi"] == "gated":
        z = s["res"].float() + s["gate"][s["request"]] * z
    s["out"].copy_(z)


def _plain_codes(s, y):
    top = y.abs().amax(1)
    scale = torch.clamp(top / 127, min=FLOOR)
    scale = torch.where(torch.isfinite(top), scale, math.nan)
    codes = torch.round(y * (1 / scale)[:, None])
    s["codes"].copy_(torch.where(torch.isfinite(codes), codes, 0.0))
    s["scales"].copy_(scale)


def _plain_modulate(s):
    x = s["x"].float()
    x = x - x.mean(1, keepdim=True)
    y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    shift, scale = s["mod"][:, 0], s["mod"][:, 1]
    _plain_codes(s, y * (1 + scale)[s["request"]] + shift[s["request"]])


def _plain_rms(s):
    x = s["x"]
    if s["z"] is not None:
        s["sum"].copy_(x.float() + s["z"].float())
        x = s["sum"]
    x = x.float()
    y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * s["gain"].float()
    if s["out"] is not None:
        s["out"].copy_(y)
    if "codes" in s:
        _plain_codes(s, y)


def _plain_rows(s):
    _plain_codes(s, s["x"].float())


# ------------------------------------------------------ the definition in 64 bits


def _exact_codes(y):
    """Rows of 64-bit values: the nearest whole numbers of steps, and the steps."""
    step = y.abs().max(dim=1, keepdim=True).values.div(127.0)
    step[step < FLOOR] = FLOOR
    return {"codes": (y / step).round(), "scales": step[:, 0]}


def exact(case, seed):
    s = _inputs(case, seed)
    cu, parts = s["cu"], []
    if case["kind"] == "linear":
        out = torch.empty(s["a"].shape[0], case["n"], dtype=torch.float64, device="cuda")
        w = s["w"].t().double() * s["w_scales"].double()    # [k, n]: the weights' own values
        for r in range(len(cu) - 1):
            for a in range(cu[r], cu[r + 1], 8192):
                b = min(a + 8192, cu[r + 1])
                x = s["a"][a:b].double() * s["a_scales"][a:b, None].double()
                z = torch.addmm(s["bias"].double(), x, w)
                if case["epi"] == "gelu":   # 1 + tanh(u) = 2 / (1 + exp(-2 u))
                    z = z / (1 + torch.exp(-z * (1 + 0.044715 * z.square()) * math.sqrt(8 / math.pi)))
                if case["epi"] == "gated":
                    z *= s["gate"][r].double()
                if "res" in s:
                    z += s["res"][a:b].double()
                out[a:b] = z
        return out
    x, w = s["x"].double(), case["width"]
    if case["kind"] == "modulate":
        for r in range(len(cu) - 1):
            var, mean = torch.var_mean(x[cu[r]:cu[r + 1]], dim=1, correction=0, keepdim=True)
            y = (x[cu[r]:cu[r + 1]] - mean) / (var + EPS).sqrt()
            parts.append(torch.addcmul(s["mod"][r, 0].double(), y, 1 + s["mod"][r, 1].double()))
        return _exact_codes(torch.cat(parts))
    if case["kind"] == "rows":
        return _exact_codes(x)
    found = {}
    if s["z"] is not None:
        found["sum"] = x + s["z"].double()
        x = found["sum"].to(s["x"].dtype).double()   # the norm is that of the stored sum
    y = x * s["gain"].double() / (x.norm(dim=1, keepdim=True).square() / w + EPS).sqrt()
    if case["out"] != "codes":
        found["out"] = y
    return found | (_exact_codes(y) if case["out"] != "values" else {})
