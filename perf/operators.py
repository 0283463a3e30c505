"""The 8-bit block operators and group norm as timed cases, with their plain forms.

Kinds of a case:

  quantize   x [batch, rows, cols] -> e4m3 values [batch, rows, cols up to whole blocks of 128] and fp32 scales
             [batch, column blocks, row blocks]; ``g`` rows (1: activations, 128: weights) share a scale with 128 columns
  product    y = act(bias + A B^T) of two such matrices, a scale of A per row, of B per ``g`` rows; batch > 1 has neither bias
             nor activation
  norm       group norm over channels-last [n, h, w, c] and an activation
  norm_fp8   the same, written as 8-bit blocks of the matrix [n * h * w, c]

``own`` False: elementary torch operations.  ``own`` True: the library's entry points.
"""
import math

import torch

own = False

BLOCK = 128
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# dense classes and activations, by the library's numbers
CLASSES = {"add": 4, "relu": 5, "gelu": 6}
ACTS = {"none": 0, "relu": 1, "relu6": 2, "gelu": 3, "silu": 4}


def _quantize(dtype, batch, rows, cols, g):
    return {"kind": "quantize", "dtype": dtype, "batch": batch, "rows": rows, "cols": cols, "g": g}


def _product(dtype, act, m, n, k, g, batch=1):
    return {"kind": "product", "dtype": dtype, "act": act, "batch": batch, "m": m, "n": n, "k": k, "g": g}


def _norm(kind, dtype, act, n, h, w, c, groups):
    return {"kind": kind, "dtype": dtype, "act": act, "n": n, "h": h, "w": w, "c": c, "groups": groups}


def listed():
    return [
        # the input of a dense layer while one sequence is decoded: latency
        dict(_quantize("bf16", 1, 1, 4096, 1), name="quantize_token_bf16"),
        # a throughput batch of activations: memory
        dict(_quantize("bf16", 1, 16384, 4096, 1), name="quantize_16384_rows_bf16"),
        # a layer's weights on their way into the format, odd sizes
        dict(_quantize("f32", 1, 1000, 2050, 128), name="quantize_weights_f32"),
        # a dense layer for a single token: the weights' bytes
        dict(_product("bf16", "add", 1, 4096, 4096, 128), name="dense_token_bf16"),
        # a classifier over a small batch, odd rows, single-precision logits
        dict(_product("f32", "add", 24, 1000, 2048, 128), name="dense_classifier_f32"),
        # a transformer encoder's projection, 8 x 128 tokens
        dict(_product("bf16", "gelu", 1024, 768, 768, 128), name="dense_encoder_bf16"),
        # the large matrix product
        dict(_product("bf16", "relu", 8192, 8192, 8192, 128), name="dense_8192_bf16"),
        # batched products of activations, a scale per row of either, nothing a whole tile
        dict(_product("bf16", "add", 197, 333, 520, 1, 24), name="matmul_ragged_bf16"),
        # a late, small map of odd sides and channels, one image: latency
        dict(_norm("norm", "f32", "gelu", 1, 9, 7, 90, 9), name="norm_small_odd_f32"),
        # a throughput batch of early maps: memory
        dict(_norm("norm", "bf16", "relu", 16, 128, 128, 256, 32), name="norm_16x128x128_bf16"),
        # one image pair in front of an 8-bit pointwise layer, ten channels a group
        dict(_norm("norm_fp8", "bf16", "silu", 2, 64, 64, 320, 32), name="norm_fp8_2x64x64_bf16"),
        # the same for a batch of deep maps
        dict(_norm("norm_fp8", "bf16", "silu", 16, 32, 32, 1280, 32), name="norm_fp8_16x32x32_bf16"),
    ]


# ---- drawn cases ---------------------------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Whole blocks, whole 16s or anything."""
    v, u = _log(rng, lo, hi), rng.random()
    unit = 128 if u < 0.3 else 16 if u < 0.6 else 1
    return max(lo, v // unit * unit) if v >= unit else v


def draw(rng):
    known = [{k: v for k, v in c.items() if k != "name"} for c in listed()]
    while True:
        case = _draw(rng)
        if case not in known:
            return case


def _draw(rng):
    u, dtype = rng.random(), rng.choice(["bf16", "bf16", "f32"])
    if u < 0.2:
        cols = _size(rng, 16, 8192)
        batch = rng.choice([1, 1, 1, _log(rng, 2, 16)])
        rows = _log(rng, 1, min(16384, max(1, (1 << 26) // (cols * batch))))
        return _quantize(dtype, batch, rows, cols, rng.choice([1, 1, 128]))
    if u < 0.5:
        m = rng.choice([_log(rng, 1, 64), _log(rng, 1, 8192)])
        return _product(dtype, rng.choice(list(CLASSES)), m, _size(rng, 16, 8192), _size(rng, 32, 8192), rng.choice([1, 128, 128]))
    if u < 0.6:
        return _product(dtype, "add", _log(rng, 1, 512), _size(rng, 16, 512), _size(rng, 32, 1024), rng.choice([1, 1, 128]),
                        _log(rng, 2, 64))
    groups = rng.choice([1, 3, 8, 16, 32, 32])
    c = groups * _log(rng, 1, max(2, 2048 // groups))
    h, w = _log(rng, 1, 128), _log(rng, 1, 128)
    n = _log(rng, 1, min(64, max(1, (1 << 26) // (h * w * c))))
    return _norm("norm" if u < 0.8 else "norm_fp8", dtype, rng.choice(list(ACTS)), n, h, w, c, groups)


# ---- states --------------------------------------------------------------------------------------------------------
def _blocks(n):
    return -(-n // BLOCK)


def _plain_quantize(x, g):
    """x [batch, rows, cols], 32 bits: (values as float8_e4m3fn [batch, rows, kp], scales [batch, kb, row blocks])."""
    batch, rows, cols = x.shape
    kb, rb = _blocks(cols), -(-rows // g)
    x = torch.nn.functional.pad(x, (0, kb * BLOCK - cols, 0, rb * g - rows)).view(batch, rb, g, kb, BLOCK)
    amax = x.abs().amax(dim=(2, 4), keepdim=True).clamp(min=2.0 ** -100)
    q = (x * (448.0 / amax)).to(torch.float8_e4m3fn).view(batch, rb * g, kb * BLOCK)[:, :rows].contiguous()
    return q, (amax / 448.0).view(batch, rb, kb).transpose(1, 2).contiguous()


def _plain_values(q, scale, g):
    """The 32-bit values that a blocked matrix stands for, [batch, rows, kp]."""
    batch, rows, kp = q.shape
    s = scale.repeat_interleave(g, dim=2)[:, :, :rows] if g > 1 else scale
    return (q.float().view(batch, rows, kp // BLOCK, BLOCK) * s.transpose(1, 2).unsqueeze(-1)).view(batch, rows, kp)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    c, dt = case, DTYPES[case["dtype"]]
    s = {"case": c}
    if c["kind"] == "quantize":
        # activations of unequal rows, as they come out of a layer
        s["x"] = (normal(c["batch"], c["rows"], c["cols"]) * torch.exp(normal(c["batch"], c["rows"], 1))).to(dt)
        if own:
            from paper_2201_05587_amd import api
            s["shape"] = api.tt_quant_shape(c["batch"], c["rows"], c["cols"], c["g"], api.TT_BF16 if dt == torch.bfloat16 else api.TT_F32)
    elif c["kind"] == "product":
        a = normal(c["batch"], c["m"], c["k"]) * torch.exp(0.5 * normal(c["batch"], c["m"], 1))
        b = normal(c["batch"], c["n"], c["k"]) / math.sqrt(c["k"])
        s["a"], s["a_scale"] = _plain_quantize(a, 1)
        s["b"], s["b_scale"] = _plain_quantize(b, c["g"])
        s["bias"] = (normal(c["n"]) * 0.1).to(dt) if c["batch"] == 1 else None
        if own:
            from paper_2201_05587_amd import api
            s["shape"] = api.tt_fp8_shape(c["batch"], c["m"], c["n"], c["k"], c["g"], api.TT_BF16 if dt == torch.bfloat16 else api.TT_F32)
            s["ws"] = torch.empty(max(16, api.tt_fp8_plan(s["shape"]).workspace_bytes), dtype=torch.uint8, device="cuda")
    else:
        # a convolution's output: channels with means and spreads of their own
        x = normal(c["n"], c["h"], c["w"], c["c"]) * torch.exp(0.5 * normal(c["c"])) + normal(c["c"])
        s["x"], s["gamma"], s["beta"] = x.to(dt), (1.0 + 0.2 * normal(c["c"])).to(dt), (0.2 * normal(c["c"])).to(dt)
        if own:
            from paper_2201_05587_amd import api
            s["shape"] = api.tt_norm_shape(c["n"], c["h"], c["w"], c["c"], c["groups"], api.TT_BF16 if dt == torch.bfloat16 else api.TT_F32)
            s["ws"] = torch.empty(max(16, api.tt_norm_plan(s["shape"], c["kind"] == "norm_fp8").workspace_bytes), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
EPS = 1e-5


def _plain_act(v, act):
    if act == "relu":
        return v.clamp(min=0.0)
    if act == "relu6":
        return v.clamp(min=0.0, max=6.0)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _plain_norm(s):
    c = s["case"]
    x = s["x"].float().view(c["n"], c["h"] * c["w"], c["groups"], c["c"] // c["groups"])
    centred = x - x.mean(dim=(1, 3), keepdim=True)
    v = centred * torch.rsqrt((centred * centred).mean(dim=(1, 3), keepdim=True) + EPS)
    v = v.view(c["n"], c["h"], c["w"], c["c"]) * s["gamma"].float() + s["beta"].float()
    return _plain_act(v, c["act"])


def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        from paper_2201_05587_amd import api
        if kind == "quantize":
            return api.tt_quantize_fp8(s["x"], s["shape"])
        if kind == "product":
            if c["batch"] > 1:
                return api.tt_batch_matmul_fp8(s["a"], s["a_scale"], s["b"], s["b_scale"], s["shape"], ws=s["ws"])
            return api.tt_dense_fp8(s["a"], s["a_scale"], s["b"], s["b_scale"], s["bias"], s["shape"], CLASSES[c["act"]], ws=s["ws"])
        norm = api.tt_group_norm_act if kind == "norm" else api.tt_group_norm_act_fp8
        return norm(s["x"], s["gamma"], s["beta"], s["shape"], ACTS[c["act"]], EPS, ws=s["ws"])
    if kind == "quantize":
        return _plain_quantize(s["x"].float(), c["g"])
    if kind == "product":
        a, b = _plain_values(s["a"], s["a_scale"], 1), _plain_values(s["b"], s["b_scale"], c["g"])
        if c["batch"] > 1:
            return torch.matmul(a, b.transpose(1, 2)).to(DTYPES[c["dtype"]])
        return _plain_act(torch.matmul(a[0], b[0].t()) + s["bias"].float(), c["act"]).to(DTYPES[c["dtype"]])
    v = _plain_norm(s)
    if kind == "norm":
        return v.to(DTYPES[c["dtype"]])
    q, scale = _plain_quantize(v.view(1, -1, c["c"]), 1)
    return q[0], scale[0]


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "quantize":
        n = c["batch"] * c["rows"] * c["cols"]
        return {"bytes": n * (e + 1) + 4 * c["batch"] * _blocks(c["cols"]) * -(-c["rows"] // c["g"]), "flops": 2 * n}
    if c["kind"] == "product":
        scales = _blocks(c["k"]) * (c["m"] + -(-c["n"] // c["g"]))
        bias = e * c["n"] if c["batch"] == 1 else 0
        return {"bytes": c["batch"] * ((c["m"] + c["n"]) * c["k"] + 4 * scales + e * c["m"] * c["n"]) + bias,
                "flops": 2 * c["batch"] * c["m"] * c["n"] * c["k"]}
    pixels = c["n"] * c["h"] * c["w"]
    out = pixels * (c["c"] * e if c["kind"] == "norm" else c["c"] + 4 * _blocks(c["c"]))
    return {"bytes": pixels * c["c"] * e + out + 2 * e * c["c"], "flops": 8 * pixels * c["c"]}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def _exact_act(v, act):
    return {"none": lambda: v, "add": lambda: v, "relu": lambda: torch.where(v > 0, v, torch.zeros_like(v)),
            "relu6": lambda: torch.minimum(torch.relu(v), torch.full_like(v, 6.0)),
            "gelu": lambda: v * torch.special.ndtr(v), "silu": lambda: v * torch.sigmoid(v)}[act]()


def _exact_blocks(x, g):
    """The 8-bit format of x [batch, rows, cols] from its definition: values are whole multiples of 2^(e - 3), e >= -6."""
    batch, rows, cols = x.shape
    out = torch.zeros(batch, rows, _blocks(cols) * BLOCK, dtype=torch.float64, device=x.device)
    scales = torch.zeros(batch, _blocks(cols), -(-rows // g), dtype=torch.float64, device=x.device)
    for b in range(_blocks(cols)):
        part = x[:, :, b * BLOCK:(b + 1) * BLOCK]
        top = part.abs().amax(dim=2)
        if g > 1:
            top = torch.stack([piece.amax(dim=1) for piece in top.split(g, dim=1)], dim=1)
        top = torch.clamp(top, min=2.0 ** -100)
        scales[:, b] = top / 448
        v = part * 448 / top.repeat_interleave(g, dim=1)[:, :rows].unsqueeze(2)
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        out[:, :, b * BLOCK:b * BLOCK + part.shape[2]] = torch.round(v / step) * step
    return out, scales


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "quantize":
        return _exact_blocks(s["x"].double(), c["g"])
    if c["kind"] == "product":
        y = torch.zeros(c["batch"], c["m"], c["n"], dtype=torch.float64, device="cuda")
        for i in range(c["batch"]):
            wide = s["b_scale"][i].double().repeat_interleave(c["g"], dim=1)[:, :c["n"]]
            for b in range(_blocks(c["k"])):
                cut = slice(b * BLOCK, (b + 1) * BLOCK)
                part = s["a"][i, :, cut].double() @ s["b"][i, :, cut].double().t().contiguous()
                y[i] += part * s["a_scale"][i, b].double().unsqueeze(1) * wide[b]
        return y if c["batch"] > 1 else _exact_act(y[0] + s["bias"].double(), c["act"])
    x = s["x"].double().view(c["n"], -1, c["c"])
    y = torch.empty_like(x)
    wide = c["c"] // c["groups"]
    for k in range(c["groups"]):
        cut = slice(k * wide, (k + 1) * wide)
        part = x[:, :, cut]
        var, mean = torch.var_mean(part, dim=(1, 2), keepdim=True, correction=0)
        v = (part - mean) / torch.sqrt(var + EPS) * s["gamma"][cut].double() + s["beta"][cut].double()
        y[:, :, cut] = _exact_act(v, c["act"])
    if c["kind"] == "norm":
        return y.view(s["x"].shape)
    q, scale = _exact_blocks(y.view(1, -1, c["c"]), 1)
    return q[0], scale[0]
