"""What lies between the products of a transformer layer that is served from decoded weights, and
the INT8 product itself: what these operators are measured on, and their plain forms.

``op``:
  rope      rotary positions of a step's queries and keys, which lie in one fused projection's rows;
            positions given, or from the requests' lengths; frequencies stretched for long contexts
  norm      h = r + alpha g u, y = N2(h): the norm before a block with what comes before it, the
            residual sum with its gate and scale, and (u = N1(x)) the norm after the last block;
            y in 16 bits, or quantised for the next product
  quant     activations to INT8 with one FP32 scale for each row (token)
  product   Y = X W^T of INT8 operands with those scales and W's scale for each row (what an INT8
            container decodes to), and a bias
  glu       y = act(a) b of an MLP's two halves, in 16 bits or quantised for the next product

Quantised outputs are E4M3 codes with an FP32 scale for each 128 of a row, or INT8 codes with one
for each row; norm's and glu's INT8 codes are returned as the values that they stand for.
Where ``own`` is false ``run`` computes in elementary 32-bit torch operations (angles in 64) and
rounds once at the end; where it is true it calls the library.  Sizes come from the workloads of
bench.py (the MLP of a 27B-class language model, the diffusion-transformer blocks) or are generic
ones of served models.
"""
import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32,
      "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1, "int8": 1}
EPS = 1e-6


def _cdiv(a, b):
    return -(-a // b)


def listed():
    return [
        # one token of one conversation: launch latency is all of it
        dict(name="rope_token", op="rope", requests=1, top_new=1, top_cached=4000, q_heads=40, k_heads=8, dim=128,
             rot=128, first=0, layout="half", dtype="bf16", stretch="none", by="lengths"),
        # two long prompts, frequencies stretched by turns: reads and writes of memory
        dict(name="rope_prompt", op="rope", requests=2, top_new=8192, top_cached=100000, q_heads=40, k_heads=8, dim=128,
             rot=128, first=0, layout="half", dtype="bf16", stretch="turns", by="lengths"),
        # one token before a block: the residual sum, the norm and the next product's FP8 operand
        dict(name="norm_token", op="norm", m=1, n=5120, post="none", pre="rms", res=True, gate=False, rows=0,
             x="bf16", r="bf16", w="bf16", out="e4m3", bias=False, alpha=1.0),
        # a long prompt with a norm after the last block and one before the next
        dict(name="norm_prompt", op="norm", m=8192, n=5120, post="rms", pre="rms", res=True, gate=False, rows=0,
             x="bf16", r="bf16", w="bf16", out="bf16", bias=False, alpha=1.0),
        # two images' tokens of a diffusion transformer: gated residual sum, modulated layer norm
        dict(name="norm_gated", op="norm", m=8222, n=3840, post="none", pre="layer", res=True, gate=True, rows=4111,
             x="bf16", r="fp32", w="bf16", out="fp16", bias=True, alpha=1.0),
        # one token before the down projection
        dict(name="quant_token", op="quant", m=1, k=17408, dtype="bf16"),
        # a long prompt before the down projection: reads and writes of memory
        dict(name="quant_prompt", op="quant", m=8192, k=17408, dtype="bf16"),
        # an odd batch of tokens between up and down projection
        dict(name="glu_batch", op="glu", m=61, n=17408, act="silu", gated=True, dtype="bf16", out="e4m3"),
        # a long prompt between them
        dict(name="glu_prompt", op="glu", m=8192, n=17408, act="silu", gated=True, dtype="bf16", out="e4m3"),
        # one token through the up projection: every weight is read once for one row
        dict(name="product_token", op="product", m=1, n=17408, k=5120, y="bf16", bias=False),
        # an odd batch of tokens through the down projection
        dict(name="product_batch", op="product", m=203, n=5120, k=17408, y="bf16", bias=True),
        # a long prompt through the down projection: the matrix instructions' rate
        dict(name="product_prompt", op="product", m=8192, n=5120, k=17408, y="bf16", bias=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One case of the listed ones' ranges, no dearer than the dearest listed one of its kind."""
    while True:
        op = rng.choice(("rope", "norm", "quant", "product", "glu"))
        if op == "rope":
            dim = rng.choice((64, 80, 96, 128, 256))
            rot = rng.choice((dim, dim, dim // 2, dim // 4))
            k_heads = rng.choice((0, 1, 2, 4, 8))
            c = dict(op=op, requests=_log(rng, 1, 200), top_new=_log(rng, 1, 8192), top_cached=_log(rng, 1, 1000000),
                     q_heads=max(1, k_heads) * rng.choice((1, 4, 5, 8)), k_heads=k_heads, dim=dim, rot=rot,
                     first=rng.choice((0, dim - rot)), layout=rng.choice(("half", "pairs")),
                     dtype=rng.choice(("bf16", "fp16", "fp32")), stretch=rng.choice(("none", "linear", "base", "turns", "index")),
                     by=rng.choice(("given", "lengths")))
        elif op == "norm":
            out = rng.choice(("bf16", "fp16", "fp32", "e4m3", "int8"))
            unit = 16 if out in ("e4m3", "int8") else 8
            m, res = _log(rng, 1, 16384), rng.random() < 0.7
            c = dict(op=op, m=m, n=unit * _log(rng, 1, 17408 // unit), post=rng.choice(("none", "rms", "layer")),
                     pre=rng.choice(("rms", "layer")), res=res, gate=res and rng.random() < 0.4,
                     rows=rng.choice((0, 0, max(1, m // 3))), x=rng.choice(("bf16", "fp16", "fp32")),
                     r=rng.choice(("bf16", "fp32")), w=rng.choice(("bf16", "fp32")), out=out, bias=rng.random() < 0.4,
                     alpha=rng.choice((1.0, 0.7)))
        elif op == "quant":
            c = dict(op=op, m=_log(rng, 1, 16384), k=16 * _log(rng, 1, 1100), dtype=rng.choice(("bf16", "fp16", "fp32")))
        elif op == "product":
            c = dict(op=op, m=_log(rng, 1, 9000), n=_log(rng, 16, 18000), k=16 * _log(rng, 1, 1100),
                     y=rng.choice(("bf16", "fp16", "fp32")), bias=rng.random() < 0.4)
        else:
            c = dict(op=op, m=_log(rng, 1, 16384), n=16 * _log(rng, 1, 1100), act=rng.choice(("silu", "gelu_tanh", "gelu")),
                     gated=rng.random() < 0.8, dtype=rng.choice(("bf16", "fp16", "fp32")),
                     out=rng.choice(("bf16", "fp16", "fp32", "e4m3", "int8")))
        most = [x for x in listed() if x["op"] == op]
        w = work(c)
        if all(w[u] <= max(work(x)[u] for x in most) for u in ("bytes", "flops")) and _values(c) <= max(map(_values, most)):
            return c


def _values(c):
    """How many values the largest intermediates of a plain form hold."""
    if c["op"] == "rope":
        return sum(_counts(c)[1]) * (c["q_heads"] + c["k_heads"]) * c["dim"]
    if c["op"] == "product":
        return c["m"] * c["k"] + c["n"] * c["k"] + c["m"] * c["n"]
    return c["m"] * c.get("n", c.get("k"))


def _counts(c):
    """(tokens cached, tokens new) of each request of a rope case: of the case alone, so that its work is known."""
    r = random.Random("counts %d %d %d" % (c["requests"], c["top_new"], c["top_cached"]))
    new = [r.randint(1, c["top_new"]) for _ in range(c["requests"])]
    new[-1] = c["top_new"]
    return [r.randint(0, c["top_cached"]) for _ in new], new


def _scale_bytes(m, n, out):
    return 4 * m * _cdiv(n, 128) if out == "e4m3" else 4 * m if out == "int8" else 0


def work(case):
    c = case
    if c["op"] == "rope":
        tokens = sum(_counts(c)[1])
        v = tokens * (c["q_heads"] + c["k_heads"]) * c["dim"]
        at = 4 * tokens if c["by"] == "given" else 8 * c["requests"]
        return {"bytes": 2 * v * SIZE[c["dtype"]] + at + 4 * c["rot"], "flops": 3 * v * c["rot"] // c["dim"]}
    if c["op"] == "norm":
        m, n = c["m"], c["n"]
        h = c["res"] or c["post"] != "none"
        groups = _cdiv(m, c["rows"]) if c["rows"] else 1
        vectors = n * SIZE[c["w"]] * ((1 + c["bias"]) * (groups + (c["post"] != "none")) + c["gate"] * groups)
        return {"bytes": m * n * (SIZE[c["x"]] + SIZE[c["out"]] + (c["res"] + h) * SIZE[c["r"]]) + vectors + _scale_bytes(m, n, c["out"]),
                "flops": 10 * m * n}
    if c["op"] == "quant":
        return {"bytes": c["m"] * c["k"] * (SIZE[c["dtype"]] + 1) + 4 * c["m"], "flops": 2 * c["m"] * c["k"]}
    if c["op"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": (m + n) * k + 4 * (m + n + n * c["bias"]) + m * n * SIZE[c["y"]], "flops": 2 * m * n * k}
    m, n = c["m"], c["n"]
    return {"bytes": m * n * ((1 + c["gated"]) * SIZE[c["dtype"]] + SIZE[c["out"]]) + _scale_bytes(m, n, c["out"]), "flops": 10 * m * n}


# ---- inputs -----------------------------------------------------------------------------
def _randn(shape, g):
    return torch.randn(shape, generator=g, device="cuda")


def _hidden(m, n, g, size=1.0):
    """Hidden states: rows of different size, a few channels far out."""
    x = _randn((m, n), g) * torch.exp(0.5 * _randn((m, 1), g)) * size
    x[:, torch.randint(0, n, (1 + n // 500,), generator=g, device="cuda")] *= 20
    return x


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c, g = case, torch.Generator("cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "rope":
        cached, new = _counts(c)
        tokens, hq, hk, d = sum(new), c["q_heads"], c["k_heads"], c["dim"]
        # queries, keys and values as the fused projection leaves them: side by side in one row for each token
        rows = _randn((tokens, hq + 2 * hk, d), g).to(DT[c["dtype"]])
        s["q"], s["k"] = rows[:, :hq], rows[:, hq: hq + hk]
        # lengths with the new tokens among them, and sums of the new ones, as the cache's tables hold them
        s["len"] = _ints([a + b for a, b in zip(cached, new)])
        s["cu"] = _ints([sum(new[:i]) for i in range(len(new) + 1)])
        s["tokens"] = tokens
        if c["by"] == "given":
            s["pos"] = torch.randint(0, c["top_cached"] + 1, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    elif c["op"] == "norm":
        m, n = c["m"], c["n"]
        groups, dt = _cdiv(m, c["rows"]) if c["rows"] else 1, DT[c["w"]]
        s["x"] = _hidden(m, n, g).to(DT[c["x"]])
        s["r"] = _hidden(m, n, g, 3.0).to(DT[c["r"]]) if c["res"] else None
        s["w1"] = (1 + 0.2 * _randn((n,), g)).to(dt) if c["post"] != "none" else None
        s["b1"] = (0.1 * _randn((n,), g)).to(dt) if c["bias"] and c["post"] != "none" else None
        # one row of modulations for each image or sequence: shift, scale and gate side by side
        mod = 0.3 * _randn((groups, 3, n), g)
        if not c["rows"]:
            mod[:, 1] += 1
        mod = mod.to(dt)
        s["b2"], s["w2"], s["g"] = mod[:, 0] if c["bias"] else None, mod[:, 1], mod[:, 2] if c["gate"] else None
    elif c["op"] == "quant":
        s["x"] = _hidden(c["m"], c["k"], g).to(DT[c["dtype"]])
    elif c["op"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        s["x"] = (_randn((m, k), g) * 32).clamp_(-127, 127).round_().to(torch.int8)
        s["w"] = (_randn((n, k), g) * 40).clamp_(-127, 127).round_().to(torch.int8)
        s["xs"], s["ws"] = 0.02 * torch.exp(0.5 * _randn((m,), g)), 2e-4 * torch.exp(0.5 * _randn((n,), g))
        s["b"] = _randn((n,), g) if c["bias"] else None
    else:
        # both halves as one projection leaves them: side by side in one row for each token
        ab = _hidden(c["m"], 2 * c["n"], g).to(DT[c["dtype"]])
        s["a"], s["b"] = ab[:, : c["n"]], ab[:, c["n"]:] if c["gated"] else None
    return s


# ---- plain forms --------------------------------------------------------------------------
BASE, FACTOR, TRAINED, LOW, HIGH = 10000.0, 8.0, 8192.0, 1.0, 4.0
INDEX_LOW, INDEX_HIGH = 1.0, 32.0


def _rates(rot, stretch):
    """Radians a position of each pair, in 64 bits."""
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    base = BASE * FACTOR ** (rot / (rot - 2)) if stretch == "base" else BASE
    rate = torch.exp(i * (-2.0 / rot * math.log(base)))
    if stretch == "linear":
        return rate / FACTOR
    if stretch == "turns":      # by the turns that a pair makes over the trained length
        keep = ((TRAINED * rate / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        return rate * (keep + (1 - keep) / FACTOR)
    if stretch == "index":      # by the pair's place between those that make so many turns
        at = [rot * math.log(TRAINED / (2 * math.pi * t)) / (2 * math.log(BASE)) for t in (INDEX_HIGH, INDEX_LOW)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        keep = 1 - ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return rate * (keep + (1 - keep) / FACTOR)
    return rate


def _amplitude(c):
    return 0.1 * math.log(FACTOR) + 1 if c["stretch"] == "index" else 1.0


def _positions(s):
    if "pos" in s:
        return s["pos"].long()
    t = torch.arange(s["tokens"], device="cuda")
    req = torch.searchsorted(s["cu"][1:].long(), t, right=True)
    return s["len"].long()[req] - s["cu"].long()[req + 1] + t


def _plain_rope(s):
    c = s["case"]
    angle = _positions(s).double()[:, None] * _rates(c["rot"], c["stretch"])
    cos, sin = [(f(angle) * _amplitude(c)).float()[:, None] for f in (torch.cos, torch.sin)]
    lo, hi, rot = c["first"], c["first"] + c["rot"], c["rot"]

    def turned(x):
        y = x.float()
        part = y[:, :, lo:hi]
        a, b = (part[..., : rot // 2], part[..., rot // 2:]) if c["layout"] == "half" else (part[..., 0::2], part[..., 1::2])
        a, b = a * cos - b * sin, a * sin + b * cos
        mid = torch.cat((a, b), 2) if c["layout"] == "half" else torch.stack((a, b), 3).flatten(2)
        return torch.cat((y[:, :, :lo], mid, y[:, :, hi:]), 2).to(x.dtype)

    return turned(s["q"]), turned(s["k"])


def _plain_normed(x, kind, w, b):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    x = x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * w
    return x if b is None else x + b


def _plain_e4m3(y):
    m, n = y.shape
    b = torch.nn.functional.pad(y, (0, -n % 128)).view(m, -1, 128)
    scale = b.abs().amax(2) * (1.0 / 448.0)
    scale = torch.where(scale == 0, 1.0, scale)
    return (b / scale[:, :, None]).clamp(-448, 448).view(m, -1)[:, :n].to(torch.float8_e4m3fn).contiguous(), scale


def _plain_int8(y):
    scale = y.abs().amax(1) * (1.0 / 127.0)
    scale = torch.where(scale == 0, 1.0, scale)
    return (y / scale[:, None]).round().clamp(-127, 127).to(torch.int8), scale


def _plain_out(y, out):
    if out == "e4m3":
        return _plain_e4m3(y)
    if out == "int8":
        q, scale = _plain_int8(y)
        return (q * scale[:, None]).to(torch.bfloat16), scale
    return (y.to(DT[out]),)


def _of_rows(v, s):
    """Modulations for each row: the same for `rows` rows at a time, or for all."""
    c = s["case"]
    if v is None:
        return None
    return v.float().repeat_interleave(c["rows"], 0)[: c["m"]] if c["rows"] else v.float()


def _plain_norm(s):
    c = s["case"]
    h = _plain_normed(s["x"].float(), c["post"], *(None if v is None else v.float() for v in (s["w1"], s["b1"])))
    if c["gate"]:
        h = h * _of_rows(s["g"], s)
    h = h * c["alpha"]
    if c["res"]:
        h = s["r"].float() + h
    w = _of_rows(s["w2"], s)
    y = _plain_normed(h, c["pre"], w + 1 if c["rows"] else w, _of_rows(s["b2"], s))
    return ((h.to(DT[c["r"]]),) if _has_h(c) else ()) + _plain_out(y, c["out"])


def _has_h(c):
    return c["res"] or c["post"] != "none"


def _plain_quant(s):
    return _plain_int8(s["x"].float())


def _plain_product(s):
    x, w = s["x"], s["w"]
    total = 0
    for lo in range(0, x.shape[1], 1024):        # sums of 1024 products are whole numbers below 2^24
        total = total + torch.matmul(x[:, lo: lo + 1024].float(), w[:, lo: lo + 1024].float().t()).int()
    y = total.float() * s["xs"][:, None] * s["ws"]
    return (y if s["b"] is None else y + s["b"]).to(DT[s["case"]["y"]])


def _plain_glu(s):
    c, a = s["case"], s["a"].float()
    if c["act"] == "silu":
        y = a / (1 + torch.exp(-a))
    elif c["act"] == "gelu":
        y = 0.5 * a * (1 + torch.erf(a * math.sqrt(0.5)))
    else:
        y = 0.5 * a * (1 + torch.tanh(math.sqrt(2 / math.pi) * (a + 0.044715 * a * a * a)))
    if c["gated"]:
        y = y * s["b"].float()
    return _plain_out(y, c["out"])


# ---- the library's operators ----------------------------------------------------------------
def _kept(s, make):
    """A user's output buffers and handles, made at the first pass and kept with its inputs."""
    if "kept" not in s:
        s["kept"] = make()
    return s["kept"]


def _empty(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _code(E, name):
    return {"bf16": E.BF16, "fp16": E.FP16, "fp32": E.FP32, "e4m3": E.FP8_E4M3, "int8": E.INT8}[name]


def _outputs(m, n, out):
    scale = (m, _cdiv(n, 128)) if out == "e4m3" else (m,)
    return _empty((m, n), DT[out]), _empty(scale, torch.float32) if out in ("e4m3", "int8") else None


def _values_of(y, scale, out):
    """What a quantised output stands for, where it is not returned as it is."""
    if out == "e4m3":
        return y, scale
    if out == "int8":
        return torch.mul(y, scale[:, None], out=_empty(y.shape, torch.bfloat16)), scale
    return (y,)


def _own_rope(s, E, stream):
    c = s["case"]

    def make():
        kind = {"none": E.ROPE_PLAIN, "linear": E.ROPE_LINEAR, "base": E.ROPE_BASE, "turns": E.ROPE_TURNS,
                "index": E.ROPE_INDEX}[c["stretch"]]
        low, high = (INDEX_LOW, INDEX_HIGH) if c["stretch"] == "index" else (LOW, HIGH)
        table = torch.from_numpy(E.rope_freqs(c["rot"], BASE, kind, factor=FACTOR, trained_len=TRAINED, low=low, high=high)).cuda()
        q, k = _empty(s["q"].shape, DT[c["dtype"]]), _empty(s["k"].shape, DT[c["dtype"]])
        row = s["q"].stride(0)
        where = dict(d_pos=s["pos"].data_ptr()) if "pos" in s else dict(d_cu=s["cu"].data_ptr(), d_len=s["len"].data_ptr(),
                                                                       n_req=c["requests"])
        call = E.rope_call(s["q"].data_ptr(), q.data_ptr(), table.data_ptr(), s["tokens"], c["q_heads"], c["dim"], _code(E, c["dtype"]),
                           d_k=s["k"].data_ptr() if c["k_heads"] else 0, d_k_out=k.data_ptr() if c["k_heads"] else 0,
                           k_heads=c["k_heads"], rot_dim=c["rot"], rot_first=c["first"],
                           layout=E.ROPE_HALF if c["layout"] == "half" else E.ROPE_PAIRS, q_row=row, k_row=row,
                           amplitude=_amplitude(c), **where)
        return call, q, k, table

    call, q, k, _ = _kept(s, make)
    E.rope(call, stream)
    return q, k


def _own_norm(s, E, stream):
    c = s["case"]
    m, n = c["m"], c["n"]

    def make():
        kind = {"none": E.NORM_NONE, "rms": E.NORM_RMS, "layer": E.NORM_LAYER}
        y, scale = _outputs(m, n, c["out"])
        h = _empty((m, n), DT[c["r"]]) if _has_h(c) else None
        ld = s["w2"].stride(0) if c["rows"] else 0
        call = E.norm_call(s["x"].data_ptr(), m, n, x_dtype=_code(E, c["x"]), d_res=_ptr(s["r"]), d_res_out=_ptr(h),
                           res_dtype=_code(E, c["r"]), d_y=y.data_ptr(), y_dtype=_code(E, c["out"]), d_y_scale=_ptr(scale),
                           post=kind[c["post"]], d_post_w=_ptr(s["w1"]), d_post_b=_ptr(s["b1"]), d_gate=_ptr(s["g"]), gate_ld=ld,
                           alpha=c["alpha"], pre=kind[c["pre"]], d_w=s["w2"].data_ptr(), d_b=_ptr(s["b2"]), w_ld=ld, b_ld=ld,
                           w_dtype=_code(E, c["w"]), group_rows=c["rows"], w_plus_one=bool(c["rows"]), eps=EPS)
        return call, h, y, scale

    call, h, y, scale = _kept(s, make)
    E.norm(call, stream)
    return ((h,) if h is not None else ()) + _values_of(y, scale, c["out"])


def _own_quant(s, E, stream):
    c = s["case"]
    q, scale = _kept(s, lambda: _outputs(c["m"], c["k"], "int8"))
    E.quant_i8_row(s["x"].data_ptr(), _code(E, c["dtype"]), c["m"], c["k"], q.data_ptr(), scale.data_ptr(), stream=stream)
    return q, scale


def _own_product(s, E, stream):
    c = s["case"]
    m, n, k = c["m"], c["n"], c["k"]
    y, room = _kept(s, lambda: (_empty((m, n), DT[c["y"]]), _empty(E.gemm_i8_scaled_workspace(m, n, k), torch.uint8)))
    E.gemm_i8_scaled(s["x"].data_ptr(), s["xs"].data_ptr(), s["w"].data_ptr(), s["ws"].data_ptr(), y.data_ptr(), m, n, k,
                     y_dtype=_code(E, c["y"]), d_bias=_ptr(s["b"]), d_ws=room.data_ptr(), ws_bytes=room.numel(), stream=stream)
    return y


def _own_glu(s, E, stream):
    c = s["case"]
    y, scale = _kept(s, lambda: _outputs(c["m"], c["n"], c["out"]))
    row = s["a"].stride(0)
    E.glu(s["a"].data_ptr(), _ptr(s["b"]), _code(E, c["dtype"]), c["m"], c["n"],
          {"silu": E.ACT_SILU, "gelu": E.ACT_GELU, "gelu_tanh": E.ACT_GELU_TANH}[c["act"]], y.data_ptr(), _code(E, c["out"]),
          d_y_scale=_ptr(scale), a_row=row, b_row=row, stream=stream)
    return _values_of(y, scale, c["out"])


_PLAIN = {"rope": _plain_rope, "norm": _plain_norm, "quant": _plain_quant, "product": _plain_product, "glu": _plain_glu}
_OWN = {"rope": _own_rope, "norm": _own_norm, "quant": _own_quant, "product": _own_product, "glu": _own_glu}


def run(state):
    if own:
        from paper_2609_34185_amd import entropack as E
        return _OWN[state["case"]["op"]](state, E, torch.cuda.current_stream().cuda_stream)
    return _PLAIN[state["case"]["op"]](state)


# ---- the definitions in 64 bits -----------------------------------------------------------
def _exact_e4m3(y):
    """Codes and scales of blocks of 128 in a row, halves to even."""
    m, n = y.shape
    padded = torch.zeros((m, _cdiv(n, 128) * 128), dtype=torch.float64, device="cuda")
    padded[:, :n] = y
    blocks = padded.view(m, -1, 128)
    top = blocks.abs().amax(2, keepdim=True)
    scale = torch.where(top > 0, top / 448, 1.0)
    v = blocks / scale
    _, e = torch.frexp(v.abs())
    step = torch.ldexp(torch.ones_like(v), e.clamp(min=-5) - 4)
    return ((v / step).round() * step).clamp(-448, 448).view(m, -1)[:, :n], scale[:, :, 0]


def _exact_out(y, out):
    if out == "e4m3":
        return _exact_e4m3(y)
    if out == "int8":
        top = y.abs().amax(1, keepdim=True)
        scale = torch.where(top > 0, top / 127, 1.0)
        return (y / scale).round() * scale, scale[:, 0]
    return (y,)


def _slices(m, n):
    step = max(1, (1 << 25) // n)
    return [slice(r, min(r + step, m)) for r in range(0, m, step)]


def _joined(parts):
    return tuple(torch.cat(p) for p in zip(*parts))


def _exact_rope(c, s):
    cached, new = _counts(c)
    where = s["pos"].tolist() if "pos" in s else [a + i for a, b in zip(cached, new) for i in range(b)]
    rates, rot = [], c["rot"]
    for i in range(rot // 2):
        base = BASE * FACTOR ** (rot / (rot - 2)) if c["stretch"] == "base" else BASE
        rate = base ** (-2 * i / rot)
        keep = 1.0
        if c["stretch"] == "linear":
            keep = 0.0
        elif c["stretch"] == "turns":
            keep = min(1.0, max(0.0, (TRAINED * rate / (2 * math.pi) - LOW) / (HIGH - LOW)))
        elif c["stretch"] == "index":
            lo, hi = [rot * math.log(TRAINED / (2 * math.pi * t)) / (2 * math.log(BASE)) for t in (INDEX_HIGH, INDEX_LOW)]
            lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rot - 1)
            keep = 1 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
        rates.append(rate * (keep + (1 - keep) / FACTOR))
    turn = torch.polar(torch.full((1, 1), _amplitude(c), dtype=torch.float64, device="cuda"),
                       torch.tensor(where, dtype=torch.float64, device="cuda")[:, None] * torch.tensor(rates, dtype=torch.float64, device="cuda"))
    outs = []
    for x in (s["q"], s["k"]):
        y = x.double()
        i = torch.arange(rot // 2, device="cuda")
        one, two = (c["first"] + i, c["first"] + rot // 2 + i) if c["layout"] == "half" else (c["first"] + 2 * i, c["first"] + 2 * i + 1)
        z = torch.complex(y[:, :, one], y[:, :, two]) * turn[:, None]
        y[:, :, one], y[:, :, two] = z.real, z.imag
        outs.append(y)
    return tuple(outs)


def _exact_norm(c, s):
    def normed(x, kind, w, b):
        if kind == "none":
            return x
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        x = (x - mean) / torch.sqrt(var + EPS) if kind == "layer" else x / torch.sqrt((x * x).sum(1, keepdim=True) / x.shape[1] + EPS)
        return x * w + (0 if b is None else b)

    def rows(v, at):
        group = torch.arange(at.start, at.stop, device="cuda") // (c["rows"] or c["m"])
        return None if v is None else v.double()[group]

    parts = []
    for at in _slices(c["m"], c["n"]):
        u = normed(s["x"][at].double(), c["post"], *(None if v is None else v.double() for v in (s["w1"], s["b1"])))
        if c["gate"]:
            u = u * rows(s["g"], at)
        h = c["alpha"] * u
        if c["res"]:
            h += s["r"][at].double()
        y = normed(h, c["pre"], rows(s["w2"], at) + (1 if c["rows"] else 0), rows(s["b2"], at))
        parts.append(((h,) if _has_h(c) else ()) + _exact_out(y, c["out"]))
    return _joined(parts)


def _exact_glu(c, s):
    parts = []
    for at in _slices(c["m"], c["n"]):
        a = s["a"][at].double()
        if c["act"] == "silu":
            y = a * torch.sigmoid(a)
        elif c["act"] == "gelu":
            y = a * torch.special.ndtr(a)
        else:       # (1 + tanh z) / 2 is the logistic function of 2 z
            y = a * torch.sigmoid(math.sqrt(8 / math.pi) * (a + 0.044715 * a ** 3))
        if c["gated"]:
            y = y * s["b"][at].double()
        parts.append(_exact_out(y, c["out"]))
    return _joined(parts)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rope":
        return _exact_rope(c, s)
    if c["op"] == "norm":
        return _exact_norm(c, s)
    if c["op"] == "quant":
        return None, s["x"].double().abs().amax(1) / 127
    if c["op"] == "product":
        y = torch.zeros((c["m"], c["n"]), dtype=torch.float64, device="cuda")
        for lo in range(0, c["k"], 4096):
            y += s["x"][:, lo: lo + 4096].double() @ s["w"][:, lo: lo + 4096].double().t()
        y *= s["xs"].double()[:, None]
        y *= s["ws"].double()
        return y if s["b"] is None else y + s["b"].double()
    return _exact_glu(c, s)
