"""GPU tests of the operators on rows between products: the INT8 quantiser (ep_quant_i8_row), bit for
bit against its definition in numpy; norms with residual and gate (ep_norm) and the gated activation
(ep_glu) with FP32 outputs against 64 bits, every element within a bound derived from how it is
computed; their other outputs bit for bit against those FP32 values rounded, or quantised by the
quantisers.

The bounds.  A sum over a row of up to 65536: a thread adds up to 64 values, a wave's 64 lanes add in
6 steps, up to 16 waves in 15: 85 roundings of 2^-24 at most, of what is added up.  A mean is off by
(85 + 2) of mean |v|; 1 / sqrt(mean square + eps) by half the sum's error and 4 roundings, below 48,
and where v is off by e, by mean(|v| |e|) over the mean square.  With u, h and y's terms S_u = (|x| +
mean |x|) r |w| + |b| for layer norm (without the mean for RMS), S_h = |res| + |alpha g| S_u and S_y
from S_h likewise, every stage is off by at most 160 2^-24 of its S: 87 for the mean, 48 for r, 8
roundings by the elements.  Two stages of norms add up: 320 2^-24 S_y.
"""
import math
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def say(*a):
    print(*a, flush=True, file=sys.stderr)


@pytest.fixture(scope="module")
def E():
    from paper_2609_34185_amd import entropack
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    entropack.lib()
    return entropack


def stream():
    return torch.cuda.current_stream().cuda_stream


def code(E, name):
    return {"bf16": E.BF16, "fp16": E.FP16, "fp32": E.FP32, "e4m3": E.FP8_E4M3, "int8": E.INT8}[name]


# ---- INT8 quantiser --------------------------------------------------------------------
def quant_ref(x):
    """Codes and scales of float32 x by the definition, in float32 arithmetic."""
    s = (np.abs(x).max(1) * (np.float32(1) / np.float32(127))).astype(np.float32)
    s = np.where(s == 0, np.float32(1), s)
    return np.clip(np.rint((x / s[:, None]).astype(np.float32)), -127, 127).astype(np.int8), s


def quant_gpu(E, x, dtype):
    m, k = x.shape
    q = torch.full((m + 1, k), 0x6E, dtype=torch.int8, device="cuda")          # a row of sentinels
    s = torch.full((m + 1,), -7.0, dtype=torch.float32, device="cuda")
    E.quant_i8_row(x.data_ptr(), code(E, dtype), m, k, q.data_ptr(), s.data_ptr(), x_row=x.stride(0), stream=stream())
    torch.cuda.synchronize()
    assert (q[m] == 0x6E).all() and s[m] == -7.0
    return q[:m].cpu().numpy(), s[:m].cpu().numpy()


LENGTHS = [16, 128, 144, 256, 272, 512, 528, 1024, 1040, 4112, 5120, 8192, 8208, 17408, 32768, 32784, 65536]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("k", LENGTHS)
@pytest.mark.parametrize("m", [1, 5, 67])
def test_quant_matches_definition(E, m, k, dtype):
    say(f"  quant {m}x{k} {dtype}")
    rng = np.random.default_rng([31, m, k])
    x = rng.standard_normal((m, k)) * np.exp(rng.standard_normal((m, 1)))
    x[rng.random((m, k)) < 0.3] = 0.0
    x[:, ::97] *= 30
    x[m // 2] = 0.0
    t = torch.from_numpy(x).to(TYPES[dtype]).cuda()
    q, s = quant_gpu(E, t, dtype)
    rq, rs = quant_ref(t.float().cpu().numpy())
    assert np.array_equal(s.view(np.uint32), rs.view(np.uint32)) and np.array_equal(q, rq)


def test_quant_extremes_and_strided_rows(E):
    """Rows of subnormals (scales that underflow or are subnormal themselves), of the largest values and
    of ties between two codes, inside a wider matrix."""
    k = 272
    x = np.zeros((7, k + 48), np.float32)
    x[1] = 1e-45
    x[2] = np.linspace(-3e-43, 3e-43, k + 48, dtype=np.float32)
    x[3] = np.linspace(-1e-38, 1e-38, k + 48, dtype=np.float32)
    x[4] = np.linspace(-3.4e38, 3.4e38, k + 48, dtype=np.float32)
    x[5] = np.linspace(-1e-20, 1e-20, k + 48, dtype=np.float32)
    x[6] = np.arange(k + 48, dtype=np.float32) % 127 + 0.5
    x[6, 16] = 127.0
    part = torch.from_numpy(x).cuda()[:, 16: 16 + k]
    q, s = quant_gpu(E, part, "fp32")
    rq, rs = quant_ref(x[:, 16: 16 + k])
    assert np.array_equal(s.view(np.uint32), rs.view(np.uint32)) and np.array_equal(q, rq)


@pytest.mark.parametrize("k", [64, 256, 2048, 40000])
def test_quant_non_finite_rows_show(E, k):
    """A NaN or infinity makes its row's scale one, and leaves the other rows alone."""
    x = torch.randn((9, k), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    clean_q, clean_s = quant_gpu(E, x.cuda(), "bf16")
    x[0, 5], x[4, k - 1], x[7, 30] = float("nan"), float("inf"), float("-inf")
    q, s = quant_gpu(E, x.cuda(), "bf16")
    rest = [1, 2, 3, 5, 6, 8]
    assert np.isnan(s[0]) and np.isinf(s[4]) and np.isinf(s[7])
    assert np.array_equal(q[rest], clean_q[rest]) and np.array_equal(s[rest], clean_s[rest])


# ---- norm ---------------------------------------------------------------------------------
def normed(x, e, kind, w, b, eps):
    """N(x) w + b in float64 and, from what x is off by, what that is off by and its own S."""
    if kind == "none":
        return x, e
    n = x.shape[1]
    size = np.abs(x)
    mean = x.mean(1, keepdims=True) if kind == "layer" else 0.0
    spread = np.abs(x).mean(1, keepdims=True) if kind == "layer" else 0.0
    d = x - mean
    r = 1 / np.sqrt((d * d).sum(1, keepdims=True) / n + eps)
    s = (size + spread) * r * np.abs(w) + np.abs(b)
    moved = e + (e.mean(1, keepdims=True) if kind == "layer" else 0.0)
    bent = np.abs(d) * r * r * (np.abs(d) * moved).mean(1, keepdims=True)
    return d * r * w + b, (moved + bent) * r * np.abs(w) + 160 * 2.0 ** -24 * s


def norm_ref(a):
    """h and y in float64, and how far off each may be."""
    def wide(t):
        return None if t is None else t.double().cpu().numpy()
    x = wide(a["x"])
    m, n = x.shape
    group = np.arange(m) // a["rows"] if a["rows"] else np.zeros(m, int)
    zero = np.zeros_like(x)
    vec = lambda t, other: other if t is None else wide(t)[group] if t.dim() == 2 else wide(t)  # noqa: E731
    u, e = normed(x, zero, a["post"], vec(a["w1"], 1.0), vec(a["b1"], 0.0), a["eps"])
    g = vec(a["g"], 1.0) * a["alpha"]
    h, e = g * u, np.abs(g) * (e + 3 * 2.0 ** -24 * np.abs(u))
    if a["r"] is not None:
        h = h + wide(a["r"])
        e = e + 2.0 ** -24 * (np.abs(h) + e)
    y, f = normed(h, e, a["pre"], vec(a["w2"], 1.0) + (1.0 if a["plus"] else 0.0), vec(a["b2"], 0.0), a["eps"])
    return h, e, y, f


def norm_gpu(E, a, y_name, x_row=None):
    m, n = a["x"].shape
    ptr = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
    kind = {"none": E.NORM_NONE, "rms": E.NORM_RMS, "layer": E.NORM_LAYER}
    name = {torch.bfloat16: "bf16", torch.float16: "fp16", torch.float32: "fp32"}
    r_dtype = a["r"].dtype if a["r"] is not None else a["h_dtype"]
    h = torch.full((m + 1, n), 7.0, dtype=r_dtype, device="cuda")
    y = scale = None
    if a["pre"] != "none":
        dt = {"e4m3": torch.uint8, "int8": torch.int8}.get(y_name) or TYPES[y_name]
        y = torch.full((m + 1, n), 7, dtype=dt, device="cuda")
        if y_name in ("e4m3", "int8"):
            scale = torch.full((m + 1, -(-n // 128) if y_name == "e4m3" else 1), -7.0, device="cuda")
    ld = lambda t: t.stride(0) if t is not None and t.dim() == 2 else 0  # noqa: E731
    w = next((t for t in (a["w1"], a["b1"], a["g"], a["w2"], a["b2"]) if t is not None), None)
    call = E.norm_call(a["x"].data_ptr(), m, n, x_dtype=code(E, name[a["x"].dtype]), d_res=ptr(a["r"]), d_res_out=h.data_ptr(),
                       res_dtype=code(E, name[r_dtype]), d_y=ptr(y), y_dtype=code(E, y_name), d_y_scale=ptr(scale), post=kind[a["post"]],
                       d_post_w=ptr(a["w1"]), d_post_b=ptr(a["b1"]), d_gate=ptr(a["g"]), gate_ld=ld(a["g"]), alpha=a["alpha"],
                       pre=kind[a["pre"]], d_w=ptr(a["w2"]), d_b=ptr(a["b2"]), w_ld=ld(a["w2"]), b_ld=ld(a["b2"]),
                       w_dtype=code(E, name[w.dtype]) if w is not None else 0, group_rows=a["rows"], w_plus_one=a["plus"], eps=a["eps"],
                       x_row=a["x"].stride(0) if m > 1 else 0, res_row=a["r"].stride(0) if m > 1 and a["r"] is not None else 0)
    E.norm(call, stream())
    torch.cuda.synchronize()
    for t, was in ((h, 7.0), (y, 7), (scale, -7.0)):
        assert t is None or (t[m] == was).all()
    return h[:m], None if y is None else y[:m], None if scale is None else scale[:m]


def norm_args(m, n, *, post="none", pre="rms", res=True, gate=False, rows=0, x="bf16", r="bf16", w="bf16", w1=True, w2=True, bias=False,
              plus=False, alpha=1.0, eps=1e-6, seed=0, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    groups = -(-m // rows) if rows else 1

    def rand(*shape):
        return torch.randn(shape, generator=g)

    def hidden(dtype, size):
        t = rand(m, n + 32) * torch.exp(0.5 * rand(m, 1)) * size + offset
        t[:, ::101] *= 20
        return t.to(TYPES[dtype]).cuda()[:, 16: 16 + n]
    mod = (0.3 * rand(groups, 3 * n)).to(TYPES[w]).cuda()
    own = lambda i: mod[:, i * n: (i + 1) * n] if rows else mod[0, i * n: (i + 1) * n]  # noqa: E731
    return dict(x=hidden(x, 1.0), r=hidden(r, 3.0) if res else None, h_dtype=TYPES[r],
                w1=(1 + 0.2 * rand(n)).to(TYPES[w]).cuda() if post != "none" and w1 else None,
                b1=(0.1 * rand(n)).to(TYPES[w]).cuda() if post != "none" and bias else None, g=own(0) if gate else None,
                w2=own(1) if w2 else None, b2=own(2) if bias else None, post=post, pre=pre, rows=rows, plus=plus, alpha=alpha, eps=eps)


def check_norm(E, a):
    h, y, _ = norm_gpu(E, a, "fp32")
    wh, eh, wy, ey = norm_ref(a)
    half = torch.finfo(h.dtype).eps / 2
    assert (np.abs(h.double().cpu().numpy() - wh) <= eh + half * (np.abs(wh) + eh) + 2.0 ** -25 * (h.dtype == torch.float16)).all()
    assert (np.abs(y.double().cpu().numpy() - wy) <= ey + 2.0 ** -24 * (np.abs(wy) + ey)).all()
    m, n = y.shape
    for t in ("bf16", "fp16"):
        h2, y2, _ = norm_gpu(E, a, t)
        assert torch.equal(h2, h) and torch.equal(y2, y.to(TYPES[t]))
    if n % 16:
        return
    _, q, s = norm_gpu(E, a, "e4m3")
    rq, rs = torch.empty((m, n), dtype=torch.uint8, device="cuda"), torch.empty((m, -(-n // 128)), device="cuda")
    y = y.contiguous()
    E.quant_fp8_block(y.data_ptr(), E.FP32, m, n, rq.data_ptr(), rs.data_ptr(), stream=stream())
    assert torch.equal(q, rq) and torch.equal(s, rs)
    _, q, s = norm_gpu(E, a, "int8")
    rq, rs = quant_gpu(E, y, "fp32")
    assert np.array_equal(q.cpu().numpy(), rq) and np.array_equal(s[:, 0].cpu().numpy(), rs)


@pytest.mark.parametrize("m,n", [(1, 8), (1, 5120), (5, 24), (67, 128), (9, 136), (33, 256), (7, 264), (5, 512), (6, 520), (3, 1024), (4, 2056),
                                 (130, 3840), (3, 8192), (2, 8208), (5, 17408), (2, 32776), (3, 65536)])
@pytest.mark.parametrize("post,pre", [("none", "rms"), ("rms", "rms"), ("layer", "layer"), ("none", "layer")])
def test_norm_matches_definition(E, m, n, post, pre):
    say(f"  norm {m}x{n} {post} {pre}")
    check_norm(E, norm_args(m, n, post=post, pre=pre, bias=post != "rms", seed=m * n))


@pytest.mark.parametrize("kw", [
    dict(res=False), dict(res=False, w2=False), dict(post="rms", w1=False, w2=False, res=False, alpha=0.5), dict(gate=True, alpha=-0.25),
    dict(gate=True, rows=7, plus=True, bias=True, pre="layer"), dict(gate=True, rows=1, w="fp32", plus=True), dict(rows=1000, bias=True, gate=True),
    dict(x="fp32", r="fp32", w="fp32", post="layer", bias=True), dict(x="fp16", r="fp16", w="fp16", post="rms"),
    dict(x="fp32", r="bf16", w="fp16"), dict(x="bf16", r="fp32", w="bf16", post="rms", bias=True), dict(eps=1e-2, plus=True),
    dict(pre="layer", offset=40.0), dict(post="layer", pre="layer", offset=-300.0, x="fp32", r="fp32", w="fp32")])
def test_norm_forms(E, kw):
    """What may be left out, types apart from each other, groups of rows, rows far from zero."""
    say("  norm", kw)
    for m, n in ((23, 144), (10, 640), (23, 2064)):
        check_norm(E, norm_args(m, n, seed=n, **kw))


def test_norm_only_the_sum(E):
    """Without a norm of h, and in place."""
    a = norm_args(11, 1024, post="rms", gate=True, pre="none", seed=5)
    h, y, _ = norm_gpu(E, a, "bf16")
    wh, eh, _, _ = norm_ref(a)
    assert y is None and (np.abs(h.double().cpu().numpy() - wh) <= eh + 2.0 ** -8 * (np.abs(wh) + eh)).all()
    r = a["r"].contiguous().clone()
    E.norm(E.norm_call(a["x"].data_ptr(), 11, 1024, x_row=a["x"].stride(0), d_res=r.data_ptr(), d_res_out=r.data_ptr(), post=E.NORM_RMS,
                       d_post_w=a["w1"].data_ptr(), d_gate=a["g"].data_ptr(), pre=E.NORM_NONE), stream())
    torch.cuda.synchronize()
    assert torch.equal(r, h)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("n", [64, 256, 1024, 4096, 65536])
def test_norm_extreme_rows(E, kind, n):
    """Rows of zeros, of values whose squares or sums pass FP32's range or fall below it, and of one
    value: every one as in 64 bits, within the bound of its own terms."""
    x = torch.zeros((8, n))
    g = torch.Generator().manual_seed(n)
    for i, size in enumerate((0.0, 1e30, 3e37, 1e-30, 1e-42, 1.0, 1e18)):
        x[i] = torch.randn(n, generator=g).clamp(-4, 4) * size
    x[5, 3] = 3e38
    x[7] = 2e38                                            # sums beyond the range
    # 1e-42 is subnormal: where a mean square is far below eps the factor is 1 / sqrt(eps) and the row's
    # own roundings count, one unit of 2^-149 for each of its few operations
    a = dict(x=x.cuda(), r=None, h_dtype=torch.float32, w1=None, b1=None, g=None, w2=None, b2=None, post="none", pre=kind, rows=0, plus=False,
             alpha=1.0, eps=1e-6)
    h, y, _ = norm_gpu(E, a, "fp32")
    wh, eh, wy, ey = norm_ref(a)
    assert torch.equal(h, a["x"])
    room = 8 * 2.0 ** -149 * 1e3
    # the row of one value: its deviations from the mean are all rounding, 87 2^-24 of it, and so is what
    # they are divided by
    rows = [i for i in range(8) if not (kind == "layer" and i == 7)]
    got = y.double().cpu().numpy()
    assert (np.abs(got - wy) <= ey + 2.0 ** -24 * (np.abs(wy) + ey) + room)[rows].all()
    assert np.isfinite(got).all()


def test_norm_non_finite_rows_stay_alone(E):
    for n in (128, 512, 5120):
        a = norm_args(9, n, post="rms", seed=3)
        h0, y0, _ = norm_gpu(E, a, "bf16")
        h0, y0 = h0.clone(), y0.clone()
        a["x"][2, 5], a["r"][6, 7] = float("nan"), float("inf")
        h, y, _ = norm_gpu(E, a, "bf16")
        rest = [0, 1, 3, 4, 5, 7, 8]
        assert torch.equal(h[rest], h0[rest]) and torch.equal(y[rest], y0[rest])
        assert not torch.isfinite(y[2]).any() and not torch.isfinite(y[6]).all()


# ---- gated activation -------------------------------------------------------------------------
def act_ref(a, act):
    if act == "silu":
        return a / (1 + np.exp(-a))
    if act == "gelu":
        return np.array([0.5 * v * math.erfc(-v * math.sqrt(0.5)) for v in a.reshape(-1)]).reshape(a.shape)
    return a / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3)))


def glu_gpu(E, a, b, act, y_name):
    m, n = a.shape
    name = {torch.bfloat16: "bf16", torch.float16: "fp16", torch.float32: "fp32"}[a.dtype]
    dt = {"e4m3": torch.uint8, "int8": torch.int8}.get(y_name) or TYPES[y_name]
    y = torch.full((m + 1, n), 7, dtype=dt, device="cuda")
    scale = torch.full((m + 1, -(-n // 128) if y_name == "e4m3" else 1), -7.0, device="cuda")
    E.glu(a.data_ptr(), 0 if b is None else b.data_ptr(), code(E, name), m, n,
          {"silu": E.ACT_SILU, "gelu": E.ACT_GELU, "gelu_tanh": E.ACT_GELU_TANH}[act], y.data_ptr(), code(E, y_name),
          d_y_scale=scale.data_ptr() if y_name in ("e4m3", "int8") else 0, a_row=a.stride(0), b_row=0 if b is None else b.stride(0),
          stream=stream())
    torch.cuda.synchronize()
    assert (y[m] == 7).all() and (scale[m] == -7.0).all()
    return y[:m], scale[:m]


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m,n,gated", [(1, 8, True), (3, 144, True), (5, 640, False), (61, 1040, True), (2, 17408, True), (1, 65536, True),
                                       (130, 72, False)])
def test_glu_matches_definition(E, m, n, gated, dtype, act):
    """With FP32 outputs.  SiLU: exp is off by 2 units of itself (a library function's bound, and
    its argument is exact), 1 + exp, the quotient and the product by half a unit each: below 8 2^-24 of the
    value.  GELU: erfc's argument is off by 2 roundings, which move it by x^2 of them, and erfc itself by up
    to 16 units: (24 + 4 a^2) 2^-24 of the value.  By tanh: the exponent z is off by 5 roundings, which
    move it by z of them: (8 + 8 |z|) 2^-24.  Values of exp, erfc or the quotient below FP32's normal range
    are off by units of 2^-149 instead, times the other factor."""
    say(f"  glu {m}x{n} {dtype} {act} {'gated' if gated else 'alone'}")
    g = torch.Generator().manual_seed(m + n)
    ab = torch.randn((m, 2 * n), generator=g) * 3
    ab[:, ::53] *= 8
    ab = ab.to(TYPES[dtype]).cuda()
    a, b = ab[:, :n], ab[:, n:] if gated else None
    y, _ = glu_gpu(E, a, b, act, "fp32")
    x = a.double().cpu().numpy()
    with np.errstate(over="ignore"):
        want = act_ref(x, act)
    z = np.abs(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))
    units = {"silu": 8, "gelu": 24 + 4 * x * x, "gelu_tanh": 8 + 8 * z}[act] + 2
    other = 1.0 if b is None else b.double().cpu().numpy()
    tol = units * 2.0 ** -24 * np.abs(want * other) + 64 * 2.0 ** -149 * (1 + np.abs(x)) * (1 + np.abs(other))
    assert (np.abs(y.double().cpu().numpy() - want * other) <= tol).all()
    for t in ("bf16", "fp16"):
        assert torch.equal(glu_gpu(E, a, b, act, t)[0], y.to(TYPES[t]))
    if n % 16:
        return
    q, s = glu_gpu(E, a, b, act, "e4m3")
    rq, rs = torch.empty((m, n), dtype=torch.uint8, device="cuda"), torch.empty((m, -(-n // 128)), device="cuda")
    E.quant_fp8_block(y.data_ptr(), E.FP32, m, n, rq.data_ptr(), rs.data_ptr(), stream=stream())
    assert torch.equal(q, rq) and torch.equal(s, rs)
    q, s = glu_gpu(E, a, b, act, "int8")
    rq, rs = quant_gpu(E, y, "fp32")
    assert np.array_equal(q.cpu().numpy(), rq) and np.array_equal(s[:, 0].cpu().numpy(), rs)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_glu_large_and_non_finite_values(E, act):
    """Far out the activation is its argument or zero; a NaN or infinity shows in its own value only."""
    a = torch.tensor([[0.0, -0.0, 100.0, -100.0, 1e30, -1e30, 3e38, -3e38, 1e-40, -1e-40, 20.0, -20.0, float("nan"), float("inf"), 1.0, 2.0]]).cuda()
    y = glu_gpu(E, a, None, act, "fp32")[0][0].tolist()
    assert y[0] == 0 and y[1] == 0 and y[2] == 100.0 and abs(y[3]) < 1e-40 and y[4] == a[0, 4] and y[5] == 0 and y[6] == a[0, 6] and y[7] == 0
    assert math.isnan(y[12]) and y[13] == math.inf and abs(y[14] - {"silu": 0.7310586, "gelu": 0.8413447, "gelu_tanh": 0.8411920}[act]) < 1e-6


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("bad", [-math.inf, math.nan])
def test_glu_what_overflowed_below_shows_in_every_output(E, bad, dtype, act):
    """-inf times 0 is a NaN for every activation: it shows in its own value of a wide output, and in
    the scale of its block or row of a quantised one, the others as without it."""
    a = torch.randn((5, 400), generator=torch.Generator().manual_seed(6)).to(TYPES[dtype]).cuda()
    outs = ("fp32", "bf16", "fp16", "e4m3", "int8")
    clean = [[t.clone() for t in glu_gpu(E, a, None, act, y)] for y in outs]
    a[2, 131] = bad
    keep = torch.ones((5, 400), dtype=torch.bool)
    for y_name, (y0, s0) in zip(outs, clean):
        y, s = glu_gpu(E, a, None, act, y_name)
        if y_name in ("e4m3", "int8"):
            block = 1 if y_name == "e4m3" else 0
            assert torch.isnan(s[2, block])
            other = torch.ones_like(s, dtype=torch.bool)
            other[2, block] = False
            assert torch.equal(s[other], s0[other])
            keep[2] = False
        else:
            assert torch.isnan(y[2, 131])
            keep[2, 131] = False
        assert torch.equal(y[keep], y0[keep])
        keep[2] = True


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_glu_error_by_its_steps(E, act, gated):
    """FP32 to FP32, in units of 2^-24 of the value; an operation that rounds adds one.
    exp: its argument's fraction of a power of two is off by 2^-24, 0.7 units of the result, and the instruction
    by one of its last places, 2: 2.7.  Reciprocal: an instruction within 2^-23, a step that squares that, and a
    rounding: 1.01.  Logistic function of Z, off by dz: 1 / (1 + e) is off by (2.7 + dz) e / (1 + e) + 1 + 1.01, the
    product adds 1; for Z < 0 the numerator is a e, another 1 and 2.7 + dz in all, of which 1 + e takes a share back.
    SiLU: Z is exact.  By tanh: Z = c a (1 + d a^2) has two rounded constants and four operations, 6 of |Z| at most.
    GELU: |a| Phi(-|a|) = |a| exp(-a^2 / 2) P(t), t = 1 / (1 + 0.24 |a|) off by 2.01 and P by 3.33 times that where it is
    steepest, at 0: 6.7; P's Horner steps 3.9 there, what P leaves out of the function 0.6, exp 2.7, three products
    and the last one 4: 17.9, less further out.  Above 0 it is taken from a: Phi(-a) / Phi(a) of 16.9, and 1.
    The other factor adds 1.  Where a step's result is below FP32's normal range it is off by 2^-150."""
    g = torch.Generator().manual_seed(12)
    far = torch.logspace(-44, 4, 16384, dtype=torch.float64)
    a = torch.cat((torch.linspace(-15, 15, 32768, dtype=torch.float64), far, -far)).float()[None]
    b = torch.randn(a.shape, generator=g) if gated else None
    y, _ = glu_gpu(E, a.cuda(), None if b is None else b.cuda(), act, "fp32")
    x = a.double().numpy()
    with np.errstate(over="ignore"):
        want = act_ref(x, act)
        z = 2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3) if act == "gelu_tanh" else x
        e = np.exp(-np.abs(z))
    if act == "gelu":
        below = np.array([0.5 * math.erfc(abs(v) * math.sqrt(0.5)) for v in x.reshape(-1)]).reshape(x.shape)   # Phi(-|a|)
        units = np.where(x < 0, 17.9, 1 + 16.9 * below / (1 - below))
    else:
        dz = 2.7 + (6 * np.abs(z) if act == "gelu_tanh" else 0)
        units = np.where(x < 0, dz + 4.01, dz * e / (1 + e) + 3.01)
    other = 1.0 if b is None else b.double().numpy()
    tol = (units + gated) * 2.0 ** -24 * np.abs(want * other) * (1 + 2.0 ** -18) + 2.0 ** -150 * (4 * (1 + np.abs(x)) * np.abs(other) + 1)
    off = np.abs(y.double().cpu().numpy() - want * other)
    assert (off <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m,n", [(1, 640), (67, 136), (9, 5120), (3, 17408)])
def test_row_operators_in_place_of_any_input(E, m, n, dtype):
    """y over a or b, y over x or the stream, the new stream over x: as into buffers of their own."""
    g = torch.Generator().manual_seed(n)
    a, b = (torch.randn((m, n), generator=g).to(TYPES[dtype]).cuda() for _ in range(2))
    act, name = E.ACT_GELU_TANH, code(E, dtype)
    want = glu_gpu(E, a, b, "gelu_tanh", dtype)[0]
    for i in range(2):
        x = [a.clone(), b.clone()]
        E.glu(x[0].data_ptr(), x[1].data_ptr(), name, m, n, act, x[i].data_ptr(), name, stream=stream())
        assert torch.equal(x[i], want) and torch.equal(x[1 - i], (a, b)[1 - i])
    h0, y0 = torch.empty_like(a), torch.empty_like(a)

    def norm(x, r, h, y):
        E.norm(E.norm_call(x.data_ptr(), m, n, x_dtype=name, res_dtype=name, y_dtype=name, d_res=r.data_ptr(), d_res_out=h.data_ptr(),
                           d_y=y.data_ptr(), post=E.NORM_LAYER, pre=E.NORM_RMS, alpha=0.5), stream())

    norm(a, b, h0, y0)
    for ih, iy in ((0, 1), (1, 0), (0, 2), (2, 0), (1, 2), (2, 1)):
        x = [a.clone(), b.clone(), torch.empty_like(a), torch.empty_like(a)]
        norm(x[0], x[1], x[ih], x[iy] if iy < 2 else x[3])
        assert torch.equal(x[ih], h0) and torch.equal(x[iy] if iy < 2 else x[3], y0), (ih, iy)


# ---- all of them ------------------------------------------------------------------------------
def test_row_operators_of_more_rows_than_a_grid_row_holds(E):
    """From 2^21 workgroups on a launch has more than one row of a grid: rows of a repeated batch get
    the batch's outputs."""
    n, step = 1024, 1 << 12
    times = (1 << 21) // step + 3
    m = step * times + 5
    if torch.cuda.mem_get_info()[0] < 8 * m * n:
        pytest.skip("needs more device memory")
    base = torch.randn((step, n), device="cuda").to(torch.bfloat16)
    x = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    for i in range(0, m, step):
        x[i: i + step] = base[: min(step, m - i)]
    q0, s0 = quant_gpu(E, base, "bf16")
    q, s = torch.empty((m, n), dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda")
    E.quant_i8_row(x.data_ptr(), E.BF16, m, n, q.data_ptr(), s.data_ptr(), stream=stream())
    q0, s0 = torch.from_numpy(q0).cuda(), torch.from_numpy(s0).cuda()
    for i in range(0, m, step):
        c = min(step, m - i)
        assert torch.equal(q[i: i + c], q0[:c]) and torch.equal(s[i: i + c], s0[:c])
    y0 = torch.empty_like(base)
    E.norm(E.norm_call(base.data_ptr(), step, n, d_y=y0.data_ptr()), stream())
    E.norm(E.norm_call(x.data_ptr(), m, n, d_res=0, d_y=x.data_ptr()), stream())      # a row is read before it is written
    for i in range(0, m, step):
        assert torch.equal(x[i: i + step], y0[: min(step, m - i)])
    del x, q
    torch.cuda.empty_cache()


def test_row_operators_repeat_their_bits(E):
    a = norm_args(300, 3840, post="rms", gate=True, seed=6)
    first = norm_gpu(E, a, "e4m3")
    for _ in range(3):
        for p, q in zip(first, norm_gpu(E, a, "e4m3")):
            assert torch.equal(p, q)


@pytest.mark.parametrize("m,n", [(1, 5120), (67, 2064), (9, 256)])
def test_row_operators_in_a_graph(E, m, n):
    """Captured on a stream of their own and replayed over other inputs: norm (the stream in place, y over
    x) and its product's other half, the activation and the quantiser, as called one by one."""
    g = torch.Generator().manual_seed(m + n)
    x, r, w, b = (torch.randn((rows, n), generator=g).to(torch.bfloat16).cuda() for rows in (m, m, 1, m))
    y, codes, q = torch.empty_like(x), torch.empty_like(x, dtype=torch.uint8), torch.empty_like(x, dtype=torch.int8)
    scale, rows = torch.empty((m, -(-n // 128)), device="cuda"), torch.empty(m, device="cuda")

    def call():
        s = stream()
        E.norm(E.norm_call(x.data_ptr(), m, n, d_res=r.data_ptr(), d_res_out=r.data_ptr(), d_y=x.data_ptr(), d_w=w.data_ptr(), alpha=0.5), s)
        E.glu(x.data_ptr(), b.data_ptr(), E.BF16, m, n, E.ACT_SILU, y.data_ptr(), stream=s)
        E.glu(x.data_ptr(), b.data_ptr(), E.BF16, m, n, E.ACT_SILU, codes.data_ptr(), E.FP8_E4M3, scale.data_ptr(), stream=s)
        E.quant_i8_row(y.data_ptr(), E.BF16, m, n, q.data_ptr(), rows.data_ptr(), stream=s)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call()
    for i in range(4):
        new = [torch.randn((m, n), generator=g).to(torch.bfloat16).cuda() for _ in range(3)]
        outs = []
        for replayed in (False, True):
            for t, value in zip((x, r, b), new):
                t.copy_(value)
            for t in (y, codes, q, scale, rows):
                t.zero_()
            graph.replay() if replayed else call()
            torch.cuda.synchronize()
            outs.append([t.clone() for t in (x, r, y, codes, scale, q, rows)])
        assert all(torch.equal(p, o) for p, o in zip(*outs)), i
        h = (new[1].double() + 0.5 * new[0].double())
        assert ((r.double() - h).abs() <= 2.0 ** -8 * h.abs() + 2.0 ** -22 * (new[1].double().abs() + new[0].double().abs())).all()
