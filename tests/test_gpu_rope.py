"""GPU tests of rotary positions (ep_rope) against the rotation in 64 bits, with angles in 50 decimal
digits, every element within a bound that is derived from how it is computed.

The bound: an angle is right to 2^-33 of a turn, rounded to FP32 and multiplied by a rounded
constant, at most pi / 4: 3 roundings of 2^-24, times 0.79, times a slope of at most 1; the series
adds under 2 roundings of values up to 1: cosine and sine are within 4 2^-24.  The amplitude's
product adds 1, the two products and their sum 2 more, each relative to |a| + |b| times the
amplitude: 8 2^-24 A (|a| + |b|), rounded up.  Then the rounding to the type: half a step.
"""
import math
import sys
from decimal import Decimal, getcontext

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494")


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
    return {"bf16": E.BF16, "fp16": E.FP16, "fp32": E.FP32}[name]


def turned(x, pos, rot, first, pairs, base=10000.0, inverse=False, amplitude=1.0):
    """x [tokens, heads, dim] in float64 rotated by its positions, and |a| + |b| of every pair."""
    getcontext().prec = 50
    theta = [Decimal(base) ** (Decimal(-2 * i) / rot) / (2 * PI) for i in range(rot // 2)]
    phi = np.array([[float((p * f) % 1) for f in theta] for p in (Decimal(int(q)) for q in pos)]) * (2 * math.pi)
    if inverse:
        phi = -phi
    co, si = np.cos(phi)[:, None] * amplitude, np.sin(phi)[:, None] * amplitude
    i = np.arange(rot // 2)
    one, two = (first + 2 * i, first + 2 * i + 1) if pairs else (first + i, first + rot // 2 + i)
    y, size = x.copy(), np.zeros_like(x)
    a, b = x[:, :, one], x[:, :, two]
    y[:, :, one], y[:, :, two] = a * co - b * si, a * si + b * co
    size[:, :, one] = size[:, :, two] = (np.abs(a) + np.abs(b)) * amplitude
    return y, size


def off(got, want, size, dtype):
    """How far got is past the bound, element by element (0: within)."""
    half = torch.finfo(TYPES[dtype]).eps / 2
    tol = 8 * 2.0 ** -24 * size
    tol = tol + (np.abs(want) + tol) * half + (2.0 ** -25 if dtype == "fp16" else 0)
    return np.maximum(np.abs(got.double().cpu().numpy() - want) - np.where(size > 0, tol, 0), 0).max(initial=0)


def table(E, rot, base=10000.0, **kw):
    return torch.from_numpy(E.rope_freqs(rot, base, **kw).view(np.int64)).cuda()


def case(tokens, q_heads, k_heads, dim, dtype, seed):
    """Queries and keys inside a fused projection's rows."""
    g = torch.Generator().manual_seed(seed)
    rows = torch.randn((tokens, (q_heads + 2 * k_heads + 1) * dim), generator=g).to(TYPES[dtype]).cuda()
    q = rows[:, : q_heads * dim].unflatten(1, (q_heads, dim))
    k = rows[:, q_heads * dim: (q_heads + k_heads) * dim].unflatten(1, (k_heads, dim)) if k_heads else None
    return rows, q, k


def positions(n, seed):
    """Small, far and extreme ones."""
    p = np.random.default_rng(seed).integers(0, 1 << 20, n)
    some = [0, 1, 2147483647, 131071, -1, -2147483648, 4095][:n]
    p[: len(some)] = some
    return p


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("tokens,q_heads,k_heads,dim,rot,first", [
    (1, 1, 0, 2, 2, 0), (1, 40, 8, 128, 128, 0), (7, 5, 1, 64, 64, 0), (33, 8, 2, 128, 64, 0), (9, 4, 4, 128, 32, 96), (17, 3, 1, 80, 20, 60),
    (5, 2, 1, 96, 96, 0), (12, 6, 2, 256, 256, 0), (8, 1, 1, 66, 6, 4), (3, 2, 2, 1024, 1024, 0), (40, 4, 2, 72, 48, 24)])
def test_rope_matches_definition(E, tokens, q_heads, k_heads, dim, rot, first, pairs, dtype):
    say(f"  rope {tokens} tokens {q_heads}/{k_heads} heads of {dim}, {rot} from {first}, pairs {pairs}, {dtype}")
    rows, q, k = case(tokens, q_heads, k_heads, dim, dtype, 3)
    pos = positions(tokens, 4)
    d_pos = torch.tensor(pos, dtype=torch.int32, device="cuda")
    freqs = table(E, rot)
    layout = E.ROPE_PAIRS if pairs else E.ROPE_HALF
    outs = [torch.full((tokens + 1, h, dim), 7.0, dtype=TYPES[dtype], device="cuda") for h in (q_heads, max(1, k_heads))]
    kw = dict(d_k=k.data_ptr(), d_k_out=outs[1].data_ptr(), k_heads=k_heads) if k_heads else {}
    E.rope(E.rope_call(q.data_ptr(), outs[0].data_ptr(), freqs.data_ptr(), tokens, q_heads, dim, code(E, dtype), rot_dim=rot,
                       rot_first=first, layout=layout, d_pos=d_pos.data_ptr(), q_row=rows.stride(0), k_row=rows.stride(0), **kw), stream())
    torch.cuda.synchronize()
    for x, y in ((q, outs[0]), (k, outs[1])):
        if x is None:
            continue
        want, size = turned(x.double().cpu().numpy(), pos, rot, first, pairs)
        assert off(y[:tokens], want, size, dtype) == 0 and (y[tokens] == 7.0).all()
    # in place, the rest of the rows untouched: the same bits
    before = rows.clone()
    if k_heads:
        kw["d_k_out"] = k.data_ptr()
    E.rope(E.rope_call(q.data_ptr(), q.data_ptr(), freqs.data_ptr(), tokens, q_heads, dim, code(E, dtype), rot_dim=rot, rot_first=first,
                       layout=layout, d_pos=d_pos.data_ptr(), q_row=rows.stride(0), q_out_row=rows.stride(0), k_row=rows.stride(0),
                       k_out_row=rows.stride(0), **kw), stream())
    torch.cuda.synchronize()
    assert torch.equal(q, outs[0][:tokens]) and (k is None or torch.equal(k, outs[1][:tokens]))
    used = (q_heads + k_heads) * dim
    assert torch.equal(rows[:, used:], before[:, used:])


@pytest.mark.parametrize("pairs", [False, True])
def test_rope_inverse_takes_it_back(E, pairs):
    """By the negative angles with the inverse amplitude: the input again, twice the bound off at most;
    and that is the gradient: <rope(x), g> = <x, inverse(g)> to FP32's sums."""
    rows, q, _ = case(19, 4, 0, 64, "fp32", 8)
    q = q.contiguous()
    pos = torch.tensor(positions(19, 9), dtype=torch.int32, device="cuda")
    freqs = table(E, 64)
    y, z, g, h = (torch.empty_like(q) for _ in range(4))

    def call(a, b, **kw):
        E.rope(E.rope_call(a.data_ptr(), b.data_ptr(), freqs.data_ptr(), 19, 4, 64, E.FP32, layout=E.ROPE_PAIRS if pairs else E.ROPE_HALF,
                           d_pos=pos.data_ptr(), **kw), stream())

    call(q, y, amplitude=1.25)
    call(y, z, amplitude=0.8, inverse=True)
    g.normal_()
    call(g, h, amplitude=1.25, inverse=True)
    torch.cuda.synchronize()
    _, size = turned(q.double().cpu().numpy(), pos.tolist(), 64, 0, pairs)
    # the second turn's pair is at most sqrt(2) the first's |a| + |b|; its own bound comes on top
    assert (np.abs((z - q).double().cpu().numpy()) <= 3 * 9 * 2.0 ** -24 * size).all()
    one, two = (y.double() * g.double()).sum(), (q.double() * h.double()).sum()
    assert abs(one - two) <= 2 * 9 * 2.0 ** -24 * 1.25 * 4 * float((q.double().abs().sum(2) * g.double().abs().amax(2)).sum())


@pytest.mark.parametrize("new,vec", [([1], 8), ([3, 0, 0, 5, 1, 0], 8), ([0, 0, 4], 1), ([1] * 70, 8), ([2, 0, 1] * 700, 8), ([1, 0] * 1024 + [5], 8),
                                     ([0] * 5000 + [3] + [0] * 2000 + [2], 1)])
def test_rope_positions_from_lengths(E, new, vec):
    """Positions from the requests' lengths, empty requests among them and rows after the last token,
    which stay as they were: bit for bit what given positions make of it."""
    dim, n = (64 if vec == 8 else 6), len(new)
    rng = np.random.default_rng(n)
    total, spare = sum(new), 5
    cached = rng.integers(0, 100000, n)
    q = torch.randn((total + spare, 2, dim), device="cuda").to(torch.bfloat16)
    cu = torch.tensor(np.concatenate(([0], np.cumsum(new))), dtype=torch.int32, device="cuda")
    lens = torch.tensor(cached + new, dtype=torch.int32, device="cuda")
    pos = np.concatenate([c + np.arange(m) for c, m in zip(cached, new)] or [[]])
    d_pos = torch.tensor(pos, dtype=torch.int32, device="cuda")
    freqs = table(E, dim)
    a, b = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    E.rope(E.rope_call(q.data_ptr(), a.data_ptr(), freqs.data_ptr(), total + spare, 2, dim, E.BF16, d_cu=cu.data_ptr(), d_len=lens.data_ptr(),
                       n_req=n), stream())
    E.rope(E.rope_call(q.data_ptr(), b.data_ptr(), freqs.data_ptr(), total, 2, dim, E.BF16, d_pos=d_pos.data_ptr()), stream())
    torch.cuda.synchronize()
    assert torch.equal(a, b) and (a[total:] == 7.0).all() and not (a[:total] == 7.0).all()


def test_rope_not_finite_values_stay_in_their_pair(E):
    q = torch.randn((4, 3, 64), device="cuda")
    pos = torch.arange(4, dtype=torch.int32, device="cuda")
    freqs = table(E, 64)
    clean, y = torch.empty_like(q), torch.empty_like(q)

    def call(out):
        E.rope(E.rope_call(q.data_ptr(), out.data_ptr(), freqs.data_ptr(), 4, 3, 64, E.FP32, d_pos=pos.data_ptr()), stream())
        torch.cuda.synchronize()

    call(clean)
    q[1, 2, 5], q[3, 0, 40], q[0, 0, 0] = float("nan"), float("inf"), float("-inf")
    call(y)
    hit = torch.zeros_like(q, dtype=torch.bool)
    for t, h, c in ((1, 2, 5), (3, 0, 8), (0, 0, 0)):
        hit[t, h, c] = hit[t, h, c + 32] = True
    assert torch.equal(y[~hit], clean[~hit]) and not torch.isfinite(y[hit]).any()


@pytest.mark.parametrize("name", ["LINEAR", "BASE", "TURNS", "INDEX"])
def test_rope_with_stretched_frequencies(E, name):
    """Whatever the table holds is what a position is multiplied by."""
    tokens, dim = 6, 128
    q = torch.randn((tokens, 2, dim), device="cuda")
    freqs = table(E, dim, stretch=getattr(E, "ROPE_" + name), factor=8.0, trained_len=8192.0, low=1.0, high=4.0)
    pos = np.array([0, 1, 5000, 8192, 131071, 1 << 30])
    y, d_pos = torch.empty_like(q), torch.tensor(pos, dtype=torch.int32, device="cuda")
    E.rope(E.rope_call(q.data_ptr(), y.data_ptr(), freqs.data_ptr(), tokens, 2, dim, E.FP32, d_pos=d_pos.data_ptr()), stream())
    torch.cuda.synchronize()
    turns = [[(int(p) * (int(f) % (1 << 64))) % (1 << 64) / 2.0 ** 64 for f in freqs.tolist()] for p in pos]
    phi = np.array(turns)[:, None] * (2 * math.pi)
    x = q.double().cpu().numpy()
    a, b = x[:, :, : dim // 2], x[:, :, dim // 2:]
    want = np.concatenate((a * np.cos(phi) - b * np.sin(phi), a * np.sin(phi) + b * np.cos(phi)), 2)
    size = np.concatenate((np.abs(a) + np.abs(b),) * 2, 2)
    assert off(y, want, size, "fp32") == 0


def test_rope_past_32_bit_offsets(E):
    """A batch of more than 2^32 elements: the last tokens get what they get alone."""
    dim, heads = 128, 8
    tokens = (1 << 32) // (dim * heads) + 300
    q = torch.zeros((tokens, heads, dim), dtype=torch.bfloat16, device="cuda")
    last = torch.randn((301, heads, dim), device="cuda").to(torch.bfloat16)
    q[-301:] = last
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    freqs = table(E, dim)
    y = torch.empty_like(last)
    E.rope(E.rope_call(last.data_ptr(), y.data_ptr(), freqs.data_ptr(), 301, heads, dim, E.BF16, d_pos=pos[-301:].data_ptr()), stream())
    E.rope(E.rope_call(q.data_ptr(), q.data_ptr(), freqs.data_ptr(), tokens, heads, dim, E.BF16, d_pos=pos.data_ptr()), stream())
    torch.cuda.synchronize()
    assert torch.equal(q[-301:], y) and int((q != 0).sum()) == int((y != 0).sum())
    del q
    torch.cuda.empty_cache()


def test_rope_in_a_graph(E):
    """Captured on a stream of its own, in place and from lengths; replayed over other lengths: as called."""
    n, dim, spare = 9, 64, 3
    freqs = table(E, dim)
    cu, lens = torch.empty(n + 1, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    rows = torch.empty((40, 6 * dim), dtype=torch.bfloat16, device="cuda")

    def call():
        E.rope(E.rope_call(rows.data_ptr(), rows.data_ptr(), freqs.data_ptr(), 40, 4, dim, E.BF16, d_k=rows.data_ptr() + 8 * dim, k_heads=1,
                           d_k_out=rows.data_ptr() + 8 * dim, d_cu=cu.data_ptr(), d_len=lens.data_ptr(), n_req=n, q_row=6 * dim,
                           q_out_row=6 * dim, k_row=6 * dim, k_out_row=6 * dim), stream())

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    rng = np.random.default_rng(12)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call()
    for i in range(4):
        new = rng.multinomial(40 - spare, np.ones(n) / n) * (rng.random(n) < 0.7)
        cu.copy_(torch.from_numpy(np.concatenate(([0], np.cumsum(new)))))
        lens.copy_(torch.from_numpy(new + rng.integers(0, 1 << 20, n)))
        value = torch.randn(rows.shape, device="cuda").to(torch.bfloat16)
        outs = []
        for replayed in (False, True):
            rows.copy_(value)
            graph.replay() if replayed else call()
            torch.cuda.synchronize()
            outs.append(rows.clone())
        total = int(new.sum())
        assert torch.equal(*outs) and torch.equal(rows[total:], value[total:]) and torch.equal(rows[:, 5 * dim:], value[:, 5 * dim:]), i
        assert not torch.equal(rows[:total, : 5 * dim], value[:total, : 5 * dim])
