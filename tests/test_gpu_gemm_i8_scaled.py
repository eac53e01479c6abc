"""GPU tests of the INT8 product with scales (ep_gemm_i8_scaled).  The sums are exact, and every step
after them is one FP32 operation in a stated order, so FP32 outputs are held bit for bit to numpy's
float32 arithmetic on exact sums, and 16-bit outputs to those rounded once."""
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


def inputs(m, n, k, seed, top=127):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randint(-top, top + 1, (m, k), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
    xs = torch.exp(torch.randn(m, generator=g, device="cuda") - 4)
    ws = torch.exp(torch.randn(n, generator=g, device="cuda") - 6)
    b = torch.randn(n, generator=g, device="cuda")
    return x, xs, w, ws, b


def sums(x, w):
    """Exact sums: products of 512 columns (below 2^23) in float32, added in int64."""
    total = torch.zeros((x.shape[0], w.shape[0]), dtype=torch.int64, device="cuda")
    for lo in range(0, x.shape[1], 512):
        total += (x[:, lo: lo + 512].float() @ w[:, lo: lo + 512].float().t()).long()
    return total


def reference(x, xs, w, ws, b, total=None):
    f = np.float32
    s = (sums(x, w) if total is None else total).cpu().numpy()
    with np.errstate(over="ignore", invalid="ignore"):
        y = s.astype(f) * xs.cpu().numpy()[:, None] * ws.cpu().numpy()[None]
        return y if b is None else y + b.cpu().numpy()[None]


def run(E, x, xs, w, ws, b, y_name, shift=0):
    """shift: elements that Y lies off an aligned address."""
    m, k, n = x.shape[0], x.shape[1], w.shape[0]
    flat = torch.full(((m + 1) * n + shift,), 7.0, dtype=TYPES[y_name], device="cuda")
    y = flat[shift:].view(m + 1, n)
    room = torch.empty(E.gemm_i8_scaled_workspace(m, n, k) + 16, dtype=torch.uint8, device="cuda")
    room[-16:] = 0x5A
    E.gemm_i8_scaled(x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), y.data_ptr(), m, n, k,
                     y_dtype={"bf16": E.BF16, "fp16": E.FP16, "fp32": E.FP32}[y_name], d_bias=0 if b is None else b.data_ptr(),
                     d_ws=room.data_ptr(), ws_bytes=room.numel() - 16, stream=stream())
    torch.cuda.synchronize()
    assert (y[m] == 7.0).all() and (flat[:shift] == 7.0).all() and (room[-16:] == 0x5A).all()
    return y[:m]


# few rows, the streaming kernels' and the tiles' edges, few and many columns, short and long k
SHAPES = [(1, 1, 16), (1, 17408, 5120), (1, 5120, 17408), (2, 7, 144), (15, 333, 2048), (16, 4096, 272), (17, 260, 16), (31, 1000, 4112),
          (32, 5120, 1024), (33, 129, 640), (61, 5120, 17408), (64, 300, 8192), (65, 64, 131056), (100, 2048, 5120), (128, 128, 128),
          (200, 17408, 512), (203, 5120, 2064), (257, 1025, 1040), (500, 63, 4096), (513, 5120, 1024), (1000, 3856, 272), (1024, 1024, 1024),
          (2048, 1300, 528), (2500, 4100, 64), (4441, 438, 1488)]
# every tile size with whole tiles, with halves in the last round (one of them without a row) and with k shared out
SHAPES += [(69, 4084, 16), (194, 4164, 160), (516, 8, 1872), (945, 2142, 1888), (1388, 2877, 352), (2989, 617, 144), (1189, 3508, 448),
           (1464, 2657, 240), (2223, 930, 6352), (2601, 5855, 144), (552, 3658, 6128), (1570, 2546, 384), (455, 2089, 6320),
           (2775, 4393, 928), (3842, 5192, 1040), (774, 5041, 5728)]
# quarters and eighths in the last round, alone and after whole tiles
SHAPES += [(166, 678, 16), (546, 9, 272), (195, 8750, 1680), (4483, 9, 144), (524, 7215, 80), (269, 4140, 176), (915, 8642, 16), (3093, 3118, 16),
           (4335, 257, 16), (2218, 4434, 16), (520, 8757, 1712), (2874, 7002, 1184), (2260, 8505, 1424), (2569, 6250, 1696), (4498, 9, 3488),
           (564, 8, 2800), (74, 8558, 5872), (2861, 4105, 1168), (3807, 5487, 1344), (68, 8401, 6192), (133, 8333, 16), (154, 5746, 5696),
           (3510, 3415, 16), (3204, 4869, 16), (4704, 9, 6224), (1303, 1282, 16), (2480, 1572, 544), (386, 8270, 16), (650, 5897, 8192)]
# tiles of 192 rows of W, and what else is chosen beside them
SHAPES += [(1435, 8685, 1168), (3472, 5081, 1696), (644, 8374, 16), (1810, 8444, 16), (2088, 5490, 16), (1356, 6789, 16), (3586, 2067, 16),
           (3077, 543, 16), (4921, 1583, 16), (3347, 4705, 16), (1703, 4857, 1872), (7420, 1058, 1008), (4228, 2875, 16), (1154, 2311, 16816)]


@pytest.mark.parametrize("y_name", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product_matches_definition(E, m, n, k, y_name):
    say(f"  product {m}x{n}x{k} {y_name}")
    x, xs, w, ws, b = inputs(m, n, k, m + n + k)
    if (m + n) % 2:
        b = None
    y = run(E, x, xs, w, ws, b, y_name)
    want = torch.from_numpy(reference(x, xs, w, ws, b)).cuda()
    assert torch.equal(y, want.to(TYPES[y_name]))


@pytest.mark.parametrize("m,n,k", [(1, 64, 131056), (40, 200, 131056), (300, 70, 131056), (1030, 260, 131056)])
def test_product_of_extreme_sums(E, m, n, k):
    """Codes of -128 throughout, sums of 2^14 k just below 2^31, of both signs."""
    x = torch.full((m, k), -128, dtype=torch.int8, device="cuda")
    w = torch.full((n, k), -128, dtype=torch.int8, device="cuda")
    w[::2] = 127
    ones_x, ones_w = torch.ones(m, device="cuda"), torch.ones(n, device="cuda")
    y = run(E, x, ones_x, w, ones_w, None, "fp32")
    want = torch.tensor([-128 * 127 * k if j % 2 == 0 else (1 << 14) * k for j in range(n)], dtype=torch.int64, device="cuda").float()
    assert torch.equal(y, want[None].expand_as(y))


@pytest.mark.parametrize("m", [1, 20, 90, 700])
def test_product_outputs_at_any_element(E, m):
    for n, shift in ((64, 1), (64, 4), (63, 0), (66, 2), (61, 3)):
        x, xs, w, ws, b = inputs(m, n, 400, m + n + shift)
        for y_name in ("bf16", "fp32"):
            y = run(E, x, xs, w, ws, b, y_name, shift)
            assert torch.equal(y, torch.from_numpy(reference(x, xs, w, ws, b)).cuda().to(TYPES[y_name]))


@pytest.mark.parametrize("m", [3, 60, 300, 1500])
def test_product_scales_that_are_not_finite_stay_in_their_row_or_column(E, m):
    """And outputs beyond a type's range are infinities."""
    x, xs, w, ws, _ = inputs(m, 200, 256, m)
    clean = run(E, x, xs, w, ws, None, "fp16").clone()
    xs[1], ws[7], ws[9] = float("nan"), float("inf"), 1e6
    y = run(E, x, xs, w, ws, None, "fp16")
    want = torch.from_numpy(reference(x, xs, w, ws, None)).cuda().half()
    assert torch.equal(torch.nan_to_num(y, 1.0, 2.0, 3.0), torch.nan_to_num(want, 1.0, 2.0, 3.0)) and torch.equal(torch.isnan(y), torch.isnan(want))
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[1] = keep[:, 7] = keep[:, 9] = False
    assert torch.equal(y[keep], clean[keep]) and torch.isnan(y[1]).all() and torch.isinf(y[:, 9]).any()


@pytest.mark.parametrize("m,n,k", [(1, 5120, 4096), (48, 5120, 4096), (200, 1024, 8192), (1100, 1024, 2048)])
def test_product_repeats_its_bits_on_another_stream_and_in_a_graph(E, m, n, k):
    x, xs, w, ws, b = inputs(m, n, k, 5)
    want = run(E, x, xs, w, ws, b, "bf16")
    y = torch.empty_like(want)
    room = torch.empty(E.gemm_i8_scaled_workspace(m, n, k), dtype=torch.uint8, device="cuda")

    def call():
        E.gemm_i8_scaled(x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), y.data_ptr(), m, n, k, d_bias=b.data_ptr(),
                         d_ws=room.data_ptr(), ws_bytes=room.numel(), stream=stream())

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert torch.equal(y, want)
    with torch.cuda.graph(graph, stream=side):
        call()
    for i in range(4):
        x.copy_(torch.roll(x, 1, 1))
        w.copy_(torch.roll(w, 1, 1))        # the same sums, every operand moved
        y.fill_(0)
        room.fill_(i)                       # what a workspace held does not matter
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i


def test_products_at_once(E):
    """Two streams' calls side by side, each with a workspace of its own: the same bits as alone."""
    sizes = [(203, 5120, 4096), (774, 5041, 5728), (9, 5120, 4096)]
    streams = [torch.cuda.Stream() for _ in sizes]
    calls = []
    for i, (m, n, k) in enumerate(sizes):
        x, xs, w, ws, b = inputs(m, n, k, 40 + i)
        want = run(E, x, xs, w, ws, b, "bf16")
        room = torch.empty(E.gemm_i8_scaled_workspace(m, n, k), dtype=torch.uint8, device="cuda")
        calls.append((x, xs, w, ws, b, want, torch.zeros((8, m, n), dtype=torch.bfloat16, device="cuda"), room))
    torch.cuda.synchronize()
    for turn in range(8):
        for (m, n, k), s, (x, xs, w, ws, b, _, y, room) in zip(sizes, streams, calls):
            E.gemm_i8_scaled(x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), y[turn].data_ptr(), m, n, k, d_bias=b.data_ptr(),
                             d_ws=room.data_ptr(), ws_bytes=room.numel(), stream=s.cuda_stream)
    torch.cuda.synchronize()
    for call in calls:
        assert all(torch.equal(y, call[5]) for y in call[6])


def test_product_of_a_decoded_container(E, oracle):
    """W and its scales as an INT8 row container decodes to, X as the quantiser leaves it: within the
    quantiser's half codes of the weights' own product."""
    from paper_2609_34185_amd import workloads as Wl
    rows, cols, m = 320, 512, 37
    blob, _ = E.encode(Wl.ragged_tensor(3, rows, cols, scale=0.03), 5.0, container=E.CONT_INT8_ROW)
    w, delta, status = E.decode(blob, E.INT8)
    x = torch.randn((m, cols), device="cuda").to(torch.bfloat16)
    q, xs = torch.empty((m, cols), dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda")
    E.quant_i8_row(x.data_ptr(), E.BF16, m, cols, q.data_ptr(), xs.data_ptr(), stream=stream())
    y = run(E, q, xs, w, delta, None, "fp32").double()
    assert int(status.item()) == 0
    wide = w.double() * delta.double()[:, None]
    bound = 0.5001 * xs.double()[:, None] * wide.abs().sum(1)[None] + 4 * 2.0 ** -24 * y.abs()
    assert ((y - x.double() @ wide.t()).abs() <= bound).all()


@pytest.mark.parametrize("m", [2, 300])
def test_product_of_a_large_weight(E, m):
    """W of more than 2^31 bytes: the last rows get what they get alone."""
    k, n = 4096, (1 << 31) // 4096 + 700
    x, xs, w, ws, b = inputs(m, 1000, k, 8)
    big = torch.zeros((n, k), dtype=torch.int8, device="cuda")
    big[-1000:] = w
    bws = torch.ones(n, device="cuda")
    bws[-1000:] = ws
    y = run(E, x, xs, big, bws, None, "bf16")
    assert torch.equal(y[:, -1000:], run(E, x, xs, w, ws, None, "bf16")) and (y[:, :-1000] == 0).all()
    del big, y
    torch.cuda.empty_cache()


# sizes whose k is shared out over workgroups: the sums pass through a workspace, and a second launch joins them
SHARED = [(203, 5120, 17408), (512, 5120, 17408), (1154, 2311, 16816), (455, 2089, 6320)]

# and paths that none of the sizes above takes: 256 x 128 tiles with k shared out, 256 x 256 tiles in several rounds without
# pieces, 192 x 128 tiles in halves after whole rounds (and as many tiles as CUs), 32 rows streamed in several rounds
# (test_i8_plan.py holds these lists to the choice)
PATHS = [(2221, 389, 9840), (685, 1998, 32192), (255, 5251, 49344), (2065, 13441, 1296), (2317, 12974, 3088), (598, 14405, 16),
         (844, 10266, 384), (1943, 3055, 1840), (18, 12503, 16), (63, 17723, 17184)]


@pytest.mark.parametrize("y_name", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m,n,k", PATHS + SHARED)
def test_product_matches_definition_on_every_path(E, m, n, k, y_name):
    test_product_matches_definition(E, m, n, k, y_name)


def shared(E, m, n, k):
    """The workspace that these sizes need; a choice of kernel that needs none would leave a test without its subject."""
    size = E.gemm_i8_scaled_workspace(m, n, k)
    assert size > 0, "k is not shared out here any more: take other sizes"
    return size


@pytest.mark.parametrize("m,n,k", SHARED)
def test_product_refuses_a_workspace_that_is_missing_short_or_misaligned(E, m, n, k):
    """On the host, before anything is launched: the outputs stay as they were."""
    size = shared(E, m, n, k)
    x, xs, w, ws, b = inputs(m, n, k, 3)
    room = torch.zeros(size + 16, dtype=torch.uint8, device="cuda")
    y = torch.full((m, n), 7.0, dtype=torch.bfloat16, device="cuda")
    for d_ws, ws_bytes in ((0, 0), (0, size), (room.data_ptr(), size - 1), (room.data_ptr(), 0), (room.data_ptr() + 8, size)):
        with pytest.raises(E.EntroPackError) as e:
            E.gemm_i8_scaled(x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), y.data_ptr(), m, n, k, d_bias=b.data_ptr(), d_ws=d_ws,
                             ws_bytes=ws_bytes, stream=stream())
        assert e.value.code == E.ERR_ARG and "workspace" in str(e.value)
    torch.cuda.synchronize()
    assert (y == 7.0).all() and (room == 0).all()


def test_product_one_workspace_for_any_size(E):
    """1 MiB for each CU is enough whatever the sizes, which one batch's own need is not."""
    most = torch.cuda.get_device_properties(0).multi_processor_count << 20
    rng = np.random.default_rng(1)
    for m, n, k in np.exp(rng.uniform(np.log((1, 1, 1)), np.log((20000, 20000, 8190)), (20000, 3))).astype(int).tolist():
        assert E.gemm_i8_scaled_workspace(m, n, 16 * k) <= most
    room = torch.empty(most, dtype=torch.uint8, device="cuda")
    n, k = 2056, 8192
    x, xs, w, ws, b = inputs(700, n, k, 4)
    for m in (700, 300, 90, 20, 1):
        y = torch.empty((m, n), dtype=torch.float32, device="cuda")
        E.gemm_i8_scaled(x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), y.data_ptr(), m, n, k, y_dtype=E.FP32, d_bias=b.data_ptr(),
                         d_ws=room.data_ptr(), ws_bytes=most, stream=stream())
        assert torch.equal(y, torch.from_numpy(reference(x[:m], xs[:m], w, ws, b)).cuda())


@pytest.mark.parametrize("m,n,k", SHARED)
def test_products_with_shared_k_in_a_graph(E, m, n, k):
    """Both launches captured, twice over one workspace, and replayed over other operands, with whatever
    the workspace and the outputs held before."""
    size = shared(E, m, n, k)
    x, xs, w, ws, b = inputs(m, n, k, 6)
    want = run(E, x, xs, w, ws, b, "bf16").clone()
    other = run(E, x, xs, w, ws, None, "fp32").clone()
    y, z, room = torch.empty_like(want), torch.empty_like(other), torch.empty(size, dtype=torch.uint8, device="cuda")

    def call():
        for out, dtype, bias in ((y, E.BF16, b.data_ptr()), (z, E.FP32, 0)):
            E.gemm_i8_scaled(x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), out.data_ptr(), m, n, k, y_dtype=dtype, d_bias=bias,
                             d_ws=room.data_ptr(), ws_bytes=size, stream=stream())

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call()
    for i in range(4):
        x.copy_(torch.roll(x, 1, 1))
        w.copy_(torch.roll(w, 1, 1))        # the same sums, every operand moved
        y.fill_(3)
        z.fill_(-3)
        room.fill_(0x5B + 17 * i)
        call() if i == 2 else graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(z, other), i


def test_products_with_shared_k_at_once(E):
    """Calls of several streams side by side, each with a workspace of its own that other calls have
    filled: the same bits as alone."""
    calls = []
    for i, (m, n, k) in enumerate(SHARED):
        x, xs, w, ws, b = inputs(m, n, k, 60 + i)
        want = run(E, x, xs, w, ws, b, "bf16").clone()
        room = torch.full((shared(E, m, n, k),), 0x7F, dtype=torch.uint8, device="cuda")
        calls.append((torch.cuda.Stream(), x, xs, w, ws, b, want, torch.zeros((6, m, n), dtype=torch.bfloat16, device="cuda"), room))
    torch.cuda.synchronize()
    for turn in range(6):
        for (m, n, k), (s, x, xs, w, ws, b, _, y, room) in zip(SHARED, calls):
            E.gemm_i8_scaled(x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), y[turn].data_ptr(), m, n, k, d_bias=b.data_ptr(),
                             d_ws=room.data_ptr(), ws_bytes=room.numel(), stream=s.cuda_stream)
    torch.cuda.synchronize()
    for call in calls:
        assert all(torch.equal(y, call[6]) for y in call[7])


def test_product_of_a_large_batch(E):
    """X of more than 2^31 bytes: the last rows get what they get alone."""
    n, k = 200, 4096
    m = (1 << 31) // k + 700
    x, xs, w, ws, b = inputs(1000, n, k, 9)
    big, bxs = torch.zeros((m, k), dtype=torch.int8, device="cuda"), torch.ones(m, device="cuda")
    big[-1000:], bxs[-1000:] = x, xs
    y = run(E, big, bxs, w, ws, None, "bf16")
    assert torch.equal(y[-1000:], run(E, x, xs, w, ws, None, "bf16")) and (y[:-1000] == 0).all()
    del big, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("m,n", [(70000, 65604), (260, 1 << 24), (1 << 24, 260), (16, 1 << 24)])
def test_product_of_a_large_output(E, m, n):
    """Y of more than 2^32 elements, and as many rows or columns as there may be: every element."""
    if torch.cuda.mem_get_info()[0] < 3 * m * n + (8 << 30):
        pytest.skip("needs more device memory")
    x, xs, w, ws, _ = inputs(m, n, 16, 10)
    y = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    room = torch.empty(E.gemm_i8_scaled_workspace(m, n, 16) + 16, dtype=torch.uint8, device="cuda")
    E.gemm_i8_scaled(x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), y.data_ptr(), m, n, 16, d_ws=room.data_ptr(),
                     ws_bytes=room.numel(), stream=stream())
    step = max(1, (1 << 27) // n)
    for i in range(0, m, step):
        want = (x[i: i + step].float() @ w.float().t()) * xs[i: i + step, None] * ws       # sums of 16 products: exact
        assert torch.equal(y[i: i + step], want.to(torch.bfloat16)), i
    del y
    torch.cuda.empty_cache()
