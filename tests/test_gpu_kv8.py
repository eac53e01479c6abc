"""GPU tests of the paged 8-bit key/value cache: block tables and slot maps (exact, against a plain
loop), the append (bit for bit against its definition in numpy), and the attention, against a
softmax in 64 bits over the codes' values.

The attention's bound, element by element.  The scores: FP32 sums of D exact products, so off by
at most d = (D + 8) 2^-23 scale sum |q k| (the row's power of two is exact), and the exponential
and its argument add 2^-21.  A weight is thus off by a factor within 2 d + 2^-21 of 1, and rounded
to 11 bits (2^-11) where it enters the product.  Sums of n weights are FP32: n 2^-23 of their
size, and joining partial ones a few units more.  With A = sum p |v| / sum p,
    |out - exact| <= A (2 (2 d + 2^-21) + 2^-11 + (n + 64) 2^-22) + half a unit of the output,
and |lse - exact| <= 2 d + (n + 64) 2^-22 + 2^-21 |lse|.
"""
import math
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


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


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---- block tables and slot maps -----------------------------------------------------------
def slots_ref(E, cached, new, page, free, n_free, table, n_slots):
    table, status, used, tok = table.copy(), 0, 0, 0
    off, lens, cu, slots, stopped = 0, [], [0], [-1] * n_slots, False
    for b, (c, w) in enumerate(zip(cached, new)):
        c, w = max(c, 0), max(w, 0)
        have, want = -(-c // page), -(-(c + w) // page)
        ok = True
        if want > table.shape[1]:
            ok, status = False, status | E.STATUS_TABLE_FULL
        if tok + w > n_slots:
            ok, status = False, status | E.STATUS_SLOTS_FULL
        need = want - have if ok else 0
        if need and off + need > n_free:
            ok, status, stopped = False, status | E.STATUS_NO_PAGES, True
        off += need
        if ok:
            if not stopped:
                used = off
            for j in range(need):
                table[b, have + j] = free[off - need + j]
            for i in range(w):
                slots[tok + i] = int(table[b, (c + i) // page]) * page + (c + i) % page
        lens.append(c + w if ok else c)
        tok += w
        cu.append(min(tok, 2 ** 31 - 1))
    return table, lens, cu, slots, used, status


def slots_gpu(E, cached, new, page, free, n_free, table, n_slots):
    n = len(cached)
    d = torch.from_numpy(table.copy()).cuda()
    fr = ints(list(free) + [-5])
    ln, cu = torch.full((n + 1,), -9, dtype=torch.int32, device="cuda"), torch.full((n + 2,), -9, dtype=torch.int32, device="cuda")
    sl = torch.full((n_slots + 1,), -9, dtype=torch.int64, device="cuda")
    used, st = ints([-9]), ints([0])
    dc, dn, df = ints(cached), ints(new), ints([n_free])
    E.kv8_slots(dc.data_ptr(), dn.data_ptr(), n, page, fr.data_ptr(), df.data_ptr(), d.data_ptr(),
                table.shape[1], ln.data_ptr(), cu.data_ptr(), sl.data_ptr(), n_slots, used.data_ptr(), st.data_ptr(), stream())
    torch.cuda.synchronize()
    assert ln[-1] == -9 and cu[-1] == -9 and sl[-1] == -9
    return d.cpu().numpy(), ln[:-1].tolist(), cu[:-1].tolist(), sl[:-1].tolist(), int(used), int(st)


SLOTS = [  # requests, most cached, most new, page, share of the pages that is free, room in the slot map
    (1, 0, 1, 16, 2.0, 0), (1, 100, 5000, 64, 1.0, 3), (3, 40, 1, 16, 1.0, 0), (7, 0, 0, 32, 1.0, 5),
    (256, 3000, 1, 64, 1.0, 0), (300, 500, 40, 16, 0.5, 9), (1023, 70, 9, 128, 1.0, 0), (1024, 70, 9, 256, 0.8, 1),
    (1025, 70, 9, 32, 1.1, 2100), (2500, 30, 33, 16, 0.3, 0), (5000, 200, 3, 16, 0.95, 0), (40, 5000, 3000, 32, 1.0, -700),
]


@pytest.mark.parametrize("n,top_c,top_w,page,share,room", SLOTS)
def test_slots_match_a_plain_loop(E, n, top_c, top_w, page, share, room):
    say(f"  slots {n} requests, page {page}")
    rng = np.random.default_rng([31, n, top_c, top_w, page])
    cached, new = rng.integers(-2, top_c + 1, n).tolist(), rng.integers(-1, top_w + 1, n).tolist()
    width = -(-(top_c + top_w) // page) + 1
    if n > 20:   # some whose row is too short
        cached[3], new[11] = page * width - 1, page * width + 5
        new[3] = 2
    need = sum(-(-(max(c, 0) + max(w, 0)) // page) - -(-max(c, 0) // page) for c, w in zip(cached, new))
    pages = rng.permutation(need * 3 + n * width + 10).astype(np.int32)
    table = pages[: n * width].reshape(n, width)
    n_free = int(need * share)
    free = pages[n * width: n * width + max(need, 1)]
    n_slots = max(0, sum(max(w, 0) for w in new) + room)
    got = slots_gpu(E, cached, new, page, free, n_free, table, n_slots)
    want = slots_ref(E, cached, new, page, free.tolist(), n_free, table, n_slots)
    for g, w in zip(got, want):
        assert np.array_equal(g, w)


def test_slots_huge_counts_are_refused_not_wrapped(E):
    """Counts near 2^31: sums do not wrap, the requests that do not fit are refused."""
    table = np.full((4, 8), 3, np.int32)
    cached, new = [2 ** 31 - 1, 5, 0, 10], [2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 7]
    a = slots_gpu(E, cached, new, 16, [7, 8], 2, table, 100)
    b = slots_ref(E, cached, new, 16, [7, 8], 2, table, 100)
    for g, w in zip(a, b):
        assert np.array_equal(g, w)
    a = slots_gpu(E, [0, 0], [3, 4], 16, [7, 8], -4, np.full((2, 2), -1, np.int32), 7)
    assert a[1] == [0, 0] and a[3] == [-1] * 7 and a[4] == 0 and a[5] == E.STATUS_NO_PAGES


def test_slots_of_earlier_requests_stay_when_the_sums_pass_32_bits(E):
    n = 9000     # several tiles of requests, the later ones past 2^32 - 2 tokens
    cached, new = [0] * n, [1] * n
    new[0], new[7], new[9] = 5, 2 ** 31 - 1, 2 ** 31 - 1
    table = np.full((n, 1), -1, np.int32)
    free = list(range(n))
    got = slots_gpu(E, cached, new, 16, free, n, table, 4000)
    want = slots_ref(E, cached, new, 16, free, n, table, 4000)
    for g, w in zip(got, want):
        assert np.array_equal(g, w)
    assert got[3][:11] == [0, 1, 2, 3, 4, 16, 32, 48, 64, 80, 96] and got[3][11:] == [-1] * 3989


def test_slots_refuse_requests_of_2_to_the_31_tokens(E):
    width = 2 ** 23 + 1
    table = np.zeros((1, width), np.int32)
    table[0, width - 2] = 77
    full, over = slots_gpu(E, [2 ** 31 - 2], [1], 256, [1], 1, table, 3), slots_gpu(E, [2 ** 31 - 1], [2], 256, [1], 1, table, 3)
    assert full[1:] == ([2 ** 31 - 1], [0, 1], [77 * 256 + 254, -1, -1], 0, 0)
    assert over[1:] == ([2 ** 31 - 1], [0, 2], [-1, -1, -1], 0, E.STATUS_TABLE_FULL) and np.array_equal(over[0], table)


# ---- append ----------------------------------------------------------------------------------
def e4m3_value(c):
    return torch.from_numpy(np.ascontiguousarray(c)).view(torch.float8_e4m3fn).float().numpy()


def nearest(v, int8):
    """Codes (as uint8) of float32 values: nearest, halves to even, saturating."""
    if int8:
        return np.clip(np.rint(v), -127, 127).astype(np.int8).view(np.uint8)
    a = np.minimum(np.abs(v.astype(np.float64)), 448.0)
    e = np.maximum(np.frexp(np.maximum(a, 1e-300))[1] - 1, -6)
    n = np.rint(np.ldexp(a, 3 - e)).astype(np.int64)
    code = np.where(n >= 16, ((e + 8) << 3), np.where(n >= 8, ((e + 7) << 3) + (n - 8), n))
    return (code | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def append_ref(k_codes, scales, x, slots, page, int8, is_v):
    """codes [pages][heads][page][dim] (values transposed first), float32 x [n][heads][dim]."""
    codes = np.ascontiguousarray(k_codes.swapaxes(2, 3)) if is_v else k_codes.copy()
    scales = scales.copy()
    top, t, n = np.float32(127 if int8 else 448), 0, len(slots)
    while t < n:
        if slots[t] < 0 or slots[t] >= len(codes) * page:
            t += 1
            continue
        e, p, o = t + 1, slots[t] // page, slots[t] % page
        while e < n and slots[e] >= 0 and slots[e] // page == p:
            e += 1
        for h in range(codes.shape[1]):
            before = scales[p, h] if o else np.float32(0)
            fresh = np.abs(x[t:e, h]).max().astype(np.float32) * (np.float32(1) / top)
            now = max(before, fresh)
            if now != before:
                old = e4m3_value(codes[p, h, :o]) if not int8 else codes[p, h, :o].view(np.int8).astype(np.float32)
                back = (old * before).astype(np.float32)
                codes[p, h, :o] = nearest((back / now).astype(np.float32) if now else 0 * back, int8)
            codes[p, h, o: o + e - t] = nearest((x[t:e, h] / now).astype(np.float32) if now else 0 * x[t:e, h], int8)
            scales[p, h] = now
        t = e
    return (codes.swapaxes(2, 3) if is_v else codes), scales


def run_append(E, kc, vc, ks, vs, k, v, code, slots, page, dim, int8):
    cache = E.kv8_cache(kc.data_ptr(), vc.data_ptr(), ks.data_ptr(), vs.data_ptr(), kc.shape[0], kc.shape[1], page, dim,
                        E.INT8 if int8 else E.FP8_E4M3)
    s = torch.tensor(slots, dtype=torch.int64, device="cuda")
    E.kv8_append(cache, k.data_ptr(), v.data_ptr(), code, k.stride(0), v.stride(0), s.data_ptr(), len(slots), stream())
    torch.cuda.synchronize()


APPENDS = [  # heads, dim, page, int8, dtype, (cached, new) of each request
    (1, 64, 16, False, "bf16", [(0, 1)]), (2, 128, 64, False, "bf16", [(5, 1), (63, 1), (64, 1), (127, 1), (0, 1)]),
    (8, 128, 32, True, "bf16", [(31, 40), (0, 33), (7, 1), (90, 100)]), (4, 64, 128, False, "fp16", [(100, 30), (3, 300), (128, 128)]),
    (2, 256, 16, True, "fp32", [(9, 3), (15, 18), (0, 50)]), (3, 256, 256, False, "fp32", [(200, 400), (17, 2), (255, 2)]),
    (1, 128, 16, True, "fp16", [(i, 1) for i in range(40)]), (2, 64, 64, True, "bf16", [(i * 7, 5 + i) for i in range(12)]),
    (2, 128, 256, True, "bf16", [(0, 700), (100, 156), (100, 157)]), (2, 128, 64, False, "bf16", [(i, 1 + i % 3) for i in range(150)]),
]


@pytest.mark.parametrize("i", range(len(APPENDS)))
def test_append_matches_definition(E, i):
    heads, dim, page, int8, dtype, requests = APPENDS[i]
    say(f"  append heads {heads} dim {dim} page {page} int8 {int8} {dtype}")
    rng = np.random.default_rng([41, i])
    pages = sum(-(-(c + w) // page) for c, w in requests) + 2
    perm, slots, at = rng.permutation(pages), [], 0
    for j, (c, w) in enumerate(requests):
        mine = perm[at: at + -(-(c + w) // page)]
        at += len(mine)
        slots += [int(mine[p // page]) * page + p % page for p in range(c, c + w)]
        if j % 2:
            slots += [-1, pages * page + 3]     # skipped
    n = len(slots)
    kc = torch.from_numpy(rng.integers(-120, 121, (pages, heads, page, dim)).astype(np.int8)).cuda().view(torch.uint8)
    vc = torch.from_numpy(rng.integers(-120, 121, (pages, heads, dim, page)).astype(np.int8)).cuda().view(torch.uint8)
    if not int8:
        kc, vc = [torch.where((c & 0x7F) == 0x7F, c & 0x80, c) for c in (kc, vc)]
    ks, vs = [torch.from_numpy(np.exp(rng.standard_normal((pages, heads)) - 4).astype(np.float32)).cuda() for _ in range(2)]
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[dtype]
    # one fused row a token: queries, then keys, then values
    qkv = torch.from_numpy(rng.standard_normal((n, heads * dim * 3)) * np.exp(rng.standard_normal((n, 1)))).to(dt).cuda()
    qkv[n // 2] = 0
    k, v = qkv[:, heads * dim: 2 * heads * dim], qkv[:, 2 * heads * dim:]
    refs = [append_ref(c.cpu().numpy(), s.cpu().numpy(), x.float().cpu().numpy().reshape(n, heads, dim), slots, page, int8, is_v)
            for c, s, x, is_v in ((kc, ks, k, False), (vc, vs, v, True))]
    run_append(E, kc, vc, ks, vs, k, v, {"bf16": E.BF16, "fp16": E.FP16, "fp32": E.FP32}[dtype], slots, page, dim, int8)
    for (rc, rs), c, s in zip(refs, (kc, vc), (ks, vs)):
        assert np.array_equal(s.cpu().numpy().view(np.uint32), rs.view(np.uint32))
        got = c.cpu().numpy()
        if not int8:    # a code of zero may carry either sign where it was rescaled from one
            assert np.array_equal(e4m3_value(got), e4m3_value(rc))
        else:
            assert np.array_equal(got, rc)


def test_append_zero_tokens_and_zero_values(E):
    """Pages of zeros get scale 0 and codes 0, and take later tokens without loss."""
    kc = torch.full((2, 1, 16, 64), 0x55, dtype=torch.uint8, device="cuda")
    vc = torch.full((2, 1, 64, 16), 0x55, dtype=torch.uint8, device="cuda")
    ks, vs = torch.ones((2, 1), device="cuda"), torch.ones((2, 1), device="cuda")
    z = torch.zeros((3, 64), dtype=torch.bfloat16, device="cuda")
    run_append(E, kc, vc, ks, vs, z, z, E.BF16, [16, 17, 18], 16, 64, False)
    assert ks[1] == 0 and vs[1] == 0 and (kc[1, 0, :3] == 0).all() and (kc[1, 0, 3:] == 0x55).all()
    assert (vc[1, 0, :, :3] == 0).all() and (vc[1, 0, :, 3:] == 0x55).all() and ks[0] == 1
    one = torch.full((1, 64), 2.0, dtype=torch.bfloat16, device="cuda")
    run_append(E, kc, vc, ks, vs, one, one, E.BF16, [19], 16, 64, False)
    assert (kc[1, 0, :3] == 0).all() and (kc[1, 0, 3] == 0x7E).all() and ks[1] == np.float32(2) * (np.float32(1) / np.float32(448))


@pytest.mark.parametrize("int8", [False, True])
def test_append_non_finite_shows_in_its_page_and_head(E, int8):
    kc = torch.zeros((2, 2, 16, 64), dtype=torch.uint8, device="cuda")
    vc = torch.zeros((2, 2, 64, 16), dtype=torch.uint8, device="cuda")
    ks, vs = torch.full((2, 2), 0.5, device="cuda"), torch.full((2, 2), 0.5, device="cuda")
    x = torch.randn((3, 128), device="cuda").to(torch.bfloat16)
    x[1, 70] = float("nan")
    y = torch.randn((3, 128), device="cuda").to(torch.bfloat16)
    y[2, 3] = float("inf")
    run_append(E, kc, vc, ks, vs, x, y, E.BF16, [3, 4, 5], 16, 64, int8)
    assert torch.isfinite(ks[0, 0]) and torch.isnan(ks[0, 1]) and torch.isinf(vs[0, 0]) and torch.isfinite(vs[0, 1])
    assert (ks[1] == 0.5).all() and (vs[1] == 0.5).all()
    # a later finite token does not bring it back
    f = torch.randn((1, 128), device="cuda").to(torch.bfloat16)
    run_append(E, kc, vc, ks, vs, f, f, E.BF16, [6], 16, 64, int8)
    assert torch.isnan(ks[0, 1]) and torch.isinf(vs[0, 0])


# ---- attention -------------------------------------------------------------------------------
class Case:
    def __init__(self, requests, q_heads, heads, dim, page, int8, dtype, causal=True, window=0, spare_q=0, seed=1,
                 first_page=0, top_scale=1.0, pages=None):
        g = torch.Generator("cuda").manual_seed(seed)
        self.requests, self.q_heads, self.heads, self.dim, self.page, self.int8 = requests, q_heads, heads, dim, page, int8
        self.causal, self.window, self.dtype = causal, window, dtype
        lens, new = [r[0] for r in requests], [r[1] for r in requests]
        width = max(1, max(-(-n // page) for n in lens))
        need = sum(-(-n // page) for n in lens)
        self.pages = pages or first_page + need + 2
        self.total = sum(new) + spare_q
        shape = (self.pages, heads, page, dim)
        if pages:      # a cache past 2^32 bytes: only the pages in use are filled
            self.kc, self.vc = [torch.zeros(self.pages * heads * page * dim, dtype=torch.uint8, device="cuda") for _ in range(2)]
            self.kc, self.vc = self.kc.view(shape), self.vc.view(self.pages, heads, dim, page)
        else:
            self.kc = self.codes(shape, g)
            self.vc = self.codes((self.pages, heads, dim, page), g)
        perm = first_page + torch.randperm(need + 2, generator=g, device="cuda")
        self.table = torch.full((len(requests), width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(lens):
            c = -(-n // page)
            self.table[b, :c] = perm[at: at + c].to(torch.int32)
            at += c
        if pages:
            for p in perm[:need].tolist():
                self.kc[p], self.vc[p] = self.codes(shape[1:], g), self.codes((heads, dim, page), g)
        self.ks, self.vs = [torch.exp(torch.randn((self.pages, heads), generator=g, device="cuda") * top_scale - 4) for _ in range(2)]
        dt = torch.float16 if dtype == "fp16" else torch.bfloat16
        self.q = (torch.randn((self.total, q_heads, dim), generator=g, device="cuda") * 2).to(dt)
        self.lens, self.cu = ints(lens), ints([sum(new[:i]) for i in range(len(new) + 1)])
        self.max_q, self.max_len = max(1, max(new)), max(lens)
        # past a request's end: not-a-numbers, in E4M3 and as scales of pages nobody owns
        if not pages:
            for b, n in enumerate(lens):
                if n % page:
                    p = int(self.table[b, n // page])
                    self.kc[p, :, n % page:] = 0x7F
                    self.vc[p, :, :, n % page:] = 0x7F
            spare = perm[need:].tolist()
            self.ks[spare], self.vs[spare] = float("nan"), float("inf")
            self.kc[spare], self.vc[spare] = 0xFF, 0x7F

    def codes(self, shape, g):
        x = torch.randn(shape, generator=g, device="cuda")
        if self.int8:
            return (x * 40).clamp(-127, 127).round().to(torch.int8).view(torch.uint8)
        return (x * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)

    def call(self, E, q=None, out=None, lse=True, on=None, **kw):
        q = self.q if q is None else q
        out = torch.full_like(self.q, float("nan")) if out is None else out
        self.lse = torch.full((self.total, self.q_heads), float("nan"), device="cuda")
        cache = E.kv8_cache(self.kc.data_ptr(), self.vc.data_ptr(), self.ks.data_ptr(), self.vs.data_ptr(), self.pages, self.heads,
                            self.page, self.dim, E.INT8 if self.int8 else E.FP8_E4M3)
        args = dict(scale=1 / math.sqrt(self.dim), causal=self.causal, window=self.window, max_q=self.max_q, max_len=self.max_len,
                    q_row=q.stride(0), out_row=out.stride(0), d_lse=self.lse.data_ptr() if lse else 0)
        args.update(kw)
        call = E.kv8_attention_args(q.data_ptr(), out.data_ptr(), self.cu.data_ptr(), self.lens.data_ptr(), self.table.data_ptr(),
                                    self.table.shape[1], len(self.requests), self.total, self.q_heads,
                                    E.FP16 if self.dtype == "fp16" else E.BF16, **args)
        n = E.kv8_attention_workspace(cache, call)
        room = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")   # NaNs: nothing is read that was not written
        E.kv8_attention(cache, call, room.data_ptr(), n, stream() if on is None else on)
        torch.cuda.synchronize()
        assert (room[n:] == 0xFF).all()
        return out

    def value(self, c):
        return (c.view(torch.int8) if self.int8 else c.view(torch.float8_e4m3fn)).double()

    def check(self, out, lse=True):
        group, at = self.q_heads // self.heads, 0
        scale = 1 / math.sqrt(self.dim)
        half, least = (2.0 ** -11, 2.0 ** -25) if self.dtype == "fp16" else (2.0 ** -8, 0.0)
        worst = 0.0
        for b, (n, m) in enumerate(self.requests):
            idx = self.table[b, : -(-n // self.page)].long()
            known = (idx >= 0) & (idx < self.pages)
            pick = idx.clamp(0, self.pages - 1)
            pos, mine = torch.arange(n, device="cuda"), torch.arange(n - m, n, device="cuda")[:, None]
            seen = known.repeat_interleave(self.page)[:n][None].expand(m, n)
            if self.causal:
                seen = seen & (pos <= mine)
                if self.window:
                    seen = seen & (pos > mine - self.window)
            for h in range(self.heads):
                key = (self.value(self.kc[pick, h]) * self.ks[pick, h].double()[:, None, None]).reshape(-1, self.dim)[:n]
                val = (self.value(self.vc[pick, h]) * self.vs[pick, h].double()[:, None, None]).transpose(1, 2).reshape(-1, self.dim)[:n]
                any_seen = seen.any(0)
                key, val = torch.where(any_seen[:, None], key, 0.0), torch.where(any_seen[:, None], val, 0.0)
                for j in range(h * group, (h + 1) * group):
                    q = self.q[at: at + m, j].double()
                    s = (q @ key.t() * scale).masked_fill(~seen, -math.inf)
                    d = (self.dim + 8) * 2.0 ** -23 * scale * ((q.abs() @ key.abs().t()) * seen).amax(1, keepdim=True) if n else torch.zeros((m, 1), device="cuda")
                    empty = ~seen.any(1, keepdim=True)
                    p = torch.where(empty, 0.0, torch.softmax(s, 1)) if n else s
                    want = p @ val
                    size = p @ val.abs()
                    tol = size * (2 * (2 * d + 2.0 ** -21) + 2.0 ** -11 + (n + 64) * 2.0 ** -22)
                    tol = tol + half * (want.abs() + tol) + least
                    off = (out[at: at + m, j].double() - want).abs()
                    assert (off <= tol).all(), (b, j, float((off - tol).max()))
                    worst = max(worst, float((off / tol.clamp(min=1e-30)).max()) if off.numel() else 0.0)
                    if lse:
                        want = torch.logsumexp(s, 1) if n else torch.full((m,), -math.inf, device="cuda")
                        got = self.lse[at: at + m, j].double()
                        gone = torch.isinf(want)
                        assert torch.equal(got[gone], want[gone].double())
                        lt = 2 * d[:, 0] + (n + 64) * 2.0 ** -22 + 2.0 ** -21 * want.abs()
                        assert ((got - want).abs()[~gone] <= lt[~gone]).all()
            at += m
        say(f"    largest share of the bound {worst:.3g}")


STEP = [(1, 1), (15, 1), (16, 1), (17, 1), (64, 1), (65, 1), (300, 1), (1000, 1), (0, 1), (2, 1), (0, 0), (9, 0)]
ATTENTION = [
    dict(requests=[(1, 1)], q_heads=1, heads=1, dim=64, page=16, int8=False, dtype="bf16"),
    dict(requests=STEP, q_heads=16, heads=2, dim=128, page=64, int8=False, dtype="bf16"),
    dict(requests=STEP, q_heads=40, heads=8, dim=128, page=16, int8=True, dtype="fp16"),
    dict(requests=STEP, q_heads=7, heads=1, dim=64, page=128, int8=True, dtype="bf16"),
    dict(requests=STEP, q_heads=4, heads=4, dim=256, page=32, int8=False, dtype="fp16"),
    dict(requests=STEP, q_heads=34, heads=2, dim=64, page=256, int8=False, dtype="bf16"),
    dict(requests=[(5000, 1), (3, 1), (9999, 1)], q_heads=10, heads=2, dim=128, page=64, int8=False, dtype="fp16"),
    dict(requests=[(700, 3), (5, 3), (64, 3), (2, 3)], q_heads=16, heads=2, dim=128, page=32, int8=False, dtype="bf16"),
    dict(requests=[(700, 5), (5, 1), (64, 2), (1, 5)], q_heads=6, heads=2, dim=128, page=32, int8=True, dtype="bf16", causal=False),
    dict(requests=[(900, 2), (2000, 1), (30, 4)], q_heads=8, heads=2, dim=64, page=16, int8=False, dtype="bf16", window=100),
    dict(requests=[(130, 130), (1, 1), (257, 256), (64, 64), (100, 3)], q_heads=4, heads=2, dim=128, page=64, int8=False, dtype="bf16"),
    dict(requests=[(333, 333), (50, 20)], q_heads=5, heads=1, dim=64, page=16, int8=True, dtype="fp16"),
    dict(requests=[(400, 100), (90, 90)], q_heads=8, heads=8, dim=256, page=128, int8=False, dtype="bf16"),
    dict(requests=[(600, 600), (700, 33)], q_heads=6, heads=2, dim=128, page=32, int8=False, dtype="fp16", window=64),
    dict(requests=[(500, 200), (65, 65), (0, 70)], q_heads=4, heads=1, dim=128, page=64, int8=True, dtype="bf16", causal=False),
    dict(requests=[(2000, 1500), (40, 200)], q_heads=8, heads=1, dim=128, page=256, int8=False, dtype="bf16"),
    dict(requests=[(300, 300), (64, 40)], q_heads=4, heads=2, dim=256, page=16, int8=True, dtype="fp16", window=33),
    dict(requests=[(1100, 90), (1500, 700)], q_heads=12, heads=2, dim=64, page=64, int8=False, dtype="fp16"),
]


@pytest.mark.parametrize("i", range(len(ATTENTION)))
def test_attention_matches_64_bits(E, i):
    """Lengths from none to long ones, queries beyond the first key, each type, head layout, page
    and mask; unowned tokens of a page and unowned pages hold not-a-numbers."""
    say(f"  attention {i}: {ATTENTION[i]}")
    c = Case(**ATTENTION[i], seed=i)
    c.check(c.call(E))


@pytest.mark.parametrize("max_q,max_len", [(1, 1), (1, 100000), (64, 40), (3000, 0)])
def test_attention_hints_size_the_launch_only(E, max_q, max_len):
    c = Case([(600, 40), (90, 1), (1000, 70), (0, 2)], 8, 2, 128, 32, False, "bf16")
    c.check(c.call(E, max_q=max_q, max_len=max_len))


@pytest.mark.parametrize("max_q,max_len,window", [(1, 900, 0), (6, 900, 0), (2, 10, 40), (40, 5000, 0)])
def test_attention_of_many_requests(E, max_q, max_len, window):
    """More requests than a workgroup counts in one round, of all lengths from none on, with one to
    six queries, or none."""
    rng = np.random.default_rng(61)
    requests = [(int(n), int(q)) for n, q in zip(rng.integers(0, 900, 700) * (rng.random(700) < 0.4), rng.integers(0, 7, 700))]
    c = Case(requests, 8, 2, 64, 16, False, "bf16", seed=13, window=window)
    c.check(c.call(E, max_q=max_q, max_len=max_len))


def test_attention_wide_spread_of_scales(E):
    """Page scales over many powers of ten: weights stay inside their type, small pages count for
    what they are."""
    for seed in range(3):
        c = Case([(900, 1), (200, 2), (333, 100)], 8, 2, 128, 16, False, "bf16", seed=seed, top_scale=4.0)
        c.ks.clamp_(max=0.05)
        c.check(c.call(E))


def place_weight(c, value_scales, heavy, gap):
    """Request 0's page i gets the value scale value_scales[i] and keys that score the same for every
    query of it: 0 in the pages of `heavy`, 2^-gap of the weight elsewhere."""
    one, minus = (1, 0xFF) if c.int8 else (0x38, 0xB8)
    for i, s in enumerate(value_scales):
        p = int(c.table[0, i])
        c.kc[p] = 0
        c.kc[p, :, :, 0] = one if i in heavy else minus
        c.ks[p], c.vs[p] = 1.0, s
    c.q[: c.requests[0][1], :, 0] = gap * math.log(2) * math.sqrt(c.dim) / 2


def check_weights(c, out):
    """Either kernel against the bound above with what a weight is rounded to in the one for many rows,
    p vs to 11 bits or 2^-37 of the row's largest p vs: n 2^-37 max(p vs) times the largest code more."""
    group, at = c.q_heads // c.heads, 0
    scale, n_heads = 1 / math.sqrt(c.dim), c.heads
    for b, (n, m) in enumerate(c.requests):
        idx = c.table[b, : -(-n // c.page)].long()
        pos, mine = torch.arange(n, device="cuda"), torch.arange(n - m, n, device="cuda")[:, None]
        seen = (pos <= mine) if c.causal else torch.ones((m, n), dtype=torch.bool, device="cuda")
        if c.window:
            seen &= pos > mine - c.window
        for h in range(n_heads):
            page_vs = c.vs[idx, h].double().repeat_interleave(c.page)[:n]
            key = (c.value(c.kc[idx, h]) * c.ks[idx, h].double()[:, None, None]).reshape(-1, c.dim)[:n]
            val = c.value(c.vc[idx, h]).transpose(1, 2).reshape(-1, c.dim)[:n] * page_vs[:, None]
            for j in range(h * group, (h + 1) * group):
                q = c.q[at: at + m, j].double()
                s = (q @ key.t() * scale).masked_fill(~seen, -math.inf)
                d = (c.dim + 8) * 2.0 ** -23 * scale * ((q.abs() @ key.abs().t()) * seen).amax(1, keepdim=True)
                p = torch.softmax(s, 1)
                want, size = p @ val, p @ val.abs()
                floor = n * 2.0 ** -37 * (p * page_vs).amax(1, keepdim=True) * (127 if c.int8 else 448)
                tol = size * (2 * (2 * d + 2.0 ** -21) + 2.0 ** -11 + (n + 64) * 2.0 ** -22) + floor
                tol = tol + 2.0 ** -8 * (want.abs() + tol)
                off = (out[at: at + m, j].double() - want).abs()
                assert bool((off <= tol).all()), (b, j, float((off / tol.clamp(min=1e-300)).max()))
                lse = torch.logsumexp(s, 1)
                assert bool(((c.lse[at: at + m, j].double() - lse).abs() <= 2 * d[:, 0] + (n + 64) * 2.0 ** -22 + 2.0 ** -21 * lse.abs()).all())
        at += m


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("r", [10, 22, 28, 32, 36, 45, 60])
def test_attention_weight_on_pages_of_small_scales(E, r, int8):
    """All of a row's weight on pages whose value scale is 2^-r of one that has next to none of it,
    before or after them, behind the causal diagonal of the same chunk, or outside the window: either
    kernel gives what the pages with the weight hold."""
    small = 1.3 * 2.0 ** -r
    for name, request, page, window, scales, heavy in (
            ("large first", (192, 64), 64, 0, [1.0, small, small], (1,)),
            ("large second", (192, 64), 64, 0, [small, 1.0, small], (0,)),
            ("behind the diagonal", (64, 64), 16, 0, [small, small, small, 1.0], (0, 1, 2)),
            ("outside the window", (192, 64), 16, 40, [small] * 4 + [1.0] + [small] * 7, tuple(range(5, 12)))):
        for dim in (64, 128, 256):
            c = Case([request, (40, 40)], 2, 2, dim, page, int8, "bf16", window=window, seed=20 + r)
            place_weight(c, scales, heavy, 64)
            for max_q in (1, 64):
                say(f"  scales 2^-{r} {name} dim {dim} max_q {max_q}")
                check_weights(c, c.call(E, max_q=max_q))


@pytest.mark.parametrize("gap", [10, 30, 60])
def test_attention_weight_on_pages_of_zeros(E, gap):
    """All of a row's weight on pages of zeros (value scale 0): the others count for their share of it."""
    for scales, heavy in (([0.0, 1.0, 1.0], (0,)), ([1.0, 0.0, 0.03], (1,)), ([0.0, 0.0, 0.0], (1,))):
        c = Case([(192, 64), (40, 40)], 2, 2, 128, 64, False, "bf16", seed=31)
        place_weight(c, scales, heavy, gap)
        for max_q in (1, 64):
            check_weights(c, c.call(E, max_q=max_q))


@pytest.mark.parametrize("spread", [2.0 ** 60, 2.0 ** 100])
def test_attention_scales_across_the_range_of_fp32(E, spread):
    """Neighbouring pages whose value scales lie up to 2^200 apart: rows that see only the small ones
    give their values, rows with weight on both give the large ones', and no sum overflows."""
    for scales, heavy in (([1 / spread, spread, 1 / spread], (0, 2)), ([spread, 1 / spread, spread], (1,)),
                          ([1 / spread, 1 / spread, spread], (0, 1, 2))):
        c = Case([(192, 192)], 2, 2, 128, 64, False, "bf16", seed=33)
        place_weight(c, scales, heavy, 64)
        for max_q in (1, 192):
            check_weights(c, c.call(E, max_q=max_q))


def test_attention_zero_scales_and_large_scores(E):
    c = Case([(500, 1), (200, 60)], 8, 2, 128, 16, True, "bf16", seed=5)
    c.vs[:, 0] = 0.0
    c.ks[:, 1] *= 300.0        # scores of thousands: one key takes all
    c.check(c.call(E))


def test_attention_missing_pages_count_as_unseen(E):
    for requests in ([(500, 1), (300, 2)], [(500, 300), (300, 30)]):
        c = Case(requests, 8, 2, 128, 32, False, "bf16", seed=6)
        c.table[0, 3], c.table[1, 0] = -1, c.pages + 7
        c.check(c.call(E))


def test_attention_not_a_number_reaches_only_those_who_see_it(E):
    """One token's value is not a number, which makes its page's scale one: causal queries before
    the page, other heads and other requests keep their bits."""
    c = Case([(200, 150), (90, 90)], 4, 2, 128, 16, False, "bf16", seed=8)
    clean = c.call(E)
    p = int(c.table[0, 10])          # tokens 160 .. 175 of the first request
    c.vs[p, 1] = float("nan")
    c.vc[p, 1, :, 5] = 0x7F
    out = c.call(E)
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[110:150, 2:] = False        # queries at positions 160 .. 199 of the heads that read kv head 1
    assert torch.equal(out[keep], clean[keep])
    assert torch.isnan(out[110:150, 2:]).all()
    c.vs[p, 1] = 0.01
    c.vc[p, 1, :, 5] = 0x11
    c.ks[p, 1] = float("nan")
    out = c.call(E)
    assert torch.equal(out[keep], clean[keep]) and torch.isnan(out[110:150, 2:]).all()


def test_attention_strided_rows_and_spare_rows(E):
    """Queries inside a fused projection's rows, outputs inside wider rows, and a batch with more
    rows than its requests use: those stay as they are."""
    for requests in ([(700, 1), (3000, 1), (20, 1)], [(300, 100), (77, 77)]):
        c = Case(requests, 8, 2, 64, 16, False, "bf16", spare_q=5, seed=9)
        n = c.total
        wide = torch.randn((n, 8 * 64 + 256), device="cuda").to(torch.bfloat16)
        wide[:, : 8 * 64] = c.q.view(n, -1)
        out = torch.full((n, 8 * 64 + 64), 7.0, dtype=torch.bfloat16, device="cuda")
        c.call(E, q=wide, out=out)
        got = out[:, : 8 * 64].reshape(n, 8, 64)
        c.check(got)
        assert (out[:, 8 * 64:] == 7.0).all() and (got[n - 5:] == 7.0).all() and torch.isnan(c.lse[n - 5:]).all()


def test_attention_repeats_its_bits(E):
    for requests in ([(4000, 1), (900, 1)], [(900, 700), (100, 40)]):
        c = Case(requests, 16, 2, 128, 64, False, "bf16", seed=10)
        a = c.call(E)
        for _ in range(3):
            assert torch.equal(a, c.call(E))


def test_attention_without_lse(E):
    c = Case([(700, 1), (64, 64)], 8, 2, 128, 64, False, "bf16", seed=11)
    c.check(c.call(E, lse=False), lse=False)


def test_attention_past_32_bit_offsets(E):
    """A cache of more than 2^32 codes, its last pages in use."""
    page, heads, dim = 64, 8, 128
    pages = (1 << 32) // (page * heads * dim) + 40
    for requests in ([(1200, 1), (300, 1)], [(1200, 100), (300, 20)]):
        c = Case(requests, 16, heads, dim, page, False, "bf16", seed=12, first_page=pages - 30, pages=pages)
        c.check(c.call(E))


def test_attention_of_far_more_queries_than_max_q(E):
    """2^28 query rows of one request in a call that says one: they fit a grid, and get what the same
    queries get in a small call."""
    some, times = 64, (1 << 18) + 1
    c = Case([(100, some)], 16, 1, 64, 64, False, "bf16", causal=False, seed=14)
    if torch.cuda.mem_get_info()[0] < 6 * c.q.numel() * times:
        pytest.skip("needs more device memory")
    want = c.call(E, lse=False)
    c.check(want, lse=False)
    q = c.q.repeat(times, 1, 1)
    out = torch.empty_like(q)
    cu = ints([0, len(q)])
    cache = E.kv8_cache(c.kc.data_ptr(), c.vc.data_ptr(), c.ks.data_ptr(), c.vs.data_ptr(), c.pages, 1, 64, 64)
    call = E.kv8_attention_args(q.data_ptr(), out.data_ptr(), cu.data_ptr(), c.lens.data_ptr(), c.table.data_ptr(), c.table.shape[1],
                                1, len(q), 16, E.BF16, scale=1 / 8, causal=False, max_q=1, max_len=100)
    assert E.kv8_attention_workspace(cache, call) == 0
    E.kv8_attention(cache, call, 0, 0, stream())
    torch.cuda.synchronize()
    del q
    for part in out.split(some * 1024):
        got = part.view(-1, some, 16, 64)
        assert torch.equal(got, want[None].expand_as(got))
    del out, part, got
    torch.cuda.empty_cache()


def test_append_past_32_bit_offsets(E):
    page, heads, dim = 64, 8, 128
    pages = (1 << 32) // (page * heads * dim) + 2
    kc, vc = [torch.zeros(pages * heads * page * dim, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ks, vs = torch.zeros((pages, heads), device="cuda"), torch.zeros((pages, heads), device="cuda")
    x = torch.ones((2, heads * dim), dtype=torch.bfloat16, device="cuda")
    cache = E.kv8_cache(kc.data_ptr(), vc.data_ptr(), ks.data_ptr(), vs.data_ptr(), pages, heads, page, dim)
    s = torch.tensor([pages * page - 2, pages * page - 1], dtype=torch.int64, device="cuda")
    E.kv8_append(cache, x.data_ptr(), x.data_ptr(), E.BF16, heads * dim, heads * dim, s.data_ptr(), 2, stream())
    torch.cuda.synchronize()
    assert (kc.view(pages, heads, page, dim)[-1, :, -2:] == 0x7E).all() and int((kc != 0).sum()) == 2 * heads * dim
    assert (vc.view(pages, heads, dim, page)[-1, :, :, -2:] == 0x7E).all() and int((vc != 0).sum()) == 2 * heads * dim


def test_step_on_another_stream_and_in_a_graph(E):
    """Slots, append and attention of one decoding step, captured once and replayed as the
    requests grow, against the same calls made one by one."""
    page, heads, q_heads, dim, n = 16, 2, 8, 64, 5
    cached = [0, 15, 16, 100, 33]
    pages, width = 80, 12
    g = torch.Generator("cuda").manual_seed(2)

    def fresh():
        perm = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).to(torch.int32)
        t = torch.full((n, width), -1, dtype=torch.int32)
        at = 0
        for b, c in enumerate(cached):
            k = -(-c // page)
            t[b, :k] = perm[at: at + k]
            at += k
        gg = torch.Generator("cuda").manual_seed(3)
        kc = torch.randint(0, 120, (pages, heads, page, dim), generator=gg, device="cuda", dtype=torch.uint8)
        vc = torch.randint(0, 120, (pages, heads, dim, page), generator=gg, device="cuda", dtype=torch.uint8)
        sc = torch.full((pages, heads), 0.02, device="cuda")
        return dict(table=t.cuda(), free=perm[at:].cuda(), n_free=ints([pages - at]), kc=kc, vc=vc, ks=sc, vs=sc.clone(),
                    cached=ints(cached), new=ints([1] * n), lens=ints([0] * n), cu=ints([0] * (n + 1)),
                    slots=torch.zeros(n, dtype=torch.int64, device="cuda"), used=ints([0]), status=ints([0]),
                    qkv=torch.zeros((n, (q_heads + 2 * heads) * dim), dtype=torch.bfloat16, device="cuda"),
                    out=torch.zeros((n, q_heads * dim), dtype=torch.bfloat16, device="cuda"), room=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))

    def step(s):
        E.kv8_slots(s["cached"].data_ptr(), s["new"].data_ptr(), n, page, s["free"].data_ptr(), s["n_free"].data_ptr(),
                    s["table"].data_ptr(), width, s["lens"].data_ptr(), s["cu"].data_ptr(), s["slots"].data_ptr(), n,
                    s["used"].data_ptr(), s["status"].data_ptr(), stream())
        cache = E.kv8_cache(s["kc"].data_ptr(), s["vc"].data_ptr(), s["ks"].data_ptr(), s["vs"].data_ptr(), pages, heads, page, dim)
        row = s["qkv"].stride(0)
        k = s["qkv"].data_ptr() + 2 * q_heads * dim
        E.kv8_append(cache, k, k + 2 * heads * dim, E.BF16, row, row, s["slots"].data_ptr(), n, stream())
        call = E.kv8_attention_args(s["qkv"].data_ptr(), s["out"].data_ptr(), s["cu"].data_ptr(), s["lens"].data_ptr(),
                                    s["table"].data_ptr(), width, n, n, q_heads, E.BF16, scale=0.125, max_q=1,
                                    max_len=width * page, q_row=row)
        assert E.kv8_attention_workspace(cache, call) <= s["room"].numel()
        E.kv8_attention(cache, call, s["room"].data_ptr(), s["room"].numel(), stream())
        # the next step's state
        s["cached"].copy_(s["lens"])
        took = s["used"].long()
        s["free"].copy_(torch.roll(s["free"], 0).gather(0, (torch.arange(len(s["free"]), device="cuda") + took).clamp(max=len(s["free"]) - 1)))
        s["n_free"].sub_(s["used"])

    eager, graphed = fresh(), fresh()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    saved = {k: v.clone() for k, v in graphed.items()}
    with torch.cuda.stream(side):
        step(graphed)
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(graphed)
    for k, v in saved.items():
        graphed[k].copy_(v)
    for i in range(20):
        x = torch.randn(eager["qkv"].shape, generator=g, device="cuda").to(torch.bfloat16)
        eager["qkv"].copy_(x)
        graphed["qkv"].copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        for k in ("table", "lens", "cu", "slots", "kc", "vc", "ks", "vs", "out", "used", "status"):
            assert torch.equal(eager[k], graphed[k]), (i, k)
    assert eager["lens"].tolist() == [c + 20 for c in cached] and int(eager["status"]) == 0
