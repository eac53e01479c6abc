"""One whole transformer layer served from compressed weights: the attention of
serve_attention_layer.py from FP8 containers, between norms and with rotary positions, and an MLP
from INT8 containers.

A step of a batch of requests, prompts and single tokens alike, on the residual stream r:

  norm of r to E4M3, a scale for each 128             ep_norm
  fused projection, pages and slots of the new tokens  ep_gemm_fp8_block, ep_kv8_slots
  queries and keys turned by their positions, in place ep_rope
  into the paged cache, attention, output projection   ep_kv8_append, ep_kv8_attention, ep_quant_fp8_block, ep_gemm_fp8_block
  r += that, and the norm of it to INT8 rows           ep_norm
  both halves of the MLP in one product                ep_gemm_i8_scaled
  their gated activation to INT8 rows                  ep_glu
  down projection; r += that                           ep_gemm_i8_scaled, ep_norm

Positions come from the lengths that ep_kv8_slots leaves on the device, so that a step of single
tokens is captured into a graph and replayed.  The residual streams are random; what comes out is
compared with the same layer in 32-bit torch operations without any quantisation of activations,
keys or values.

    python examples/serve_transformer_layer.py [--steps N] [--cache e4m3|int8]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import serve_attention_layer as A  # noqa: E402
from serve_attention_layer import DIM, E, HIDDEN, KV_HEADS, PAGE, PAGES, Q_HEADS, QKV, W, WIDTH  # noqa: E402

INNER = 2816                             # of the MLP
BASE, FACTOR, TRAINED = 10000.0, 4.0, 128.0   # frequencies stretched for four times the trained length


def empty(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda")


class Layer(A.Layer):
    """The attention's weights and cache, the MLP's weights, norm weights and frequencies."""

    def __init__(self, requests, cache_dtype):
        super().__init__(requests, cache_dtype)
        blobs = [E.encode(W.ragged_tensor(seed, rows, cols, scale=0.03), 4.0, container=E.CONT_INT8_ROW)[0]
                 for seed, rows, cols in ((3, 2 * INNER, HIDDEN), (4, HIDDEN, INNER))]
        decoded = []
        for blob in blobs:                   # INT8 codes and a scale for each row
            w, delta, status = E.decode(blob, E.INT8)
            if int(status.item()):
                raise RuntimeError("corrupt blob")
            decoded.append((w, delta))
        (self.w_in, self.d_in), (self.w_down, self.d_down) = decoded
        self.w1, self.w2 = [(1 + 0.1 * torch.randn(HIDDEN, device="cuda")).to(torch.bfloat16) for _ in range(2)]
        freqs = E.rope_freqs(DIM, BASE, E.ROPE_TURNS, factor=FACTOR, trained_len=TRAINED, low=1.0, high=4.0)
        self.freqs = torch.from_numpy(freqs.view("int64")).cuda()

    def i8_product(self, q, s, w, delta):
        m, k, n, stream = q.shape[0], q.shape[1], w.shape[0], torch.cuda.current_stream().cuda_stream
        y, room = empty(m, n), empty(E.gemm_i8_scaled_workspace(m, n, k), dtype=torch.uint8)
        E.gemm_i8_scaled(q.data_ptr(), s.data_ptr(), w.data_ptr(), delta.data_ptr(), y.data_ptr(), m, n, k, d_ws=room.data_ptr(),
                         ws_bytes=room.numel(), stream=stream)
        return y

    def step(self, r, new, max_new):
        """The residual stream of the requests' new tokens, after the layer."""
        stream, m = torch.cuda.current_stream().cuda_stream, r.shape[0]
        x, xs, qkv = empty(m, HIDDEN, dtype=torch.float8_e4m3fn), empty(m, HIDDEN // 128, dtype=torch.float32), empty(m, QKV)
        E.norm(E.norm_call(r.data_ptr(), m, HIDDEN, d_y=x.data_ptr(), y_dtype=E.FP8_E4M3, d_y_scale=xs.data_ptr(), d_w=self.w1.data_ptr()),
               stream)
        E.gemm_fp8_block(x.data_ptr(), xs.data_ptr(), self.w_qkv.data_ptr(), self.d_qkv.data_ptr(), qkv.data_ptr(), m, QKV, HIDDEN,
                         w_scales=E.SCALE_ROW, stream=stream)
        slots = empty(m, dtype=torch.int64)
        E.kv8_slots(self.cached.data_ptr(), new.data_ptr(), self.n, PAGE, self.free.data_ptr(), self.n_free.data_ptr(),
                    self.table.data_ptr(), WIDTH, self.lens.data_ptr(), self.cu.data_ptr(), slots.data_ptr(), m, self.used.data_ptr(),
                    self.status.data_ptr(), stream)
        k = qkv.data_ptr() + 2 * Q_HEADS * DIM          # keys, then values, behind the queries in a row
        E.rope(E.rope_call(qkv.data_ptr(), qkv.data_ptr(), self.freqs.data_ptr(), m, Q_HEADS, DIM, E.BF16, d_k=k, d_k_out=k, k_heads=KV_HEADS,
                           d_cu=self.cu.data_ptr(), d_len=self.lens.data_ptr(), n_req=self.n, q_row=QKV, q_out_row=QKV, k_row=QKV,
                           k_out_row=QKV), stream)
        E.kv8_append(self.cache, k, k + 2 * KV_HEADS * DIM, E.BF16, QKV, QKV, slots.data_ptr(), m, stream)
        heads = empty(m, Q_HEADS * DIM)
        call = E.kv8_attention_args(qkv.data_ptr(), heads.data_ptr(), self.cu.data_ptr(), self.lens.data_ptr(), self.table.data_ptr(),
                                    WIDTH, self.n, m, Q_HEADS, E.BF16, scale=1 / math.sqrt(DIM), max_q=max_new, max_len=WIDTH * PAGE,
                                    q_row=QKV)
        room = empty(E.kv8_attention_workspace(self.cache, call), dtype=torch.uint8)
        E.kv8_attention(self.cache, call, room.data_ptr(), room.numel(), stream)
        # the pages taken leave the list of free ones; the lengths become the next step's
        self.cached.copy_(self.lens)
        at = torch.arange(PAGES, device="cuda") + self.used
        self.free.copy_(self.free[at.clamp_(max=PAGES - 1)])
        self.n_free.sub_(self.used)

        block = self.project(heads, self.w_out, self.d_out)
        h, q, s = empty(m, HIDDEN), empty(m, HIDDEN, dtype=torch.int8), empty(m, dtype=torch.float32)
        E.norm(E.norm_call(block.data_ptr(), m, HIDDEN, d_res=r.data_ptr(), d_res_out=h.data_ptr(), d_y=q.data_ptr(), y_dtype=E.INT8,
                           d_y_scale=s.data_ptr(), d_w=self.w2.data_ptr()), stream)
        both = self.i8_product(q, s, self.w_in, self.d_in)
        q, s = empty(m, INNER, dtype=torch.int8), empty(m, dtype=torch.float32)
        E.glu(both.data_ptr(), both.data_ptr() + 2 * INNER, E.BF16, m, INNER, E.ACT_SILU, q.data_ptr(), E.INT8, s.data_ptr(),
              a_row=2 * INNER, b_row=2 * INNER, stream=stream)
        block = self.i8_product(q, s, self.w_down, self.d_down)
        E.norm(E.norm_call(block.data_ptr(), m, HIDDEN, d_res=h.data_ptr(), d_res_out=h.data_ptr(), pre=E.NORM_NONE), stream)
        return h


def plain(layer, stream_in):
    """The layer in 32 bits on one request's residual stream, none of it quantised but the weights."""
    def normed(x, w):
        return x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6) * w.float()

    def turned(x):                           # [tokens, heads, DIM]
        i = torch.arange(DIM // 2, dtype=torch.float64, device="cuda")
        theta = BASE ** (-2 * i / DIM)
        keep = ((TRAINED * theta / (2 * math.pi) - 1) / 3).clamp(0, 1)
        angle = torch.arange(len(x), device="cuda").double()[:, None] * theta * (keep + (1 - keep) / FACTOR)
        co, si = angle.cos().float()[:, None], angle.sin().float()[:, None]
        a, b = x[..., : DIM // 2], x[..., DIM // 2:]
        return torch.cat((a * co - b * si, a * si + b * co), 2)

    r = stream_in.float()
    n = len(r)
    qkv = normed(r, layer.w1) @ (layer.w_qkv.float() * layer.d_qkv[:, None]).t()
    q, k, v = [t.view(n, -1, DIM) for t in qkv.split([Q_HEADS * DIM, KV_HEADS * DIM, KV_HEADS * DIM], 1)]
    q = turned(q).transpose(0, 1).contiguous()
    k, v = [t.transpose(0, 1).repeat_interleave(Q_HEADS // KV_HEADS, 0).contiguous() for t in (turned(k), v)]
    score = q @ k.transpose(1, 2).contiguous() / math.sqrt(DIM)
    score.masked_fill_(torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1), -math.inf)
    heads = (torch.softmax(score, -1) @ v).transpose(0, 1).reshape(n, -1)
    r = r + heads @ (layer.w_out.float() * layer.d_out[:, None]).t()
    a, b = (normed(r, layer.w2) @ (layer.w_in.float() * layer.d_in[:, None]).t()).split(INNER, 1)
    return r + (a / (1 + torch.exp(-a)) * b) @ (layer.w_down.float() * layer.d_down[:, None]).t()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40, help="single-token steps after the prompts")
    ap.add_argument("--cache", choices=("e4m3", "int8"), default="e4m3")
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    prompts = [70, 301, 5]
    layer = Layer(len(prompts), E.FP8_E4M3 if a.cache == "e4m3" else E.INT8)
    stream_in = [torch.randn((p + a.steps, HIDDEN), device="cuda").to(torch.bfloat16) for p in prompts]
    outs = [[] for _ in prompts]

    new = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    y = layer.step(torch.cat([r[:p] for r, p in zip(stream_in, prompts)]), new, max(prompts))
    for i, part in enumerate(y.split(prompts)):
        outs[i].append(part)

    if a.steps:
        # single tokens: the first step as it is, the others from a graph of the second
        ones, x = torch.ones(len(prompts), dtype=torch.int32, device="cuda"), empty(len(prompts), HIDDEN)
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        for s in range(a.steps):
            x.copy_(torch.stack([r[p + s] for r, p in zip(stream_in, prompts)]))
            if s == 0:
                side.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(side):
                    y = layer.step(x, ones, 1)
                torch.cuda.current_stream().wait_stream(side)
            else:
                if s == 1:
                    torch.cuda.synchronize()
                    with torch.cuda.graph(graph, stream=side):
                        captured = layer.step(x, ones, 1)
                graph.replay()
                y = captured
            for i in range(len(prompts)):
                outs[i].append(y[i: i + 1].clone())
    torch.cuda.synchronize()
    if int(layer.status.item()):
        raise RuntimeError(f"cache tables: status {int(layer.status.item())}")
    worst = 0.0
    for r, o in zip(stream_in, outs):
        got, want = torch.cat(o).float(), plain(layer, r)
        worst = max(worst, float(((got - want).norm() / (want - r.float()).norm())))
    print(f"{len(prompts)} requests, {sum(prompts)} prompt tokens, {a.steps} steps, {a.cache} cache: what the layer adds is "
          f"off the unquantised layer's by {100 * worst:.2f} % (2-norm)", flush=True)
    return worst


if __name__ == "__main__":
    main()
