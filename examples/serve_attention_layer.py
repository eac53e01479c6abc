"""One attention layer served from compressed weights, everything between its ends in 8 bits.

The fused query/key/value projection and the output projection are entropy-coded FP8 containers
(ep_encode_cpu).  They are decoded once, by a prepared stack, to E4M3 codes with a scale for each
row.  A step of a batch of requests, prompts and single tokens alike, is then

  activations to E4M3, a scale for each 128            ep_quant_fp8_block
  fused projection                                     ep_gemm_fp8_block
  pages and slots of the new tokens                    ep_kv8_slots
  their keys and values into the 8-bit paged cache     ep_kv8_append
  attention of their queries over the cache            ep_kv8_attention
  the result to E4M3, output projection                ep_quant_fp8_block, ep_gemm_fp8_block

Nothing in a step waits for the GPU, and its buffers come from torch's pool: a step of single tokens is
captured into a graph and replayed.  The hidden states are random; what comes out is compared with the same layer in
32-bit torch operations without any quantisation of activations, keys or values.

    python examples/serve_attention_layer.py [--steps N] [--cache e4m3|int8]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_34185_amd import entropack as E  # noqa: E402
from paper_2609_34185_amd import workloads as W  # noqa: E402

HIDDEN, Q_HEADS, KV_HEADS, DIM = 1024, 8, 2, 128
QKV = (Q_HEADS + 2 * KV_HEADS) * DIM
PAGE, WIDTH, PAGES = 64, 16, 64          # tokens of a page, pages of a request at most, pages in all


def compressed(rows, cols, seed):
    """An FP8-container blob of a random projection at 4 bits a weight."""
    blob, stats = E.encode(W.ragged_tensor(seed, rows, cols, scale=0.03), 4.0, container=E.CONT_FP8_ROW)
    print(f"projection {rows} x {cols}: {stats['rate_stored']:.2f} bits a weight stored", flush=True)
    return blob


def decoded(blobs):
    """E4M3 codes and row scales of every blob, one launch for all of them."""
    layers, out, keep = [], [], []
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for blob in blobs:
        info, d = E.blob_info(blob), E.to_device(blob)
        w = torch.empty((info.rows, info.cols), dtype=torch.float8_e4m3fn, device="cuda")
        delta = torch.empty(info.rows, device="cuda")
        layers.append((info, d.data_ptr(), w.data_ptr(), delta.data_ptr(), E.FP8_E4M3))
        out.append((w, delta))
        keep.append(d)
    room = torch.empty(E.stack_workspace(len(layers)), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    E.stack_decode(E.stack_prepare(layers, room.data_ptr(), room.numel(), stream), status.data_ptr(), stream)
    torch.cuda.synchronize()
    if int(status.item()):
        raise RuntimeError("corrupt blob")
    return out


class Layer:
    """The layer's weights, its cache, and what its requests hold of it."""

    def __init__(self, requests, cache_dtype):
        dev = "cuda"
        self.n = requests
        (self.w_qkv, self.d_qkv), (self.w_out, self.d_out) = decoded([compressed(QKV, HIDDEN, 1), compressed(HIDDEN, Q_HEADS * DIM, 2)])
        self.kc = torch.zeros((PAGES, KV_HEADS, PAGE, DIM), dtype=torch.uint8, device=dev)
        self.vc = torch.zeros((PAGES, KV_HEADS, DIM, PAGE), dtype=torch.uint8, device=dev)
        self.ks, self.vs = torch.zeros((PAGES, KV_HEADS), device=dev), torch.zeros((PAGES, KV_HEADS), device=dev)
        self.cache = E.kv8_cache(self.kc.data_ptr(), self.vc.data_ptr(), self.ks.data_ptr(), self.vs.data_ptr(), PAGES, KV_HEADS,
                                 PAGE, DIM, cache_dtype)
        self.table = torch.full((requests, WIDTH), -1, dtype=torch.int32, device=dev)
        self.free = torch.randperm(PAGES, device=dev).to(torch.int32)
        self.n_free = torch.full((1,), PAGES, dtype=torch.int32, device=dev)
        self.cached, self.lens = [torch.zeros(requests, dtype=torch.int32, device=dev) for _ in range(2)]
        self.cu = torch.zeros(requests + 1, dtype=torch.int32, device=dev)
        self.used, self.status = [torch.zeros(1, dtype=torch.int32, device=dev) for _ in range(2)]

    def project(self, x, w, delta):
        m, k, n = x.shape[0], x.shape[1], w.shape[0]
        q = torch.empty((m, k), dtype=torch.float8_e4m3fn, device="cuda")
        s, y = torch.empty((m, -(-k // 128)), device="cuda"), torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
        stream = torch.cuda.current_stream().cuda_stream
        E.quant_fp8_block(x.data_ptr(), E.BF16, m, k, q.data_ptr(), s.data_ptr(), stream=stream)
        E.gemm_fp8_block(q.data_ptr(), s.data_ptr(), w.data_ptr(), delta.data_ptr(), y.data_ptr(), m, n, k, w_scales=E.SCALE_ROW,
                         stream=stream)
        return y

    def step(self, x, new, max_new):
        """Hidden states x of the requests' new tokens (new: how many each has, on the device)."""
        stream, total = torch.cuda.current_stream().cuda_stream, x.shape[0]
        qkv = self.project(x, self.w_qkv, self.d_qkv)
        slots = torch.empty(total, dtype=torch.int64, device="cuda")
        E.kv8_slots(self.cached.data_ptr(), new.data_ptr(), self.n, PAGE, self.free.data_ptr(), self.n_free.data_ptr(),
                    self.table.data_ptr(), WIDTH, self.lens.data_ptr(), self.cu.data_ptr(), slots.data_ptr(), total,
                    self.used.data_ptr(), self.status.data_ptr(), stream)
        k = qkv.data_ptr() + 2 * Q_HEADS * DIM          # keys, then values, behind the queries in a row
        E.kv8_append(self.cache, k, k + 2 * KV_HEADS * DIM, E.BF16, QKV, QKV, slots.data_ptr(), total, stream)
        heads = torch.empty((total, Q_HEADS * DIM), dtype=torch.bfloat16, device="cuda")
        call = E.kv8_attention_args(qkv.data_ptr(), heads.data_ptr(), self.cu.data_ptr(), self.lens.data_ptr(), self.table.data_ptr(),
                                    WIDTH, self.n, total, Q_HEADS, E.BF16, scale=1 / math.sqrt(DIM), max_q=max_new,
                                    max_len=WIDTH * PAGE, q_row=QKV)
        room = torch.empty(E.kv8_attention_workspace(self.cache, call), dtype=torch.uint8, device="cuda")
        E.kv8_attention(self.cache, call, room.data_ptr(), room.numel(), stream)
        # the pages taken leave the list of free ones; the lengths become the next step's
        self.cached.copy_(self.lens)
        at = torch.arange(PAGES, device="cuda") + self.used
        self.free.copy_(self.free[at.clamp_(max=PAGES - 1)])
        self.n_free.sub_(self.used)
        return self.project(heads, self.w_out, self.d_out)


def plain(layer, hidden):
    """The layer in 32 bits on one request's hidden states, none of them, nor keys or values, quantised."""
    x = hidden.float()
    qkv = x @ (layer.w_qkv.float() * layer.d_qkv[:, None]).t()
    q, k, v = qkv.split([Q_HEADS * DIM, KV_HEADS * DIM, KV_HEADS * DIM], 1)
    n = len(x)
    q = q.view(n, Q_HEADS, DIM).transpose(0, 1)
    k, v = [t.view(n, KV_HEADS, DIM).transpose(0, 1).repeat_interleave(Q_HEADS // KV_HEADS, 0).contiguous() for t in (k, v)]
    score = q.contiguous() @ k.transpose(1, 2).contiguous() / math.sqrt(DIM)
    score.masked_fill_(torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1), -math.inf)
    heads = torch.softmax(score, -1) @ v
    return heads.transpose(0, 1).reshape(n, -1) @ (layer.w_out.float() * layer.d_out[:, None]).t()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40, help="single-token steps after the prompts")
    ap.add_argument("--cache", choices=("e4m3", "int8"), default="e4m3")
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    prompts = [70, 301, 5]
    layer = Layer(len(prompts), E.FP8_E4M3 if a.cache == "e4m3" else E.INT8)
    hidden = [torch.randn((p + a.steps, HIDDEN), device="cuda").to(torch.bfloat16) for p in prompts]
    outs = [[] for _ in prompts]

    new = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    y = layer.step(torch.cat([h[:p] for h, p in zip(hidden, prompts)]), new, max(prompts))
    for i, part in enumerate(y.split(prompts)):
        outs[i].append(part)

    if a.steps:
        # single tokens: the first step as it is, the others from a graph of the second
        ones, x = torch.ones(len(prompts), dtype=torch.int32, device="cuda"), torch.empty((len(prompts), HIDDEN), dtype=torch.bfloat16, device="cuda")
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        for s in range(a.steps):
            x.copy_(torch.stack([h[p + s] for h, p in zip(hidden, prompts)]))
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
    for h, o in zip(hidden, outs):
        got, want = torch.cat(o).float(), plain(layer, h)
        worst = max(worst, float((got - want).norm() / want.norm()))
    print(f"{len(prompts)} requests, {sum(prompts)} prompt tokens, {a.steps} steps, {a.cache} cache: "
          f"off the unquantised layer by {100 * worst:.2f} % (2-norm)", flush=True)
    return worst


if __name__ == "__main__":
    main()
