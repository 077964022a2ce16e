"""A decoder layer whose weights stay compressed in GPU memory: a prompt, then tokens one by one, for sequences that share a prefix.

The seven matrices of a Llama-shaped layer are quantised and compressed once.  A prompt decodes them to bf16 (dc_decompress_dequant_bf16_layer)
and multiplies its rows together; a generated token goes through the products that decode as they multiply (dc_decompress_gemv_layer).
Between the products, both ways: rotary positions and the append to the paged cache (dc_kv_append) and the attention over it
(dc_attention_paged), with a sliding window and sinks if wanted.  The cache is of bf16, or of 8 bits with a scale for every 32 tokens of a head.

  python examples/decoder_layer.py [--hidden 4096 --heads 32 --kv-heads 32 --ffn 11008 --prompt 1024 --tokens 32 --window 0 --sinks 0 --cache bf16|i8]
"""
import argparse
import os
import sys
import time

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2502_15443_amd as dc  # noqa: E402

PAGE, SCALE_TOKENS = 64, 32


def compressed(matrices, seed):
    """Random weights, quantised per row with small values pruned, in one blob: the blob, the table and each matrix's scales."""
    p = dc.Params(65536, 256)
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = torch.cuda.current_stream().cuda_stream
    blobs, tables, scales, first, at, chunks = [], [], [], [], 0, 0
    for rows, cols in matrices:
        w = torch.randn(rows, cols, generator=g, device="cuda") * cols ** -0.5
        scale = w.abs().amax(1) / 127
        q = torch.round(w / scale[:, None]).clamp_(-127, 127)
        q[q.abs() <= 1] = 0
        q = q.to(torch.int8)
        cap, n = dc.compress_bound(q.numel(), p)
        blob, table = torch.zeros(cap, dtype=torch.uint8, device="cuda"), torch.zeros(n, 2, dtype=torch.int64, device="cuda")
        ws_bytes = dc.compress_chunks_dev_workspace(q.numel(), p)
        ws, result = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
        dc.compress_chunks_dev(q, q.numel(), p, blob, cap, table, n, ws, ws_bytes, result, st)
        size, err = result.tolist()
        if err:
            raise RuntimeError("the blob does not fit its bound")
        table[:, 0] += at
        blobs.append(blob[:size])
        tables.append(table)
        scales.append(scale)
        first.append(chunks)
        at += size
        chunks += n
    return p, torch.cat(blobs), torch.cat(tables), scales, first


class DecoderLayer:
    def __init__(self, hidden, heads, kv_heads, ffn, pages, n_positions, window=0, sinks=0, seed=0, head_dim=128, cache="bf16"):
        self.hidden, self.heads, self.kv_heads, self.d = hidden, heads, kv_heads, head_dim
        self.window, self.sinks = window, sinks
        width, kv_width = heads * head_dim, kv_heads * head_dim
        # (rows, cols): q k v o gate up down
        self.shapes = [(width, hidden), (kv_width, hidden), (kv_width, hidden), (hidden, width), (ffn, hidden), (ffn, hidden), (hidden, ffn)]
        self.params, self.blob, self.table, self.scales, self.first = compressed(self.shapes, seed)
        self.first.append(self.table.shape[0])
        self.weights = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in self.shapes]  # the decompression buffer of prompts
        ws = dc.decompress_gemv_workspace(self.table.shape[0])
        self.gemv_ws = torch.empty(ws, dtype=torch.uint8, device="cuda")
        angle = torch.arange(n_positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(head_dim // 2, dtype=torch.float64) / (head_dim // 2))
        self.cos, self.sin, self.n_positions = angle.cos().float().cuda(), angle.sin().float().cuda(), n_positions
        shape = (pages, kv_heads, PAGE, head_dim)
        self.k_pool, self.v_pool = (torch.zeros(shape, dtype=torch.int8 if cache == "i8" else torch.bfloat16, device="cuda") for _ in range(2))
        if cache == "i8":
            self.k_scale, self.v_scale = (torch.zeros((pages, kv_heads, PAGE // SCALE_TOKENS), device="cuda") for _ in range(2))
            self.cache = dc.KVCache(self.k_pool, self.v_pool, pages, kv_heads, head_dim, PAGE, dc.TYPE_I8, rows_type=dc.TYPE_BF16,
                                    scale_tokens=SCALE_TOKENS, k_scale_dev=self.k_scale, v_scale_dev=self.v_scale)
        else:
            self.cache = dc.KVCache(self.k_pool, self.v_pool, pages, kv_heads, head_dim, PAGE)

    def gemv(self, which, x, out):
        """One token: products of consecutive matrices with the same activations, decoded as they are multiplied; fp32 results."""
        st = torch.cuda.current_stream().cuda_stream
        a, b = self.first[which[0]], self.first[which[-1] + 1]
        mats, at = [], 0
        for i in which:
            rows, cols = self.shapes[i]
            mats.append(dc.Matrix(self.first[i] - a, rows, cols, self.scales[i], x_bf16_dev=x, y_accum_dev=out[at:at + rows]))
            at += rows
        dc.decompress_gemv_layer(self.blob, self.blob.numel(), self.table[a:], b - a, self.params, mats, self.gemv_ws, self.gemv_ws.numel(), st)
        return out

    def decode_weights(self):
        st = torch.cuda.current_stream().cuda_stream
        mats = [dc.Matrix(self.first[i], r, c, self.scales[i], dst_bf16_dev=self.weights[i], dst_cap_elems=r * c) for i, (r, c) in enumerate(self.shapes)]
        dc.decompress_dequant_bf16_layer(self.blob, self.blob.numel(), self.table, self.table.shape[0], self.params, mats, st)

    def attend(self, qkv, batch):
        """Rows [rows, heads + 2 kv_heads, head_dim] (fp32 or bf16): turned, put into the cache, attended; bf16 [rows, heads * head_dim]."""
        st = torch.cuda.current_stream().cuda_stream
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
        turned = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        rows = dc.KVRows(dc.TYPE_F32 if qkv.dtype == torch.float32 else dc.TYPE_BF16, self.heads, k, v, q, turned, rot_dim=self.d,
                         cos_dev=self.cos, sin_dev=self.sin, n_positions=self.n_positions)
        dc.kv_append(self.cache, batch, rows, st)
        out = torch.empty_like(turned)
        attention = dc.Attention(self.heads, turned, out, None, self.d ** -0.5, window=self.window, sinks=self.sinks)
        n = dc.attention_paged_workspace(self.cache, batch, attention)
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        dc.attention_paged(self.cache, batch, attention, ws, n, st)
        return out.flatten(1)

    @staticmethod
    def norm(x):
        x = x.float()
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).to(torch.bfloat16)

    def prompt(self, x, batch):
        """x fp32 [rows, hidden]; the weights are decoded once for all rows."""
        self.decode_weights()
        wq, wk, wv, wo, wg, wu, wd = self.weights
        h = self.norm(x)
        qkv = torch.cat([h @ w.t() for w in (wq, wk, wv)], 1).reshape(len(x), -1, self.d)
        x = x + (self.attend(qkv, batch) @ wo.t()).float()
        h = self.norm(x)
        return x + ((torch.nn.functional.silu((h @ wg.t()).float()) * (h @ wu.t()).float()).to(torch.bfloat16) @ wd.t()).float()

    def token(self, x, batch):
        """x fp32 [1, hidden]: nothing decoded reaches memory."""
        empty = lambda i: torch.empty(sum(self.shapes[k][0] for k in i), dtype=torch.float32, device="cuda")  # noqa: E731
        qkv = self.gemv([0, 1, 2], self.norm(x).flatten(), empty([0, 1, 2])).reshape(1, -1, self.d)
        x = x + self.gemv([3], self.attend(qkv, batch).flatten(), empty([3]))
        gate, up = self.gemv([4, 5], self.norm(x).flatten(), empty([4, 5])).chunk(2)
        return x + self.gemv([6], (torch.nn.functional.silu(gate) * up).to(torch.bfloat16), empty([6]))


def batch_of(lens, news, tables, prefix_len=0, prefix_pages=None):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    return dc.KVBatch(len(lens), starts[-1], max(news), max(lens), i32(lens), i32(tables), len(tables[0]), row_start_dev=i32(starts),
                      prefix_len=prefix_len, prefix_pages_dev=i32(prefix_pages) if prefix_len else None)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("hidden", 4096), ("heads", 32), ("kv-heads", 32), ("ffn", 11008), ("prompt", 1024), ("tokens", 32), ("window", 0), ("sinks", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--cache", choices=("bf16", "i8"), default="bf16")
    a = ap.parse_args()
    total = a.prompt + a.tokens
    table = [list(range(-(-total // PAGE)))]
    layer = DecoderLayer(a.hidden, a.heads, a.kv_heads, a.ffn, len(table[0]), total, a.window, a.sinks, cache=a.cache)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(total, a.hidden, generator=g, device="cuda")
    for turn in range(2):  # the first turn warms up
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        layer.prompt(x[:a.prompt], batch_of([a.prompt], [a.prompt], table))
        torch.cuda.synchronize()
        t1 = time.perf_counter()
        for t in range(a.prompt, total):
            layer.token(x[t:t + 1], batch_of([t + 1], [1], table))
        torch.cuda.synchronize()
        t2 = time.perf_counter()
    raw = sum(r * c for r, c in layer.shapes)
    print(f"layer of {raw / 1e6:.0f} MB int8, compressed {raw / layer.blob.numel():.3f}: prompt of {a.prompt} tokens {1e3 * (t1 - t0):.2f} ms, "
          f"{1e6 * (t2 - t1) / max(1, a.tokens):.0f} us a token")


if __name__ == "__main__":
    main()
