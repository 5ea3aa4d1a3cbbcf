"""One attention layer of a served multi-adapter batch, start to end on the library.

A step takes the hidden states of its new tokens (prompt chunks and single decode tokens together):

    base projection (the caller's matmul)  ->  adapters of the fused QKV projection added in place
    block tables and slots of the batch    ->  norm and rotation, keys and values into the 4-bit cache
    attention over the cache               ->  base output projection, its adapters added in place

    python examples/attention_step.py [--requests 32] [--steps 16]

runs a prompt step and a number of decode steps with random weights and prints their times.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_24044_b200 import binding as lb          # noqa: E402
from paper_2602_24044_b200.harness import KVCache         # noqa: E402


class AttentionLayer:
    """QKV and output projections with resident adapters, and a paged cache, on the current device."""

    QKV, OUT = 0, 1

    def __init__(self, d_model=1024, num_q_heads=8, num_kv_heads=2, head_dim=128, adapters=4, rank=8, pages=256,
                 page_size=16, max_positions=4096, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.hq, self.hkv, self.d, self.d_model = num_q_heads, num_kv_heads, head_dim, d_model
        qkv = (num_q_heads + 2 * num_kv_heads) * head_dim
        dev = torch.cuda.current_device()

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device="cuda") * rows ** -0.5).bfloat16()

        self.w_qkv, self.w_out = weight(d_model, qkv), weight(num_q_heads * head_dim, d_model)
        self.q_weight = (1 + 0.2 * torch.randn(head_dim, generator=g, device="cuda")).bfloat16()
        self.k_weight = (1 + 0.2 * torch.randn(head_dim, generator=g, device="cuda")).bfloat16()
        f = 10000.0 ** (-torch.arange(0, head_dim, 2, device="cuda") / head_dim)
        a = torch.arange(max_positions, device="cuda")[:, None] * f
        self.angles = torch.cat([a.cos(), a.sin()], -1).contiguous()
        # adapter slots of both projections
        targets = [(d_model, qkv), (num_q_heads * head_dim, d_model)]
        self.num_slots = adapters
        buf = torch.empty(lb.pool_bytes(adapters, rank, targets, dev) + 256, dtype=torch.uint8, device="cuda")
        off = (-buf.data_ptr()) % 256
        self._pool_buf, mem = buf, buf[off:]
        self.pool = lb.pool_create(adapters, rank, targets, mem, dev)
        host = []
        for s in range(adapters):
            A = [(torch.randn(rank, i) * i ** -0.5).bfloat16().pin_memory() for i, _ in targets]
            B = [(torch.randn(rank, o) * 0.1).bfloat16().pin_memory() for _, o in targets]
            lb.pool_load_slot(self.pool, s, rank, 1.0, A, B, lb.A_RANK_MAJOR)
            host += A + B
        torch.cuda.synchronize()
        # the cache, with every page free
        self.kv = KVCache(1, pages, page_size, num_q_heads, num_kv_heads, head_dim, dev)
        self.free = torch.arange(pages, dtype=torch.int32, device="cuda")
        self.free_count = torch.tensor([pages], dtype=torch.int32, device="cuda")
        self.pages, self.page_size = pages, page_size

    def admit(self, requests, max_tokens):
        """State of a new set of requests: lengths and block table."""
        blocks = -(-max_tokens // self.page_size)
        self.lengths = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.table = torch.full((requests, blocks), -1, dtype=torch.int32, device="cuda")

    def release(self, requests):
        self.kv.release(torch.as_tensor(requests, dtype=torch.int32, device="cuda"), self.lengths, self.table,
                        self.free, self.free_count, stream=torch.cuda.current_stream())

    def _adapt(self, target, x, y, slots, prompt):
        T, n = x.shape[0], self.num_slots
        tile = 128 if prompt else 16
        meta = torch.empty(lb.segments_bytes(T, n, tile), dtype=torch.uint8, device="cuda")
        ws = torch.empty(max(lb.workspace_bytes(self.pool, T), 16), dtype=torch.uint8, device="cuda")
        stream = torch.cuda.current_stream()
        lb.build_segments(self.pool, slots, T, tile, 128, meta, stream=stream)
        if prompt:
            lb.sgmv_apply(self.pool, target, x, x.stride(0), y, y.stride(0), y, y.stride(0), meta, T, ws, stream=stream)
        else:
            lb.bgmv_apply(self.pool, target, x, x.stride(0), y, y.stride(0), y, y.stride(0), slots, T, meta, ws,
                          stream=stream)

    def step(self, x, q_len, adapters):
        """x: bf16 [T, d_model], the new tokens of all requests in order; q_len: tokens of each request (host
        list); adapters: int32 [T] adapter slot of each token.  Returns (layer output, attention output, the
        fused projection's rows)."""
        T, stream = x.shape[0], torch.cuda.current_stream()
        qkv = x @ self.w_qkv
        self._adapt(self.QKV, x, qkv, adapters, max(q_len) > 1)
        kv, hq, hkv, d = self.kv, self.hq, self.hkv, self.d
        kv.build_tables(self.lengths, torch.tensor(q_len, dtype=torch.int32, device="cuda"), T, self.free,
                        self.free_count, self.table, max_q=max(q_len), stream=stream)
        q = torch.empty((T, hq * d), dtype=torch.bfloat16, device="cuda")
        args = lb.qk_args(num_q_heads=hq, num_kv_heads=hkv, head_dim=d, q=qkv, ldq=qkv.stride(0), k=qkv[:, hq * d:],
                          ldk=qkv.stride(0), v=qkv[:, (hq + hkv) * d:], ldv=qkv.stride(0), q_weight=self.q_weight,
                          k_weight=self.k_weight, eps=1e-6, cos_sin=self.angles, positions=kv.positions, q_out=q,
                          device=x.device.index)
        kv.append(0, args, stream=stream)
        attn = torch.empty_like(q)
        kv.attention(0, q, attn, scale=d ** -0.5, stream=stream)
        out = attn @ self.w_out
        self._adapt(self.OUT, attn, out, adapters, max(q_len) > 1)
        return out, attn, qkv

    def close(self):
        if self.pool:
            torch.cuda.synchronize()
            self.kv.close()
            lb.pool_destroy(self.pool)
            self.pool = 0


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=32)
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args()
    rng = np.random.default_rng(0)
    lens = [int(n) for n in np.clip(np.exp(rng.normal(np.log(512), 1, a.requests)), 32, 2048)]
    tokens = sum(lens) + a.requests * a.steps
    layer = AttentionLayer(d_model=4096, num_q_heads=32, num_kv_heads=8, adapters=16, rank=16,
                           pages=tokens // 16 + a.requests + 1)
    layer.admit(a.requests, max(lens) + a.steps)
    mine = torch.from_numpy(rng.integers(0, 16, a.requests).astype(np.int32)).cuda()

    def timed(x, q_len, adapters):
        e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        e[0].record()
        layer.step(x, q_len, adapters)
        e[1].record()
        torch.cuda.synchronize()
        return e[0].elapsed_time(e[1])

    x = torch.randn(sum(lens), 4096, device="cuda").bfloat16()
    ms = timed(x, lens, torch.repeat_interleave(mine, torch.tensor(lens, device="cuda")))
    print("%d prompts, %d tokens: %.2f ms (first use of the kernels included)" % (a.requests, sum(lens), ms))
    times = [timed(torch.randn(a.requests, 4096, device="cuda").bfloat16(), [1] * a.requests, mine)
             for _ in range(a.steps)]
    print("decode step of %d requests: %.3f ms (median of %d)" % (a.requests, sorted(times)[len(times) // 2], a.steps))
    layer.release(list(range(a.requests)))
    print("pages free again: %d of %d; status %s" % (int(layer.free_count), layer.pages, layer.kv.status()))
    layer.close()


if __name__ == "__main__":
    main()
