"""One attention layer of a served multi-adapter batch, and a whole step around it, start to end on the library.

A step takes the hidden states of its new tokens (prompt chunks and single decode tokens together):

    base projection (the caller's matmul)  ->  adapters of the fused QKV projection added in place
    block tables and slots of the batch    ->  norm and rotation, keys and values into the 4-bit cache
    attention over the cache               ->  base output projection, its adapters added in place

ServedStep goes from token ids to the next token ids, with that layer in the middle:

    rows of the embedding                  ->  norm  ->  the attention layer (positions of images on three axes)
    residual addition and norm             ->  logits of each request's last token  ->  the next tokens

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
from paper_2602_24044_b200.harness import KVCache, media_spans  # noqa: E402


class AttentionLayer:
    """QKV and output projections with resident adapters, and a paged cache, on the current device."""

    QKV, OUT = 0, 1

    def __init__(self, d_model=1024, num_q_heads=8, num_kv_heads=2, head_dim=128, adapters=4, rank=8, pages=256,
                 page_size=16, max_positions=4096, seed=0, axis_of_pair=None):
        """axis_of_pair: which of time, height and width turns each rotation pair (requests may then have media)."""
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
        self.axis_of_pair, self.spans = axis_of_pair, None

    def admit(self, requests, max_tokens, media=None):
        """State of a new set of requests: lengths, block table, and (media: for each request what media_spans
        takes) where their images and videos are."""
        if self.axis_of_pair is not None:
            spans, begin = media_spans(media or [[]] * requests)
            self.spans, self.span_begin = torch.from_numpy(spans).cuda(), torch.from_numpy(begin).cuda()
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
        positions = kv.positions
        if self.axis_of_pair is not None:
            positions = torch.empty((3, T), dtype=torch.int32, device="cuda")
            kv.axis_positions(self.spans, self.span_begin, positions, stream=stream)
        args = lb.qk_args(num_q_heads=hq, num_kv_heads=hkv, head_dim=d, q=qkv, ldq=qkv.stride(0), k=qkv[:, hq * d:],
                          ldk=qkv.stride(0), v=qkv[:, (hq + hkv) * d:], ldv=qkv.stride(0), q_weight=self.q_weight,
                          k_weight=self.k_weight, eps=1e-6, cos_sin=self.angles, positions=positions,
                          axis_of_pair=self.axis_of_pair, q_out=q, device=x.device.index)
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


class ServedStep:
    """Token ids to next token ids: embedding, norm, the attention layer, residual and norm, logits, sampling."""

    def __init__(self, vocab=8000, eps=1e-6, seed=0, **layer):
        self.layer = AttentionLayer(seed=seed, **layer)
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        n = self.layer.d_model
        self.eps = eps
        self.embedding = torch.randn(vocab, n, generator=g, device="cuda").bfloat16()
        self.w_head = (torch.randn(n, vocab, generator=g, device="cuda") * 2.5 * n ** -0.5).bfloat16()
        self.norms = [(1 + 0.2 * torch.randn(n, generator=g, device="cuda")).bfloat16() for _ in range(2)]

    def _norm(self, x, weight, residual=None):
        """(the stream after adding x to it, its norm)"""
        out = torch.empty_like(x)
        lb.add_norm(lb.norm_args(x=x, weight=weight, eps=self.eps, residual=residual, residual_out=residual, out=out,
                                 device=x.device.index), x.shape[0], stream=torch.cuda.current_stream())
        return (x if residual is None else residual), out

    def step(self, ids, q_len, adapters, uniform, temperature, top_k=None, top_p=None, min_p=None):
        """ids: the new tokens of all requests in order; q_len: how many each has (one at least); the sampling
        parameters: one a request, on the device.  Returns (next tokens, their logprobs, the logits)."""
        stream, h = self._norm(self.embedding[ids.long()], self.norms[0])
        out, _, _ = self.layer.step(h, q_len, adapters)
        stream, h = self._norm(out, self.norms[1], residual=stream)
        last = torch.cumsum(torch.tensor(q_len, device="cuda"), 0) - 1
        logits = h[last] @ self.w_head
        R = len(q_len)
        token = torch.empty(R, dtype=torch.int32, device="cuda")
        logprob = torch.empty(R, dtype=torch.float32, device="cuda")
        lb.sample(lb.sample_args(logits=logits, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p,
                                 uniform=uniform, token=token, logprob=logprob, device=logits.device.index), R,
                  stream=torch.cuda.current_stream())
        return token, logprob, logits

    def close(self):
        self.layer.close()


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
