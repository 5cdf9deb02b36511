"""A small decoder whose linear layers are DBF layers, run as a server runs one: requests of different lengths in one batch, their keys and values in pages of 4 bits,
prompts and single tokens by the same calls, texts judged by the log probabilities of their tokens.

    python examples/serve_decoder.py

Per pass: dbf_block_tables (where the new tokens go); per block dbf_gemv / dbf_gemm (query, key, value), dbf_cache_append (norm, rotation, 4 bits, the write),
dbf_cache_attend, the other layers; then dbf_token_logprobs.  Embedding, residual sums, the norms of whole activations and the gate are torch's.
Weights are random; the sizes are those of a toy."""
import math
import os
import sys
from dataclasses import dataclass

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2505_11076_amd import binding as B  # noqa: E402
from paper_2505_11076_amd import inputs as I  # noqa: E402


@dataclass
class Config:
    vocab: int = 1000
    hidden: int = 256
    q_heads: int = 8
    kv_heads: int = 2
    head_dim: int = 64
    mlp: int = 640
    blocks: int = 2
    bits: float = 2.0       # of a weight
    page: int = 32          # tokens of a page
    pages: int = 64
    max_len: int = 512      # tokens of a request
    eps: float = 1e-6


def make_layer(n_in, n_out, bits, seed):
    """A random DBF layer, its vectors such that an input of unit size gives an output of unit size."""
    k = int(bits * n_in * n_out / (n_in + n_out))
    rng = np.random.default_rng(seed)
    scale = (n_in * k) ** (-1 / 6)
    vectors = [(scale * rng.uniform(0.5, 1.5, n)).astype(np.float16).view(np.uint16) for n in (n_out, k, n_in)]
    return I.LayerInputs(n_in, n_out, k, I.random_sign_words(rng, n_out, k), I.random_sign_words(rng, k, n_in), *vectors)


class Decoder:
    def __init__(self, cfg: Config, seed: int = 0):
        self.cfg = cfg
        c, rng = cfg, np.random.default_rng(seed)
        sizes = dict(q=(c.hidden, c.q_heads * c.head_dim), k=(c.hidden, c.kv_heads * c.head_dim), v=(c.hidden, c.kv_heads * c.head_dim), o=(c.q_heads * c.head_dim, c.hidden),
                     gate=(c.hidden, c.mlp), up=(c.hidden, c.mlp), down=(c.mlp, c.hidden))
        self.inputs = [{name: make_layer(*s, c.bits, 1000 * seed + 10 * b + i) for i, (name, s) in enumerate(sizes.items())} for b in range(c.blocks)]
        self.head_inputs = make_layer(c.hidden, c.vocab, c.bits, 1000 * seed + 999)
        pack = lambda L: B.dbf_pack_bits(L.n_in, L.n_out, L.k, L.A_bits, L.B_bits, L.a, L.m, L.b)  # noqa: E731
        self.layers = [{name: pack(L) for name, L in block.items()} for block in self.inputs]
        self.head = pack(self.head_inputs)
        half = lambda x: torch.from_numpy(np.asarray(x, np.float16)).cuda()  # noqa: E731
        self.embedding = half(rng.normal(size=(c.vocab, c.hidden)))
        self.norms = [{name: half(rng.uniform(0.8, 1.2, n)) for name, n in (("in", c.hidden), ("mlp", c.hidden), ("q", c.head_dim), ("k", c.head_dim))} for _ in range(c.blocks)]
        self.last_norm = half(rng.uniform(0.8, 1.2, c.hidden))
        angle = np.arange(c.max_len)[:, None] * np.exp(-np.arange(0, c.head_dim, 2) * math.log(10000.0) / c.head_dim)
        self.rope = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)).cuda()
        # the caches of the blocks have one table: a page is the same place in each
        self.memory = [torch.zeros(B.dbf_cache_bytes(c.pages, c.page, c.kv_heads, c.head_dim), dtype=torch.uint8, device="cuda") for _ in range(c.blocks)]
        self.caches = [B.Cache(data=m.data_ptr(), n_pages=c.pages, page_tokens=c.page, n_kv_heads=c.kv_heads, head_dim=c.head_dim) for m in self.memory]
        self.free = list(range(c.pages))

    def start(self, requests: int):
        """Requests that hold nothing yet."""
        c = self.cfg
        self.lengths = [0] * requests
        self.table = torch.full((requests, -(-c.max_len // c.page)), -1, dtype=torch.int32, device="cuda")

    def linear(self, layer, x):
        y = torch.empty(x.shape[0], layer.n_out, dtype=torch.float16, device="cuda")
        stream = torch.cuda.current_stream().cuda_stream
        if x.shape[0] <= B.MAX_BATCH:
            B.dbf_gemv(layer, x.data_ptr(), y.data_ptr(), x.shape[0], stream)
        else:
            ws = torch.empty(B.dbf_gemm_workspace_bytes(layer, x.shape[0]), dtype=torch.uint8, device="cuda")
            B.dbf_gemm(layer, x.data_ptr(), y.data_ptr(), x.shape[0], ws.data_ptr(), ws.numel(), stream)
        return y

    def norm(self, x, weight):
        x = x.float()
        return (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + self.cfg.eps) * weight.float()).half()

    def forward(self, new, targets, top=0):
        """One pass over the new tokens of each request (lists, possibly empty) that go behind those it holds: log probabilities of `targets`
        (as the tokens, -1: none), entropies and the `top` likeliest tokens of every new token's place, and the logits."""
        c, stream = self.cfg, torch.cuda.current_stream().cuda_stream
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        T, n = sum(map(len, new)), len(new)
        if not T:
            raise ValueError("no request has a new token")
        empty = lambda *shape, dtype=torch.int32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
        start, kv, pos, slots, status = empty(n + 1), empty(n), empty(T), empty(T), empty(2)
        cached, added, free = ints(self.lengths), ints([len(t) for t in new]), ints(self.free)
        B.dbf_block_tables(cached.data_ptr(), added.data_ptr(), n, c.page, free.data_ptr(), len(self.free), self.table.data_ptr(), self.table.shape[1], T, start.data_ptr(),
                           kv.data_ptr(), pos.data_ptr(), slots.data_ptr(), status.data_ptr(), stream)
        # (what the device takes of the free pages follows from the lengths: no need to ask it)
        after = [a + len(t) for a, t in zip(self.lengths, new)]
        taken = sum(-(-b // c.page) - -(-a // c.page) for a, b in zip(self.lengths, after))
        if taken > len(self.free) or max(after) > c.max_len:
            raise RuntimeError("the cache is full")
        self.free = self.free[taken:]
        self.lengths = after

        x = self.embedding[ints(sum(new, [])).long()]
        D, hq, hk = c.head_dim, c.q_heads, c.kv_heads
        for layer, norm, cache in zip(self.layers, self.norms, self.caches):
            h = self.norm(x, norm["in"])
            q, k, v = (self.linear(layer[name], h) for name in "qkv")
            heads = B.Heads(q=q.data_ptr(), q_stride=hq * D, k=k.data_ptr(), k_stride=hk * D, v=v.data_ptr(), v_stride=hk * D, q_out=q.data_ptr(), q_out_stride=hq * D,
                            q_weight=norm["q"].data_ptr(), k_weight=norm["k"].data_ptr(), eps=c.eps, rope=self.rope.data_ptr(), rope_len=c.max_len, rot_dim=D,
                            positions=pos.data_ptr(), dtype=B.F16, n_tokens=T, n_q_heads=hq, n_kv_heads=hk, head_dim=D)
            B.dbf_cache_append(heads, cache, slots.data_ptr(), stream)
            out = torch.empty_like(q)
            attend = B.Attend(q=q.data_ptr(), q_stride=hq * D, out=out.data_ptr(), out_stride=hq * D, q_start=start.data_ptr(), kv_len=kv.data_ptr(),
                              block_table=self.table.data_ptr(), table_stride=self.table.shape[1], dtype=B.F16, n_tokens=T, n_seq=n, n_q_heads=hq, max_q=max(map(len, new)),
                              max_kv=max(after), causal=1, scale=1 / math.sqrt(D))
            ws = torch.empty(max(256, B.dbf_cache_attend_workspace_bytes(attend, cache)), dtype=torch.uint8, device="cuda")
            B.dbf_cache_attend(attend, cache, ws.data_ptr(), ws.numel(), stream)
            x = x + self.linear(layer["o"], out)
            h = self.norm(x, norm["mlp"])
            x = x + self.linear(layer["down"], torch.nn.functional.silu(self.linear(layer["gate"], h)) * self.linear(layer["up"], h))
        logits = self.linear(self.head, self.norm(x, self.last_norm))
        lp, entropy, ids, tops = empty(T, dtype=torch.float32), empty(T, dtype=torch.float32), empty(T, top), empty(T, top, dtype=torch.float32)
        wanted = ints(sum(targets, []))
        ws = torch.empty(max(256, B.dbf_token_logprobs_workspace_bytes(T, c.vocab, top)), dtype=torch.uint8, device="cuda")
        B.dbf_token_logprobs(logits.data_ptr(), B.F16, c.vocab, T, c.vocab, wanted.data_ptr(), top, lp.data_ptr(), entropy.data_ptr(), ids.data_ptr() if top else 0,
                             tops.data_ptr() if top else 0, ws.data_ptr(), ws.numel(), stream)
        return lp, entropy, ids, tops, logits

    def close(self):
        for layer in [l for block in self.layers for l in block.values()] + [self.head]:
            layer.close()


def main():
    cfg = Config()
    decoder, rng = Decoder(cfg), np.random.default_rng(1)
    texts = [[int(t) for t in rng.integers(0, cfg.vocab, n)] for n in (70, 3, 200)]
    # the texts, judged: a token's log probability is that of the place before it
    decoder.start(len(texts))
    lp, entropy, _, _, _ = decoder.forward(texts, [t[1:] + [-1] for t in texts])
    torch.cuda.synchronize()
    for text, part in zip(texts, lp.split([len(t) for t in texts])):
        print("text of %d tokens: perplexity %.1f (of %d equal tokens: %d)" % (len(text), math.exp(-float(part[:-1].mean())), cfg.vocab, cfg.vocab))
    # and continued, the likeliest token at a time
    last = [t[-1] for t in texts]
    decoder.start(len(texts))
    decoder.free = list(range(cfg.pages))
    _, _, ids, _, _ = decoder.forward(texts, [[-1] * len(t) for t in texts], top=1)
    last = [int(ids[sum(map(len, texts[: i + 1])) - 1, 0]) for i in range(len(texts))]
    for _ in range(5):
        _, entropy, ids, tops, _ = decoder.forward([[t] for t in last], [[-1]] * len(last), top=3)
        print("after", last, "likeliest", ids.cpu().tolist(), "entropy", [round(float(e), 2) for e in entropy])
        last = [int(i) for i in ids[:, 0]]
    decoder.close()


if __name__ == "__main__":
    main()
