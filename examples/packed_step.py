"""One fine-tuning step of a layer on a packed batch, and the next token over its cache.

Documents of different lengths lie end to end in rows of one length.  Forward: frozen projections, rotary positions that start
anew with every document, attention inside the documents (capped scores), the sparse FFN with its LoRA branch.  Backward: the
same calls in reverse, and the gradients of the LoRA matrices clipped by their global norm.  Then the first document is continued
by a token: its keys lie in a cache, and the query attends all of them.

    python examples/packed_step.py [--width 2048 --heads 32 --kv-heads 8 --ffn 8192 --rows 4 --tokens 1024]

prints the norm of the gradients and how far a document in the pack is from the same document alone."""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2510_15964_amd import lx  # noqa: E402

CAP = 15.0


def pack(lengths, S):
    """Documents of these lengths in rows of S tokens, each in the first row with room for it: (rows, begin, end), indices into
    all tokens."""
    room, at = [], []
    for n in lengths:
        assert 0 < n <= S
        r = next((i for i, x in enumerate(room) if x >= n), len(room))
        if r == len(room):
            room.append(S)
        at.append(r * S + S - room[r])
        room[r] -= n
    return len(room), at, [a + n for a, n in zip(at, lengths)]


class Layer:
    """Frozen weights, the LoRA matrices (rank 16 of 64) and what a step's calls need: made once."""

    def __init__(self, d, heads, kv_heads, F, max_tokens, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(*shape, std):
            return (torch.randn(shape, device="cuda", generator=g) * std).to(dtype)
        self.d, self.Hq, self.Hkv, self.D, self.F = d, heads, kv_heads, d // heads, F
        kv = kv_heads * self.D
        self.Wqkv, self.Wo = w(d + 2 * kv, d, std=d ** -0.5), w(d, d, std=d ** -0.5)
        self.W_up, self.W_down = w(F, d, std=d ** -0.5), w(d, F, std=F ** -0.5)
        self.W_up_t, self.W_down_t = lx.lx_ffn_pack_weights(self.W_up, self.W_down)
        self.A, self.B = torch.zeros((64, d), dtype=dtype, device="cuda"), torch.zeros((F, 64), dtype=dtype, device="cuda")
        self.A[:16], self.B[:, :16] = w(16, d, std=d ** -0.5), w(F, 16, std=0.02)
        self.table = lx.lx_rope_table(self.D, max_tokens)
        self.dA, self.dB = torch.zeros((64, d), device="cuda"), torch.zeros((F, 64), device="cuda")
        self.grads, self.norm = lx.GradSet([self.dA, self.dB]), torch.zeros(1, device="cuda")

    def split(self, qkv):
        """[B,S,(Hq + 2 Hkv) D] as Q, K, V [B,heads,S,D]: views, the tokens' heads side by side."""
        B, S, _ = qkv.shape
        t = qkv.view(B, S, self.Hq + 2 * self.Hkv, self.D).transpose(1, 2)
        return t[:, :self.Hq], t[:, self.Hq:self.Hq + self.Hkv], t[:, self.Hq + self.Hkv:]

    def attend(self, x, positions, lo, hi):
        """(Q, K, V, O, LSE): Q and K turned in place; O [B,S,Hq,D] in memory."""
        B, S, _ = x.shape
        Q, K, V = self.split((x.view(B * S, -1) @ self.Wqkv.t()).view(B, S, -1))
        lx.lx_rope(Q, K, self.table, positions, Q, K)
        O = torch.empty((B, S, self.Hq, self.D), dtype=x.dtype, device="cuda").transpose(1, 2)
        LSE = torch.empty((B, self.Hq, S), device="cuda")
        lx.lx_score_attn_fwd(Q, K, V, self.D ** -0.5, True, O, LSE, cap=CAP, key_lo=lo, key_hi=hi)
        return Q, K, V, O, LSE

    def forward(self, x, positions, lo, hi, blocks):
        B, S, d = x.shape
        kept = self.attend(x, positions, lo, hi)
        y = (x.view(B * S, d) + kept[3].transpose(1, 2).reshape(B * S, d) @ self.Wo.t())
        out, H, U = torch.empty_like(y), torch.empty(blocks.nnz_cap * 4096, dtype=x.dtype, device="cuda"), torch.empty((B * S, 64), dtype=x.dtype, device="cuda")
        lx.lx_sparse_ffn_lora_fwd(y, self.W_up, self.A, self.B, self.W_down, blocks, out, H, U)
        return (out + y).view(B, S, d), (*kept, y, H, U)

    def backward(self, dout, kept, positions, lo, hi, blocks):
        """dx; dA and dB into self.dA, self.dB."""
        Q, K, V, O, LSE, y, H, U = kept
        B, S, d = dout.shape
        dout = dout.view(B * S, d)
        room = torch.empty(lx.lx_sparse_ffn_lora_bwd_workspace_bytes(B * S, d, self.F, blocks.nnz_cap), dtype=torch.uint8, device="cuda")
        dy = torch.empty_like(y)
        lx.lx_sparse_ffn_lora_bwd(y, dout, H, U, self.W_up_t, self.W_down_t, self.A, self.B, blocks, dy, self.dA, self.dB, room)
        dy += dout
        dO = (dy @ self.Wo).view(B, S, self.Hq, self.D).transpose(1, 2)
        dqkv = torch.empty((B, S, (self.Hq + 2 * self.Hkv) * self.D), dtype=dout.dtype, device="cuda")
        dQ, dK, dV = self.split(dqkv)
        lx.lx_score_attn_bwd(Q, K, V, O, LSE, dO, self.D ** -0.5, True, dQ, dK, dV, cap=CAP, key_lo=lo, key_hi=hi)
        lx.lx_rope(dQ, dK, self.table, positions, dQ, dK, inverse=True)
        return (dqkv.view(B * S, -1) @ self.Wqkv + dy).view(B, S, d)

    def clip(self, max_norm):
        return lx.lx_grad_norm_clip(self.grads, max_norm, self.norm)

    def next_token(self, x, cache_k, cache_v, length):
        """Attention's result [B,Hq,1,D] of one token (x [B,1,d]) per sequence: its key and value enter the cache
        [B,Hkv,C,D] at `length` (int32 [B]), and it attends that many and itself."""
        Q, K, V = self.split((x.view(x.shape[0], -1) @ self.Wqkv.t()).view(x.shape[0], 1, -1))
        lx.lx_rope(Q, K, self.table, length.view(-1, 1), Q, K)
        at = length.long().view(-1, 1, 1, 1).expand(-1, self.Hkv, 1, self.D)
        cache_k.scatter_(2, at, K)
        cache_v.scatter_(2, at, V)
        O = torch.empty((x.shape[0], 1, self.Hq, self.D), dtype=x.dtype, device="cuda").transpose(1, 2)
        LSE = torch.empty((x.shape[0], self.Hq, 1), device="cuda")
        lx.lx_score_attn_fwd(Q, cache_k, cache_v, self.D ** -0.5, True, O, LSE, cap=CAP, q_start=length)
        return O


def ranges(begin, end, rows, S):
    """Positions inside the documents, and the key interval of every token."""
    b, e = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (begin, end))
    lo, hi = (torch.empty((rows, S), dtype=torch.int32, device="cuda") for _ in range(2))
    lx.lx_attn_key_ranges(b, e, None, True, lo, hi)
    s = torch.arange(S, dtype=torch.int32, device="cuda").expand(rows, S)
    return torch.where(hi > lo, s - lo, 0).to(torch.int32), lo, hi


def run(width=2048, heads=32, kv_heads=8, ffn=8192, rows=4, tokens=1024, seed=0, max_norm=1.0):
    """The step and the token; a dict of what to look at."""
    g = torch.Generator().manual_seed(seed)
    lengths, total = [], 0
    while total < rows * tokens * 3 // 4:
        lengths.append(int(torch.randint(max(tokens // 16, 2), tokens // 2, (1,), generator=g)))
        total += lengths[-1]
    B, begin, end = pack(lengths, tokens)
    layer = Layer(width, heads, kv_heads, ffn, tokens + 1, seed=seed)
    x = torch.randn((B, tokens, width), generator=g).to("cuda", torch.bfloat16)
    dout = torch.randn((B, tokens, width), generator=g).to("cuda", torch.bfloat16)
    positions, lo, hi = ranges(begin, end, B, tokens)
    dout.masked_fill_((hi == lo)[..., None], 0)          # padding has no loss
    mask = (torch.rand((B * tokens // 64, ffn // 64), generator=g) < 0.25).to(torch.uint8).cuda()
    blocks = lx.lx_mask_compact(mask)
    out, kept = layer.forward(x, positions, lo, hi, blocks)
    dx = layer.backward(dout, kept, positions, lo, hi, blocks)
    raw = [t.clone() for t in (layer.dA, layer.dB)]
    norm = layer.clip(max_norm).item()

    # the first document by itself, and its last token as one that is decoded
    n = end[0] - begin[0]
    alone = layer.attend(x[:1, :n].contiguous(), None, None, None)
    C = tokens
    cache_k, cache_v = (torch.zeros((1, kv_heads, C, layer.D), dtype=x.dtype, device="cuda") for _ in range(2))
    cache_k[:, :, :n - 1], cache_v[:, :, :n - 1] = alone[1][:, :, :n - 1], alone[2][:, :, :n - 1]
    token = layer.next_token(x[:1, n - 1:n].contiguous(), cache_k, cache_v, torch.tensor([n - 1], dtype=torch.int32, device="cuda"))
    return {"out": out, "dx": dx, "raw": raw, "clipped": [layer.dA, layer.dB], "norm": norm, "max_norm": max_norm, "padding": hi == lo,
            "documents": len(lengths), "rows": B, "tokens": total, "packed": kept[3][:1, :, :n], "alone": alone[3], "token": token}


def main():
    p = argparse.ArgumentParser()
    for name, v in (("width", 2048), ("heads", 32), ("kv-heads", 8), ("ffn", 8192), ("rows", 4), ("tokens", 1024)):
        p.add_argument("--" + name, type=int, default=v)
    r = run(**vars(p.parse_args()))

    def far(a, b):
        return ((a.float() - b.float()).norm() / b.float().norm()).item()
    print(f"{r['documents']} documents, {r['tokens']} tokens in {r['rows']} rows; norm of the LoRA gradients {r['norm']:.4g}, "
          f"clipped to {sum(t.double().square().sum() for t in r['clipped']).sqrt().item():.4g}")
    print(f"attention of the first document, in the pack against alone {far(r['packed'], r['alone']):.1e}; its last token over the "
          f"cache {far(r['token'], r['alone'][:, :, -1:]):.1e}")


if __name__ == "__main__":
    main()
