"""A whole fine-tuning step of a layer on a packed batch, from the residual stream to the loss over the vocabulary and back.

    y1 = norm(x);  h = x + dropout(attention(y1));  y2 = norm(h);  h' = h + dropout(FFN(y2));  loss(norm(h'))

The addition to the residual stream, the dropout and the norm that follows are one call each way; the masks of the dropout are made again
from a seed, a step and a place.  Tokens of prompts and padding have no target: the loss leaves them out of its products.  Only the
norms' weights and the LoRA matrices are trained; their gradients are clipped by the global norm.  Attention, positions, the sparse FFN
and their layer are those of packed_step.py.

    python examples/finetune_step.py [--width 2048 --heads 32 --kv-heads 8 --ffn 8192 --vocabulary 50272 --rows 4 --tokens 1024]

prints the mean loss and the norm of the gradients."""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from packed_step import CAP, Layer, pack, ranges  # noqa: E402
from paper_2510_15964_amd import lx  # noqa: E402

EPS = 1e-5


class Tuned(Layer):
    """The layer of packed_step.py with its norms, dropout and the vocabulary's matrix (frozen)."""

    def __init__(self, d, heads, kv_heads, F, V, max_tokens, p=0.1, dtype=torch.bfloat16, seed=0):
        super().__init__(d, heads, kv_heads, F, max_tokens, dtype, seed)
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.p, self.rng = p, torch.tensor([seed, 0], dtype=torch.int64, device="cuda")      # seed and step of the dropout
        self.norms = [(1 + 0.1 * torch.randn(d, device="cuda", generator=g)).to(dtype) for _ in range(3)]
        self.W_vocab = (torch.randn((V, d), device="cuda", generator=g) * 2 * d ** -0.5).to(dtype)
        self.dnorms = [torch.zeros(d, device="cuda") for _ in range(3)]
        self.grads = lx.GradSet([self.dA, self.dB, *self.dnorms])

    def add_norm(self, i, x, residual=None):
        """(h, y): h = residual + dropout(x), x itself without a residual; y = norm(h)."""
        y = torch.empty_like(x)
        if residual is None:
            lx.lx_rms_norm_fwd(x, self.norms[i], EPS, y)
            return x, y
        h = torch.empty_like(x)
        lx.lx_rms_norm_fwd(x, self.norms[i], EPS, y, residual=residual, H=h, p=self.p, rng=self.rng, site=i)
        return h, y

    def add_norm_back(self, i, dy, h, dh=None, inner=True):
        """The gradients of x (without `inner` there is none) and of the residual."""
        dx, dr = torch.empty_like(h) if inner else None, torch.empty_like(h)
        lx.lx_rms_norm_bwd(dy, h, self.norms[i], EPS, dx, dH=dh, dR=dr, dW=self.dnorms[i], p=self.p if inner else 0.0, rng=self.rng, site=i)
        return dx, dr

    def step(self, x, positions, lo, hi, blocks, targets, weights):
        """(loss per token, gradient of x); the other gradients into dA, dB and dnorms."""
        B, S, d = x.shape
        T = B * S
        x = x.view(T, d)
        _, y1 = self.add_norm(0, x)
        Q, K, V, O, LSE = self.attend(y1.view(B, S, d), positions, lo, hi)
        h, y2 = self.add_norm(1, O.transpose(1, 2).reshape(T, d) @ self.Wo.t(), x)
        f, H, U = torch.empty_like(y2), torch.empty(blocks.nnz_cap * 4096, dtype=x.dtype, device="cuda"), torch.empty((T, 64), dtype=x.dtype, device="cuda")
        lx.lx_sparse_ffn_lora_fwd(y2, self.W_up, self.A, self.B, self.W_down, blocks, f, H, U)
        h2, y3 = self.add_norm(2, f, h)

        loss, dy3 = torch.empty(T, device="cuda"), torch.empty_like(y3)
        lx.lx_vocab_loss(y3, self.W_vocab, targets, loss, weights=weights, dX=dy3)

        df, dh = self.add_norm_back(2, dy3, h2)
        room = torch.empty(lx.lx_sparse_ffn_lora_bwd_workspace_bytes(T, d, self.F, blocks.nnz_cap), dtype=torch.uint8, device="cuda")
        dy2 = torch.empty_like(y2)
        lx.lx_sparse_ffn_lora_bwd(y2, df, H, U, self.W_up_t, self.W_down_t, self.A, self.B, blocks, dy2, self.dA, self.dB, room)
        da, dx = self.add_norm_back(1, dy2, h, dh)
        dO = (da @ self.Wo).view(B, S, self.Hq, self.D).transpose(1, 2)
        dqkv = torch.empty((B, S, (self.Hq + 2 * self.Hkv) * self.D), dtype=x.dtype, device="cuda")
        dQ, dK, dV = self.split(dqkv)
        lx.lx_score_attn_bwd(Q, K, V, O, LSE, dO, self.D ** -0.5, True, dQ, dK, dV, cap=CAP, key_lo=lo, key_hi=hi)
        lx.lx_rope(dQ, dK, self.table, positions, dQ, dK, inverse=True)
        _, dx = self.add_norm_back(0, dqkv.view(T, -1) @ self.Wqkv, x, dx, inner=False)
        self.rng[1:] += 1          # on the device: a captured step draws other masks at every replay
        return loss, dx.view(B, S, d)


def run(width=2048, heads=32, kv_heads=8, ffn=8192, vocabulary=50272, rows=4, tokens=1024, seed=0, p=0.1, max_norm=1.0, active=0.25):
    """The step; a dict of what to look at."""
    g = torch.Generator().manual_seed(seed)
    lengths, total = [], 0
    while total < rows * tokens * 3 // 4:
        lengths.append(int(torch.randint(max(tokens // 16, 2), tokens // 2, (1,), generator=g)))
        total += lengths[-1]
    B, begin, end = pack(lengths, tokens)
    layer = Tuned(width, heads, kv_heads, ffn, vocabulary, tokens + 1, p, seed=seed)
    x = torch.randn((B, tokens, width), generator=g).to("cuda", torch.bfloat16)
    positions, lo, hi = ranges(begin, end, B, tokens)
    targets = torch.full((B * tokens,), -100, dtype=torch.int32)
    for b, e in zip(begin, end):          # the first third of a document is its prompt; its last token foresees nothing
        answer = torch.arange(b + (e - b) // 3, e - 1)
        targets[answer] = torch.randint(0, vocabulary, (len(answer),), generator=g, dtype=torch.int32)
    count = int((targets >= 0).sum())
    targets = targets.cuda()
    weights = torch.full((B * tokens,), 1.0 / max(count, 1), device="cuda")
    mask = (torch.rand((B * tokens // 64, ffn // 64), generator=g) < active).to(torch.uint8).cuda()
    blocks = lx.lx_mask_compact(mask)
    loss, dx = layer.step(x, positions, lo, hi, blocks, targets, weights)
    raw = [t.clone() for t in (layer.dA, layer.dB, *layer.dnorms)]
    norm = layer.clip(max_norm).item()
    return {"layer": layer, "x": x, "positions": positions, "lo": lo, "hi": hi, "targets": targets, "weights": weights, "mask": mask, "loss": loss,
            "dx": dx, "raw": raw, "clipped": [layer.dA, layer.dB, *layer.dnorms], "norm": norm, "max_norm": max_norm, "answers": count}


def main():
    p = argparse.ArgumentParser()
    for name, v in (("width", 2048), ("heads", 32), ("kv-heads", 8), ("ffn", 8192), ("vocabulary", 50272), ("rows", 4), ("tokens", 1024)):
        p.add_argument("--" + name, type=int, default=v)
    r = run(**vars(p.parse_args()))
    print(f"{r['answers']} of {r['loss'].numel()} tokens have a target: mean loss {r['loss'].sum().item() / max(r['answers'], 1):.4f}; norm of the "
          f"gradients {r['norm']:.4g}, clipped to {sum(t.double().square().sum() for t in r['clipped']).sqrt().item():.4g}")


if __name__ == "__main__":
    main()
