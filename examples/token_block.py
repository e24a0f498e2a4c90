"""An attention block over a convolution's feature map, trained and then served.

    python3 examples/token_block.py

A 3 x 3 convolution (``multi``) turns a small image into a feature map; its
pixels, read row by row behind one class token, are the tokens of a block:

    norm -> projection -> rotate(q, k) -> attend -> projection
         -> norm, gate, residual sum, norm (join) -> classifier

``train`` runs a few steps of gradient descent through the operators' own
gradients; ``serve`` feeds the same tokens one at a time over a cache of keys
and values, the way a decoder does, and gives the same outputs; ``serve_in_pages``
keeps them in pages, the first tokens as one chunk.  The matrix products are torch's.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2212_00404_amd as dc  # noqa: E402


class Attend(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, how):
        out, lse = dc.attend(q, k, v, return_lse=True, **how)
        ctx.save_for_backward(q, k, v, out, lse)
        ctx.how = how
        return out

    @staticmethod
    def backward(ctx, dout):
        return (*dc.attend_backward(dout.contiguous(), *ctx.saved_tensors, **ctx.how), None)


class Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, freq, axis):
        ctx.save_for_backward(positions, freq, axis)
        return dc.rotate(x, positions, freq, axis)

    @staticmethod
    def backward(ctx, dy):
        return dc.rotate(dy.contiguous(), *ctx.saved_tensors, inverse=True), None, None, None


class Join(torch.autograd.Function):
    """(h, y), or y alone without a branch."""
    VECTORS = ("post_weight", "gate", "pre_weight", "pre_bias")

    @staticmethod
    def forward(ctx, branch, x, post_weight, gate, pre_weight, pre_bias, how):
        vectors = dict(zip(Join.VECTORS, (post_weight, gate, pre_weight, pre_bias)))
        h, y, stats = dc.join(branch, x, return_stats=True, **vectors, **how)
        ctx.save_for_backward(branch, x, post_weight, gate, pre_weight, pre_bias, stats)
        ctx.how = how
        return y if branch is None else (h, y)

    @staticmethod
    def backward(ctx, *grads):
        branch, x, *vectors, stats = ctx.saved_tensors
        dh, dy = grads if branch is not None else (None, grads[0])
        g = dc.join_backward(None if dh is None else dh.contiguous(), dy.contiguous(), branch, x, stats,
                             **dict(zip(Join.VECTORS, vectors)), **ctx.how)
        return tuple(g.get(n) for n in ("branch", "x") + Join.VECTORS) + (None,)


class TokenBlock:
    """One block over the tokens of a map of ``channels`` x ``rows`` x ``cols``: Hq
    query heads share Hkv key heads; a token sees ``left`` tokens before it and
    the class token."""

    def __init__(self, channels=64, rows=14, cols=14, Hq=4, Hkv=2, head=32, left=40, classes=10,
                 dtype=torch.bfloat16, device="cuda", seed=0):
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, std=1.0, mean=0.0):
            w = (torch.randn(shape, generator=g) * std + mean).to(device=device, dtype=dtype)
            return w.requires_grad_()

        self.C, self.Hq, self.Hkv, self.head, self.dtype = channels, Hq, Hkv, head, dtype
        self.see = dict(left=left, right=0, sinks=1)
        self.stem = torch.randn((channels, 3, 3, 3), generator=g).div(27 ** 0.5).to(device)
        self.cls = normal(1, 1, channels)
        self.qkv = normal(channels, (Hq + 2 * Hkv) * head, std=channels ** -0.5)
        self.proj = normal(Hq * head, channels, std=(Hq * head) ** -0.5)
        self.norm_in = normal(channels, std=0.02, mean=1.0)
        self.post, self.gate = normal(channels, std=0.02, mean=1.0), normal(channels, std=0.02, mean=0.5)
        self.pre, self.bias = normal(channels, std=0.02, mean=1.0), normal(channels, std=0.02)
        self.out = normal(channels, classes, std=channels ** -0.5)
        self.parameters = [self.cls, self.qkv, self.proj, self.norm_in, self.post, self.gate, self.pre,
                           self.bias, self.out]
        # the class token stands at (0, 0), the map's tokens after it
        at = dc.map_positions(1, rows, cols, device=device)[1:] + 1
        self.positions = torch.cat([torch.zeros_like(at[:, :1]), at], 1)
        self.freq, self.axis = dc.rotary_table((head // 4, head // 4), device=device)

    def tokens(self, images):
        """fp32 images [B, 3, rows + 2, cols + 2] -> tokens [B, 1 + rows * cols, C]."""
        maps = [dc.multi(im, self.stem).flatten(1).t() for im in images]
        x = torch.stack(maps).to(self.dtype)
        return torch.cat([self.cls.expand(x.shape[0], -1, -1), x], 1)

    def project(self, x, positions):
        y = Join.apply(None, x, None, None, self.norm_in, None, dict(norm="rms"))
        qkv = (y @ self.qkv).unflatten(-1, (-1, self.head))
        qk = Rotate.apply(qkv[:, :, :self.Hq + self.Hkv], positions, self.freq, self.axis)
        return qk[:, :, :self.Hq], qk[:, :, self.Hq:], qkv[:, :, self.Hq + self.Hkv:]

    def finish(self, attended, x):
        branch = attended.flatten(2) @ self.proj
        _, y = Join.apply(branch, x, self.post, self.gate, self.pre, self.bias,
                          dict(norm="rms", post=True, branch_scale=1.0))
        return y

    def __call__(self, x):
        q, k, v = self.project(x, self.positions)
        return self.finish(Attend.apply(q, k, v, self.see), x)

    def train(self, images, labels, steps=8, rate=0.2):
        """Losses of some steps of gradient descent on the last token's logits."""
        losses = []
        for _ in range(steps):
            # (causal: the last token is the one that has seen the others)
            logits = self(self.tokens(images))[:, -1].float() @ self.out.float()
            loss = torch.nn.functional.cross_entropy(logits, labels)
            grads = torch.autograd.grad(loss, self.parameters)
            with torch.no_grad():
                for p, g in zip(self.parameters, grads):
                    p -= rate * g
            losses.append(loss.item())
        return losses

    @torch.no_grad()
    def serve(self, x):
        """The same outputs, one token at a time over a cache."""
        B, T, _ = x.shape
        cache_k = torch.empty((B, T, self.Hkv, self.head), dtype=x.dtype, device=x.device)
        cache_v = torch.empty_like(cache_k)
        out = []
        for t in range(T):
            now = x[:, t:t + 1]
            q, k, v = self.project(now, self.positions[:, t:t + 1])
            cache_k[:, t:t + 1], cache_v[:, t:t + 1] = k, v
            lengths = torch.full((B,), t + 1, dtype=torch.int32, device=x.device)
            out.append(self.finish(dc.attend(q, cache_k, cache_v, lengths=lengths, **self.see), now))
        return torch.cat(out, 1)

    @torch.no_grad()
    def serve_in_pages(self, x, prompt=100, kind=None, page=16):
        """The same over a cache in pages (of ``kind``, else of the block's type): the
        first ``prompt`` tokens (all, if there are fewer) in a chunk, then one at a time."""
        B, T, _ = x.shape
        prompt = min(max(prompt, 0), T)
        each = -(-T // page)
        cache = dc.Cache.new(B * each, page, self.Hkv, self.head, kind or x.dtype, device=x.device)
        table = torch.arange(B * each, dtype=torch.int32, device=x.device).view(B, each)
        out = []
        for t0, t1 in [(0, prompt)] + [(t, t + 1) for t in range(prompt, T)]:
            now = x[:, t0:t1]
            q, k, v = (y.flatten(0, 1) for y in self.project(now, self.positions[:, t0:t1]))
            lengths = torch.full((B,), t1, dtype=torch.int32, device=x.device)
            dc.cache_write(cache, k, v, table, lengths)
            attended = dc.attend_cache(q, cache, table, lengths, **self.see)
            out.append(self.finish(attended.unflatten(0, (B, -1)), now))
        return torch.cat(out, 1)


def main():
    block = TokenBlock()
    g = torch.Generator().manual_seed(1)
    images = torch.rand((4, 3, 16, 16), generator=g).cuda()
    labels = torch.arange(4).cuda()
    losses = block.train(images, labels)
    print("loss %s" % " ".join("%.3f" % x for x in losses))
    with torch.no_grad():
        x = block.tokens(images)
        whole, served = block(x), block.serve(x)
    off = (whole.float() - served.float()).abs().max().item()
    print("one token at a time: off by at most %.4f of %.2f" % (off, whole.float().abs().max().item()))
    for kind in (None, "e4m3", "e2m1"):
        paged = block.serve_in_pages(x, kind=kind)
        print("over pages of %s: off by at most %.4f" % (kind or "bf16", (whole.float() - paged.float()).abs().max().item()))
    return losses, off


if __name__ == "__main__":
    main()
