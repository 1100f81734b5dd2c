"""A long generation through two kinds of attention layers on synthetic data.

Both layers take a prompt of visual and text tokens and then decode one token
per step.

``FullLayer`` attends to its whole cache with ``vp_attend_new`` and bounds it
with ``vp_evict``: the prompt in one call, its last tokens once more as an
observation window that gives every cached token its first accumulated weight,
and then one call per step that attends and adds to the weights.  When the
cache passes ``high`` tokens it is cut to ``keep``: the first tokens, the most
recent ones and those with the largest weights.

``PrunedLayer`` runs ``vp_attend_new`` for the prompt and ``vp_decode_step`` for
the steps: all text, and the visual tokens that the step's query selects.

    python examples/long_generation.py [--batch 8 --steps 512 ...]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_31457_gb300 import vp  # noqa: E402


class Layer:
    def __init__(self, batch, heads, kv_heads, dim, max_visual, max_seq, dtype, max_new, max_weight_new=0):
        self.B, self.H, self.D = batch, heads, dim
        self.k = torch.zeros(batch, kv_heads, max_seq, dim, dtype=dtype, device="cuda")
        self.v = torch.zeros_like(self.k)
        self.seq = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.ctx = vp.vp_init(vp.make_config(batch, heads, kv_heads, dim, max_visual, max_seq,
                                             vp.VP_FP32 if dtype == torch.float32 else vp.VP_BF16))
        vp.vp_reserve_new(self.ctx, max_new, max_weight_new)
        self.kc, self.vc = vp.kv_contiguous(self.k), vp.kv_contiguous(self.v)
        self.everything = vp.make_visible()

    def append(self, k, v):
        """k, v [B, Hkv, n, D]: the keys and values of n new tokens (random here, so not rotated)."""
        self.seq += k.shape[2]
        vp.vp_append(self.ctx, self.B, k.shape[2], None, vp.rows(k.transpose(1, 2)), vp.rows(v.transpose(1, 2)), self.seq,
                     None, None, self.kc, self.vc)

    def attend(self, q, **weights):
        """q [B, n, H, D] of the newest n tokens."""
        out = torch.empty_like(q)
        vp.vp_attend_new(self.ctx, self.B, q.shape[1], vp.rows(q), self.kc, self.vc, self.seq, self.everything,
                         vp.rows(out), **weights)
        return out

    def close(self):
        vp.vp_check_errors(self.ctx)
        vp.vp_free(self.ctx)


class FullLayer(Layer):
    def __init__(self, batch, heads, kv_heads, dim, max_seq, dtype, prompt, high, keep, sinks, recent, observe):
        super().__init__(batch, heads, kv_heads, dim, 0, max_seq, dtype, prompt, observe)
        self.high, self.observe = high, observe
        self.weight = torch.zeros(batch, kv_heads, max_seq, device="cuda")
        self.w = vp.token_weights(self.weight)
        self.policy = vp.make_evict(keep, sinks, recent, granularity=1)
        self.kept = torch.empty(batch, kv_heads, keep, dtype=torch.int32, device="cuda")
        self.keep, self.longest = keep, 0  # longest: tokens of the longest sequence, counted on the host

    def prompt(self, q, k, v):
        self.append(k, v)
        self.longest = k.shape[2]
        out = self.attend(q)
        self.attend(q[:, -self.observe:], weight_out=self.w)
        return out

    def step(self, q, k, v):
        evicted = self.longest >= self.high
        if evicted:
            vp.vp_evict(self.ctx, self.B, self.kc, self.vc, self.seq, self.policy, self.kc, self.vc, self.w, self.w,
                        self.kept, self.keep, self.seq)
            self.longest = min(self.longest, self.keep)
        self.append(k, v)
        self.longest += 1
        return self.attend(q, weight_in=self.w, weight_out=self.w), evicted


class PrunedLayer(Layer):
    def __init__(self, batch, heads, kv_heads, dim, max_seq, dtype, prompt, n_visual):
        super().__init__(batch, heads, kv_heads, dim, n_visual, max_seq, dtype, prompt)
        dev = "cuda"
        self.vis_start = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.vis_len = torch.full((batch,), n_visual, dtype=torch.int32, device=dev)
        self.visual = vp.span(self.vis_start, self.vis_len)  # pointers: the tensors stay with the layer
        self.text = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.n_visual = n_visual
        self.budget = vp.make_budget(vp.VP_ADAPTIVE, tau=0.1)
        self.cap = vp.vp_max_kept(self.budget, n_visual)
        self.kept = torch.empty(batch, self.cap, dtype=torch.int32, device=dev)
        self.count = torch.empty(batch, dtype=torch.int32, device=dev)
        self.mass = torch.empty(batch, heads, device=dev)

    def prompt(self, q, k, v):
        self.append(k, v)
        return self.attend(q)

    def step(self, q, k, v):
        self.append(k, v)
        torch.sub(self.seq, self.n_visual, out=self.text)
        out = torch.empty_like(q)
        vp.vp_decode_step(self.ctx, self.B, q[:, 0], self.kc, self.vc, self.visual, self.text, self.budget, out[:, 0],
                          self.kept, self.cap, self.count, self.mass)
        return out


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in dict(batch=8, heads=28, kv_heads=4, dim=128, visual=2304, text=512, steps=512, high=2816,
                              keep=2304, sinks=4, recent=512, observe=16).items():
        ap.add_argument("--" + name.replace("_", "-"), type=int, default=default)
    a = ap.parse_args()
    gen = torch.Generator("cuda").manual_seed(0)
    prompt = a.visual + a.text

    def tokens(n):
        shape = lambda h: (a.batch, h, n, a.dim)  # noqa: E731
        q = torch.randn(a.batch, n, a.heads, a.dim, device="cuda", generator=gen).bfloat16()
        k, v = (torch.randn(shape(a.kv_heads), device="cuda", generator=gen).bfloat16() for _ in range(2))
        return q, k, v

    full = FullLayer(a.batch, a.heads, a.kv_heads, a.dim, max(prompt, a.high) + 1, torch.bfloat16, prompt, a.high,
                     a.keep, a.sinks, a.recent, a.observe)
    pruned = PrunedLayer(a.batch, a.heads, a.kv_heads, a.dim, prompt + a.steps, torch.bfloat16, prompt, a.visual)
    t = tokens(prompt)
    full.prompt(*t)
    pruned.prompt(*t)
    one = tokens(1)
    evictions = 0
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    for _ in range(a.steps):
        out, evicted = full.step(*one)
        evictions += evicted
        pruned.step(*one)
    end.record()
    torch.cuda.synchronize()
    print(f"{a.steps} steps of both layers, {a.batch} sequences: {start.elapsed_time(end) / a.steps * 1e3:.1f} us a step")
    print(f"full layer: {evictions} evictions, {full.seq.tolist()} tokens cached; "
          f"pruned layer: {pruned.seq.tolist()} cached, {pruned.count.tolist()} visual tokens kept in the last step")
    full.close()
    pruned.close()


if __name__ == "__main__":
    main()
