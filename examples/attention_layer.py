"""A transformer layer over voxel tokens from the framework's operators.

The tokens' features stand for what the lattice filter gives at a volume's voxels.  The layer is

    x0 = drop(features)                                          pam_dropout
    h  = N(x0) w_pre                                             pam_norm_gate_fwd
    q, k, v = h W;  q, k turned by the voxels' coordinates       pam_rotary_table, pam_rotary
    o  = differential attention of q, k, v                       pam_diff_attn_fwd
    r  = x0 + drop(scale gate N(o W_o))                          pam_norm_gate_fwd

with its backward pass written out (pam_norm_gate_bwd, pam_diff_attn_bwd, pam_rotary with ``inverse``, and
pam_dropout again).  ``train`` fits the layer to a target; ``generate`` runs a causal layer over a prompt at once and
then token by token over a cache of keys and values, which gives the same outputs.  The projections are plain matrix
products (torch).

    python examples/attention_layer.py            # a few steps on the GPU, one line each
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1907_00641_amd as pam  # noqa: E402


class Layer:
    """Weights of the layer and its passes.  Activations are of type ``dtype``, as are the matrices; the norms'
    vectors are fp32."""

    def __init__(self, channels, heads, kv_heads, dim, dtype, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def matrix(n, m):
            return (torch.randn(n, m, generator=g, device=device) * n ** -0.5).to(dtype)

        self.channels, self.heads, self.kv_heads, self.dim = channels, heads, kv_heads, dim
        self.w = {"wq": matrix(channels, heads * 2 * dim), "wk": matrix(channels, kv_heads * 2 * dim),
                  "wv": matrix(channels, kv_heads * 2 * dim), "wo": matrix(heads * 2 * dim, channels),
                  "lam": torch.full((heads,), 0.5, device=device).to(dtype),
                  "w_pre": torch.ones(channels, device=device), "w_post": torch.ones(channels, device=device),
                  "scale": torch.full((channels,), 0.5, device=device)}

    def _project(self, h, b, n):
        w, (hq, hk, d) = self.w, (self.heads, self.kv_heads, self.dim)
        return ((h @ w["wq"]).view(b, n, hq, 2, d), (h @ w["wk"]).view(b, n, hk, 2, d),
                (h @ w["wv"]).view(b, n, hk, 2 * d))

    def _turn(self, q, k, table, start=0, inverse=False):
        """Both maps of every head, turned as heads of their own."""
        b, n, d = q.shape[0], q.shape[1], self.dim
        q2, k2 = pam.pam_rotary(q.reshape(b, n, -1, d), k.reshape(b, n, -1, d), table, start=start, inverse=inverse)
        return q2.view_as(q), k2.view_as(k)

    def forward(self, x, table, gate=None, p=0.0, seed=0, causal=False):
        """x: b x n x channels; gate: b x channels.  Returns r and what ``backward`` needs."""
        b, n, c = x.shape
        w = self.w
        x0 = pam.pam_dropout(x, p, seed, 0) if p else x
        flat = x0.view(b * n, c)
        _, h = pam.pam_norm_gate_fwd(flat, w_pre=w["w_pre"])
        q, k, v = self._project(h, b, n)
        q, k = self._turn(q, k, table)
        o, saved = pam.pam_diff_attn_fwd(q, k, v, w["lam"], causal=causal, save=True)
        z = o.view(b * n, -1) @ w["wo"]
        how = dict(z=z, w_post=w["w_post"], gate=gate, scale=w["scale"], p=p, seed=seed, offset=1)
        r, _ = pam.pam_norm_gate_fwd(flat, **how, next_norm=False)
        return r.view(b, n, c), (flat, h, q, k, v, o, saved, how, (b, n, p, seed, causal, table))

    def backward(self, kept, grad_r):
        """Gradients of the weights by their names, of the gate as "gate", of the features as "x"."""
        flat, h, q, k, v, o, saved, how, (b, n, p, seed, causal, table) = kept
        w = self.w
        post = pam.pam_norm_gate_bwd(flat, grad_r=grad_r.reshape(b * n, -1), grad_h=None, **how)
        out = {"w_post": post["w_post"], "scale": post["scale"], "gate": post["gate"]}
        out["wo"] = o.view(b * n, -1).t() @ post["z"]
        gq, gk, gv, out["lam"] = pam.pam_diff_attn_bwd(q, k, v, w["lam"], saved, (post["z"] @ w["wo"].t()).view_as(o),
                                                       causal=causal)
        gq, gk = self._turn(gq, gk, table, inverse=True)
        gq, gk, gv = (t.reshape(b * n, -1) for t in (gq, gk, gv))
        for name, t in (("wq", gq), ("wk", gk), ("wv", gv)):
            out[name] = h.t() @ t
        gh = gq @ w["wq"].t() + gk @ w["wk"].t() + gv @ w["wv"].t()
        pre = pam.pam_norm_gate_bwd(flat, grad_r=post["x"], grad_h=gh, w_pre=w["w_pre"])
        out["w_pre"] = pre["w_pre"]
        gx = pre["x"].view(b, n, -1)
        out["x"] = pam.pam_dropout(gx, p, seed, 0) if p else gx
        return out

    def cache(self, b, size):
        w = self.w["wk"]
        shape = (b, size, self.kv_heads)
        return w.new_zeros(*shape, 2, self.dim), w.new_zeros(*shape, 2 * self.dim)

    def extend(self, x, cache, at, table, gate=None):
        """The causal layer on tokens x (b x n x channels) that follow the ``at`` tokens in the cache, whose keys and
        values are added to it."""
        b, n, c = x.shape
        w, flat = self.w, x.reshape(b * n, c)
        _, h = pam.pam_norm_gate_fwd(flat, w_pre=w["w_pre"])
        q, k, v = self._project(h, b, n)
        q, k = self._turn(q, k, table, start=at)
        cache[0][:, at:at + n], cache[1][:, at:at + n] = k, v
        length = torch.full((b,), at + n, dtype=torch.int32, device=x.device)
        o = pam.pam_diff_attn_fwd(q, cache[0], cache[1], w["lam"], causal=True, k_len=length)
        r, _ = pam.pam_norm_gate_fwd(flat, z=o.view(b * n, -1) @ w["wo"], w_post=w["w_post"], gate=gate,
                                     scale=w["scale"], next_norm=False)
        return r.view(b, n, c)


def voxel_table(side, dim, device="cuda"):
    """Rotary table of the voxels of a cube, the pairs dealt to its three axes in turn."""
    pairs = dim // 2
    freq, mag = pam.pam_rotary_frequencies(2 * max((pairs + 2) // 3, 1), base=100.0)
    grid = torch.stack(torch.meshgrid(*[torch.arange(side, dtype=torch.float32)] * 3, indexing="ij"), -1)
    which = torch.arange(pairs)
    return pam.pam_rotary_table(freq[which // 3].to(device), coord=grid.reshape(-1, 3).to(device),
                                axis=(which % 3).to(torch.int32).to(device), magnitude=mag)


def train(steps=8, side=8, batch=2, channels=64, heads=4, kv_heads=2, dim=32, p=0.1, rate=0.5, dtype=torch.bfloat16,
          say=print):
    """Fits the layer to a target that a layer with other weights gives; returns the losses."""
    n = side ** 3
    table = voxel_table(side, dim)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.randn(batch, n, channels, generator=gen, device="cuda").to(dtype)
    gate = torch.rand(batch, channels, generator=gen, device="cuda").add(0.5).to(dtype)
    target = Layer(channels, heads, kv_heads, dim, dtype, seed=7).forward(x, table, gate)[0]
    layer, losses = Layer(channels, heads, kv_heads, dim, dtype), []
    master = {name: t.float() for name, t in layer.w.items()}
    for step in range(steps):
        r, kept = layer.forward(x, table, gate, p=p, seed=step)
        diff = r.float() - target.float()
        losses.append(float(diff.square().mean()))
        say(f"step {step}: loss {losses[-1]:.4f}", flush=True)
        grads = layer.backward(kept, (2.0 / (batch * n) * diff).to(dtype))
        for name, t in master.items():
            t -= rate * grads[name].float()
            layer.w[name] = t.to(layer.w[name].dtype)
    return losses


def generate(tokens=70, prompt=40, batch=2, channels=64, heads=4, kv_heads=2, dim=32, dtype=torch.bfloat16):
    """The causal layer over all tokens at once, and over a prompt and then token by token; returns both."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    x = torch.randn(batch, tokens, channels, generator=gen, device="cuda").to(dtype)
    freq, mag = pam.pam_rotary_frequencies(dim)
    table = pam.pam_rotary_table(freq.cuda(), entries=tokens, magnitude=mag)
    layer = Layer(channels, heads, kv_heads, dim, dtype)
    whole = layer.forward(x, table, causal=True)[0]
    cache = layer.cache(batch, tokens)
    parts = [layer.extend(x[:, :prompt], cache, 0, table)]
    for at in range(prompt, tokens):
        parts.append(layer.extend(x[:, at:at + 1], cache, at, table))
    return whole, torch.cat(parts, 1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--side", type=int, default=16, help="voxels along each axis of the cube")
    args = ap.parse_args(argv)
    train(steps=args.steps, side=args.side, channels=128)
    whole, parts = generate()
    off = (whole.float() - parts.float()).abs().max().item()
    print(f"token by token: largest difference from the whole pass {off:.4f}")


if __name__ == "__main__":
    main()
