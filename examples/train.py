"""Training a small model end to end on one GPU: a table of item embeddings, layer norms in front of the model, the model's loss and
gradients, their global norm, and AdamW.

    python examples/train.py [--steps 40] [--users 64] [--max-norm 1.0] [--lr 2e-3]

A step is
    H = norm(E[items])                     longer_layer_norm (and G likewise, from a table of global tokens)
    loss, gradients                        longer_forward_backward
    dE, d norm                             longer_layer_norm_backward, then a sum over the places where an item stands
    |gradients|, the factor that bounds it longer_grad_norm, over every parameter at once
    p, m, v, weights                       longer_adamw_step, the factor read on the GPU

Master values and moments are fp32, in one buffer each, in the order of longer_forward_backward's gradients; the kernels read bf16
copies.  The data is synthetic: a user's label says whether a few marked items are among the items of the history."""
import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import longer_synth as synth                     # noqa: E402
import paper_2505_04421_amd as lg                # noqa: E402


def leaves(tree):
    """The tensors of a parameter tree (DeviceModel.parameters, model_grad_views), in its order."""
    if isinstance(tree, dict):
        return [t for k in ("inner", "cross", "self", "head_w", "head_b", "q_learn") + lg.binding.BLOCK_FIELDS if k in tree for t in leaves(tree[k])]
    return [t for x in tree for t in leaves(x)] if isinstance(tree, list) else [tree]


class Trainer:
    """Model, tables, norms, optimizer state and scratch of a run; everything is allocated here."""

    def __init__(self, cfg, items, lr=2e-3, beta1=0.9, beta2=0.98, eps=1e-8, decay=0.01, max_norm=1.0, seed=0):
        self.cfg, self.how, self.max_norm, self.done = cfg, (lr, beta1, beta2, eps), max_norm, 0
        self.model = lg.DeviceModel(cfg, synth.draw_weights(cfg))
        dev = self.model.device
        B, L, d = cfg.B, cfg.L, cfg.d
        r = torch.Generator(device=dev).manual_seed(seed)
        n_model = lg.longer_model_grad_floats(self.model.ccfg)
        # behind the model's parameters: the tables of items and of global tokens, and the two norms' [gain, bias]
        self.extra = [("items", (items, cfg.d_in)), ("globals", (cfg.m, d)), ("norm_h", (2, cfg.d_in)), ("norm_g", (2, d))]
        self.n = n_model + sum(a * b for _, (a, b) in self.extra)
        zeros = lambda dtype=torch.float32: torch.zeros(self.n, dtype=dtype, device=dev)
        self.p, self.m, self.v, self.g, self.w = zeros(), zeros(), zeros(), zeros(), zeros(torch.bfloat16)
        self.model_g = self.g[:n_model]

        def views(flat):
            out, o = {}, n_model
            for name, shape in self.extra:
                out[name] = flat[o:o + shape[0] * shape[1]].view(shape)
                o += shape[0] * shape[1]
            return out

        self.pv, self.gv, self.wv = views(self.p), views(self.g), views(self.w)
        self.pv["items"].normal_(generator=r)
        self.pv["globals"].normal_(generator=r)
        for name in ("norm_h", "norm_g"):
            self.pv[name][0].fill_(1.0)
        weights = leaves(self.model.parameters)
        cut = lambda flat: leaves(lg.model_grad_views(cfg, flat[:n_model])) + [views(flat)[k] for k, _ in self.extra]
        p, m, v, g = (cut(t) for t in (self.p, self.m, self.v, self.g))
        w = weights + [self.wv[k] for k, _ in self.extra]
        for a, b in zip(p[:len(weights)], weights):
            a.copy_(b.view(a.shape))                                     # the model starts from its bf16 weights
        for k, _ in self.extra:
            self.wv[k].copy_(self.pv[k])
        # matrices and tables decay, vectors (biases, gains) do not
        self.params = lg.AdamWList(p, m, v, g, w, [decay if min(t.shape) > 2 else 0.0 for t in (x.view(1, -1) if x.dim() < 2 else x for x in p)])
        self.grads = lg.TensorList(g)
        scratch = lambda n: torch.empty(n, dtype=torch.uint8, device=dev)
        self.ws = scratch(lg.longer_forward_backward_workspace_bytes(self.model.ccfg, B, L))
        self.ws_h = scratch(lg.longer_layer_norm_backward_workspace_bytes(B, L, cfg.d_in))
        self.ws_g = scratch(lg.longer_layer_norm_backward_workspace_bytes(1, cfg.m, d))
        self.ws_n = scratch(lg.longer_grad_norm_workspace_bytes(self.grads))
        self.H, self.G1 = self.model.empty(B, L, cfg.d_in), self.model.empty(1, cfg.m, d)
        f32 = lambda *shape: torch.empty(*shape, device=dev)
        self.dH, self.dG, self.loss, self.norm = f32(B, L, cfg.d_in), f32(B, cfg.m, d), f32(4), f32(2)
        self.last_norm, self.last = torch.empty(2, pin_memory=True), None        # the last step's norm on the host, and when it is there

    def updates(self):
        """The updates so far, which the moments hold and the bias correction counts: every step but those that longer_adamw_step dropped
        because the norm was not finite.  Waits for the last step only."""
        if self.last is not None:
            self.last.synchronize()
            self.done += bool(torch.isfinite(self.last_norm[0]))
            self.last = None
        return self.done

    def step(self, ids, lens, labels):
        """One step on item ids [B, L] (int64), lengths [B] (int32 or None), labels [B]; the loss stays on the GPU."""
        cfg, w, eps = self.cfg, self.wv, self.cfg.ln_eps
        E, G = w["items"][ids], w["globals"][None]
        lg.longer_layer_norm(E, w["norm_h"][0], w["norm_h"][1], lens, eps, self.H)
        lg.longer_layer_norm(G, w["norm_g"][0], w["norm_g"][1], None, eps, self.G1)
        lg.longer_forward_backward(self.model.ccfg, self.model.weights, self.H, self.G1.expand(cfg.B, -1, -1).contiguous(), lens, cfg.B, cfg.L,
                                   labels, self.loss, None, self.dH, self.dG, self.model_g, self.ws)
        lg.longer_layer_norm_backward(E, w["norm_h"][0], self.dH, lens, eps, self.dH, self.gv["norm_h"], self.ws_h)
        dG = self.dG.sum(0, keepdim=True)
        lg.longer_layer_norm_backward(G, w["norm_g"][0], dG, None, eps, dG, self.gv["norm_g"], self.ws_g)
        self.gv["globals"].copy_(dG[0])
        self.gv["items"].zero_().index_add_(0, ids.reshape(-1), self.dH.reshape(-1, cfg.d_in))
        lg.longer_grad_norm(self.grads, self.max_norm, self.norm, self.ws_n)
        # (here the GPU has this step's passes to do while the host waits for the last step's end)
        lg.longer_adamw_step(self.params, self.norm, *self.how, self.updates() + 1)
        self.last_norm.copy_(self.norm, non_blocking=True)
        self.last = torch.cuda.Event()
        self.last.record()


def batch(cfg, items, seed, device):
    """Histories of 1 to L items, and whether one of the first eight items is in them."""
    r = np.random.default_rng(seed)
    ids = r.integers(8, items, (cfg.B, cfg.L))
    lens = r.integers(1, cfg.L + 1, cfg.B).astype(np.int32)
    labels = (r.random(cfg.B) < 0.5).astype(np.float32)
    for u in np.flatnonzero(labels):
        ids[u, r.integers(0, lens[u], 1 + lens[u] // 8)] = r.integers(0, 8)
    up = lambda a: torch.from_numpy(a).to(device)
    return up(ids), up(lens), up(labels)


def small_config(users):
    return synth.CONFIGS["C2"].replace(B=users, L=96, n_self=1, k_recent=16)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--users", type=int, default=64)
    ap.add_argument("--items", type=int, default=1000)
    ap.add_argument("--max-norm", type=float, default=1.0)
    ap.add_argument("--lr", type=float, default=2e-3)
    a = ap.parse_args()
    cfg = small_config(a.users)
    t = Trainer(cfg, a.items, lr=a.lr, max_norm=a.max_norm)
    data = [batch(cfg, a.items, k, t.model.device) for k in range(4)]
    for k in range(a.steps):
        t.step(*data[k % len(data)])
        if k % 4 == 3 or k == a.steps - 1:
            print("step %3d  loss %.4f  gradient norm %.3f  factor %.3f" % (k + 1, float(t.loss[0]), *t.norm.tolist()), flush=True)


if __name__ == "__main__":
    main()
