"""A small sequence model over random walks: one attention layer predicts each walk's next node.

    python examples/walk_encoder.py [--steps 60] [--nodes 20000] [--dim 128] [--heads 4] [--dtype bf16]
                                    [--mixer attention|recurrence] [--norm] [--kept]

One training step: walks from gs_random_walks, their node embeddings gathered, attention of every position
over the positions before it (a walk that met a dead end is shorter), a score of the position's result against
the next node's output embedding and against a few random nodes, the gradients of all parameters clipped to
a joint norm, and a plain SGD update.  Prints the loss, which starts at log(2) per term.
--mixer recurrence puts a gated linear recurrence in the place of attention: its state carries a walk on one node at a time
(WalkEncoder.encode with a state).  --norm normalises the layer's input, --kept keeps that input for the backward pass in 8 bits.
"""
import argparse
import math
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

from paper_2407_15452_b200 import binding as B                       # noqa: E402
from paper_2407_15452_b200 import workloads as WL                    # noqa: E402
from paper_2407_15452_b200.attention import attention, walk_lengths  # noqa: E402
from paper_2407_15452_b200.layers import gated_recurrence, layer_norm  # noqa: E402

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


class WalkEncoder:
    def __init__(self, n_nodes, dim, heads, dtype, seed, device="cuda", mixer="attention", norm=False, kept=False):
        self.heads, self.dtype, self.mixer, self.kept = heads, dtype, mixer, kept
        gen = torch.Generator(device=device).manual_seed(seed)
        table = torch.empty((n_nodes, dim), dtype=torch.float32, device=device)
        B.gs_init_embeddings(table, None, seed)
        rand = lambda *shape: torch.randn(shape, generator=gen, device=device) / math.sqrt(shape[0])      # noqa: E731
        self.params = {"nodes_in": table.mul_(dim).contiguous(), "nodes_out": torch.zeros_like(table),
                       "qkv": rand(dim, 3 * dim), "proj": rand(dim, dim)}
        if mixer == "recurrence":
            self.params["gates"] = self.params.pop("qkv")[:, :2 * dim].contiguous()
        if norm:
            self.params["norm_weight"] = torch.ones(dim, device=device)
            self.params["norm_bias"] = torch.zeros(dim, device=device)
        for p in self.params.values():
            p.requires_grad_(True)

    def encode(self, walks, state=None):
        """Vectors of walks[n, length] at every position, and the recurrence's state after it (None with attention).  The state
        continues the same walks: encode(next_nodes[n, 1], state)."""
        p, (n, length) = self.params, walks.shape
        lens = walk_lengths(walks)
        x = p["nodes_in"][walks.clamp(min=0).long()]
        y = layer_norm(x, p["norm_weight"], p["norm_bias"], lens=lens, checkpoint=self.kept) if "norm_weight" in p else x
        if self.mixer == "recurrence":
            gate, value = (y @ p["gates"]).to(self.dtype).chunk(2, dim=-1)
            out, state = gated_recurrence(gate, value, state, lens)
        else:
            qkv = (y @ p["qkv"]).to(self.dtype).view(n, length, 3, self.heads, -1)
            out = attention(qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2], window=(-1, 0), q_lens=lens, k_lens=lens)
        return x + out.reshape(n, length, -1).float() @ p["proj"], state

    def loss(self, walks, negatives):
        """Logistic loss of the next node (positive) and of `negatives`[n_walks, walk_len - 1, k]:
        (sum per walk, mean per term)."""
        p, n = self.params, walks.shape[0]
        h, _ = self.encode(walks)
        h, nxt = h[:, :-1], walks[:, 1:]
        keep = (nxt >= 0).float()
        pos = (h * p["nodes_out"][nxt.clamp(min=0).long()]).sum(-1)
        neg = torch.einsum("nld,nlkd->nlk", h, p["nodes_out"][negatives])
        per_pos = torch.nn.functional.softplus(-pos) + torch.nn.functional.softplus(neg).sum(-1)
        total = (per_pos * keep).sum()
        return total / n, total.detach() / (keep.sum() * (1 + negatives.shape[2])).clamp(min=1.0)

    def step(self, walks, negatives, lr, max_norm):
        loss, per_term = self.loss(walks, negatives)
        for p in self.params.values():
            p.grad = None
        loss.backward()
        grads = [p.grad for p in self.params.values()]
        norm = B.gs_clip_gradients(grads, max_norm)
        with torch.no_grad():
            for p in self.params.values():
                p.sub_(p.grad, alpha=lr)
        return per_term, norm


def train(steps=60, nodes=20000, dim=128, heads=4, dtype="bf16", walks_per_step=512, walk_len=40, n_neg=5,
          lr=2.0, max_norm=1.0, seed=7, log=None, mixer="attention", norm=False, kept=False):
    graph = WL.chung_lu_graph(nodes, 10, 2.3, seed=seed)
    g = B.gs_graph_load_csr(graph.offsets.to("cuda"), graph.cols.to("cuda"), B.GS_VALIDATE)
    model = WalkEncoder(graph.n_nodes, dim, heads, DTYPES[dtype], seed, mixer=mixer, norm=norm, kept=kept)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    losses, norms = [], []
    for s in range(steps):
        walks = B.gs_random_walks(g, None, walks_per_step, s * walks_per_step, walk_len, seed)
        negatives = torch.randint(0, graph.n_nodes, (walks_per_step, walk_len - 1, n_neg), generator=gen, device="cuda")
        loss, norm = model.step(walks, negatives, lr, max_norm)
        losses.append(loss)
        norms.append(norm)
        if log and (s % 10 == 0 or s == steps - 1):
            log(f"step {s:4d}  loss per term {loss.item():.4f}  gradient norm {norm.item():.3f}")
    return torch.stack(losses).cpu(), torch.cat(norms).cpu(), model


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--nodes", type=int, default=20000)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--heads", type=int, default=4)
    ap.add_argument("--dtype", choices=sorted(DTYPES), default="bf16")
    ap.add_argument("--mixer", choices=["attention", "recurrence"], default="attention")
    ap.add_argument("--norm", action="store_true")
    ap.add_argument("--kept", action="store_true")
    a = ap.parse_args()
    train(a.steps, a.nodes, a.dim, a.heads, a.dtype, log=print, mixer=a.mixer, norm=a.norm or a.kept, kept=a.kept)
