"""Train a small FLARE++ sequence classifier on one GPU, every layer by libflarepp.

    python examples/train_sequences.py [--steps 60] [--state-bits 8]

Byte-like sequences of different lengths, padded with -1, of ten classes (a class favours its own
bytes). The model: token embedding, one block (x + mixer(x), then x + MLP(x) with GELU, ratio 2),
mean over the positions that exist, logits. The embedding, the mixer layer, the linear layers with
their bias, activation and residual, all gradients and the AdamW step run in the library; torch holds
the tensors, adds the mixer's residual, takes the mean and computes the loss."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_11519_gb300 import flarepp  # noqa: E402

CLASSES = 10


def batch(gen, B, N, vocab, dev):
    """Sequences [B, N] (-1 from each one's end on) and their classes [B]."""
    cls = torch.randint(0, CLASSES, (B,), generator=gen, device=dev)
    any_id = torch.randint(0, vocab, (B, N), generator=gen, device=dev)
    own_id = cls.unsqueeze(1) * (vocab // CLASSES) + any_id % (vocab // CLASSES)
    ids = torch.where(torch.rand(B, N, generator=gen, device=dev) < 0.2, own_id, any_id)
    ends = torch.randint(N // 2, N + 1, (B, 1), generator=gen, device=dev)
    return ids.masked_fill(torch.arange(N, device=dev) >= ends, -1), cls


class Model:
    def __init__(self, vocab=257, H=8, D=32, M=64, dev="cuda", seed=0):
        self.V, self.H, self.D, self.M, self.C = vocab, H, D, M, H * D
        C, gen = self.C, torch.Generator(device=dev).manual_seed(seed)

        def normal(*shape, std):
            return (torch.randn(*shape, generator=gen, device=dev) * std).bfloat16()

        def zeros(n):
            return torch.zeros(n, dtype=torch.bfloat16, device=dev)

        self.p = {"emb": normal(vocab, C, std=C ** -0.5), "W_in": normal(4 * C, C, std=C ** -0.5),
                  "Wo": normal(C, C, std=C ** -0.5), "seeds": normal(H, M, D, std=1.0),
                  "W1": normal(2 * C, C, std=C ** -0.5), "b1": zeros(2 * C),
                  "W2": normal(C, 2 * C, std=(2 * C) ** -0.5), "b2": zeros(C),
                  "Wc": normal(CLASSES, C, std=C ** -0.5), "bc": zeros(CLASSES)}
        self.g = {k: torch.zeros_like(v) for k, v in self.p.items()}

    def step(self, ids, cls):
        """Loss (a device scalar) and this batch's gradients in ``self.g``."""
        p, g, scale = self.p, self.g, math.sqrt(self.C)
        here = (ids >= 0).unsqueeze(-1)
        count = here.sum(1, keepdim=True)
        # forward
        x = flarepp.embedding_fwd(ids, p["emb"], scale)
        o, kept = flarepp.mixer_fwd_train(x, p["W_in"], p["Wo"], p["seeds"])
        h = x + o
        a, z = flarepp.linear_fwd_train(h, p["W1"], p["b1"], act="gelu")
        y, _ = flarepp.linear_fwd_train(a, p["W2"], p["b2"], residual=h)
        pooled = ((y.float() * here).sum(1) / count.squeeze(1)).bfloat16()
        logits = flarepp.linear_fwd(pooled, p["Wc"], p["bc"]).float()
        logp = torch.log_softmax(logits, -1)
        loss = -logp.gather(1, cls.unsqueeze(1)).mean()
        # backward
        dlogits = logp.exp()
        dlogits.scatter_add_(1, cls.unsqueeze(1), torch.full_like(logits, -1.0))
        dlogits = (dlogits / len(cls)).bfloat16()
        dpooled, _, _ = flarepp.linear_bwd(pooled, p["Wc"], dlogits, dW=g["Wc"], db=g["bc"])
        dy = (dpooled.float().unsqueeze(1) / count * here).bfloat16()
        da, _, _ = flarepp.linear_bwd(a, p["W2"], dy, dW=g["W2"], db=g["b2"])
        dh, _, _ = flarepp.linear_bwd(h, p["W1"], da, z, "gelu", dW=g["W1"], db=g["b1"])
        dh = dh + dy  # the MLP's residual
        dx = torch.empty_like(x)
        flarepp.mixer_bwd(x, p["W_in"], p["Wo"], p["seeds"], kept, dh,
                          grads=(dx, g["W_in"], g["Wo"], g["seeds"]))
        flarepp.embedding_bwd(ids, dx + dh, self.V, scale, dtable=g["emb"])
        return loss, logits


def check(dev):
    """Stop where a layer's kernel gave up or met an id beyond the table: what it wrote is no result."""
    status = flarepp.layers_status(dev)
    if status != flarepp.OK:
        raise flarepp.FlareppError(status, "a layer's kernel")


def train(steps=60, B=16, N=1024, state_bits=8, lr=2e-3, seed=0, log=None):
    """The losses of ``steps`` steps, and the accuracy on a fresh batch at the end."""
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev).manual_seed(seed + 1)
    model = Model(dev=dev, seed=seed)
    names = list(model.p)
    opt = flarepp.AdamW([model.p[k] for k in names], [model.g[k] for k in names], lr=lr,
                        state_bits=state_bits, masters=True,
                        state_rounding="unbiased" if state_bits == 8 else "nearest")
    losses = []
    for k in range(steps):
        loss, _ = model.step(*batch(gen, B, N, model.V, dev))
        opt.lr = lr * (1 - k / steps)
        opt.step()
        losses.append(loss)
        if log and k % 10 == 0:
            log(f"step {k:3d}  loss {float(loss):.4f}")
            check(dev)
    ids, cls = batch(gen, 4 * B, N, model.V, dev)
    _, logits = model.step(ids, cls)
    check(dev)
    return [float(x) for x in losses], float((logits.argmax(1) == cls).float().mean())


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    args = ap.parse_args()
    _, accuracy = train(args.steps, state_bits=args.state_bits, log=print)
    print(f"accuracy on a fresh batch: {accuracy:.3f}")
