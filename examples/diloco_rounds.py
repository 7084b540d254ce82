"""A few DiLoCo rounds on one GPU: K workers train a small language model from the same
parameters, the IsoLoCo outer step merges them.

The inner steps run on the package's operators (embedding, gated feed-forward block,
token log probabilities, gradient clipping) around torch's matrix products, the outer
step on ``IsoLoCoPlan``.  Parameters, replicas and gradients are flat float32 buffers of
one layout; the compute is bfloat16.  The data is a synthetic source whose next token
mostly follows from the last one, so the model needs no attention.

    python examples/diloco_rounds.py --rounds 4 --workers 4 --inner-steps 20
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_03011_amd as iso  # noqa: E402


def token_loss(logits, targets):
    """The mean of -log p(target); targets of -1 are ignored."""
    return -iso.token_logprobs(logits, targets).logprob.sum() / (targets >= 0).sum().clamp(min=1)


class Model:
    """Tied embedding and ``blocks`` gated feed-forward blocks in a flat buffer."""

    def __init__(self, vocab, dim, hidden, blocks):
        self.shapes = [(vocab, dim)]
        for _ in range(blocks):
            self.shapes += [(dim,), (hidden, dim), (hidden, dim), (dim, hidden)]
        self.layout, self.n = [], 0
        for s in self.shapes:
            # 1-D tensors take the plain mean, matrices the corrected one
            self.layout.append((self.n, s[0], s[1] if len(s) > 1 else 1, 0 if len(s) > 1 else 1))
            self.n += math.prod(s)
        self.scale = math.sqrt(dim)

    def views(self, flat):
        return [flat[off:off + rows * cols].view(s) for (off, rows, cols, _), s in zip(self.layout, self.shapes)]

    def init(self, flat, generator):
        for p in self.views(flat):
            if p.dim() == 1:
                p.fill_(1.0)
            else:
                p.copy_(torch.randn(p.shape, generator=generator, device=p.device) * 0.02)

    def logits(self, params, ids):
        table = params[0]
        h = iso.embedding(table, ids, scale=self.scale, out_dtype=torch.bfloat16)
        for gain, w_gate, w_up, w_down in zip(*[iter(params[1:])] * 4):
            x = torch.nn.functional.rms_norm(h.float(), gain.shape, gain).bfloat16()
            h = h + iso.gated_ffn(x, w_gate.bfloat16(), w_up.bfloat16()) @ w_down.bfloat16().T
        return h @ table.bfloat16().T


class Source:
    """Tokens whose successor is fixed nine times in ten."""

    def __init__(self, vocab, seed, device):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.vocab, self.next = vocab, torch.randperm(vocab, generator=g, device=device)

    def batch(self, tokens, generator):
        dev = self.next.device
        ids = torch.randint(0, self.vocab, (tokens,), generator=generator, device=dev)
        targets = self.next[ids]
        noise = torch.rand(tokens, generator=generator, device=dev) < 0.1
        targets[noise] = torch.randint(0, self.vocab, (int(noise.sum()),), generator=generator, device=dev)
        return ids, targets


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rounds", type=int, default=4)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--inner-steps", type=int, default=20)
    ap.add_argument("--tokens", type=int, default=1024, help="tokens of a worker's batch")
    ap.add_argument("--vocab", type=int, default=512)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--hidden", type=int, default=344)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--max-norm", type=float, default=1.0)
    a = ap.parse_args(argv)

    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev)
    g.manual_seed(0)
    model, source = Model(a.vocab, a.dim, a.hidden, a.blocks), Source(a.vocab, 1, dev)
    theta, momentum = torch.empty(model.n, device=dev), torch.zeros(model.n, device=dev)
    model.init(theta, g)
    workers = torch.empty(a.workers, (model.n + 3) // 4 * 4, device=dev)[:, :model.n]
    # each worker's parameters are views of its replica, with gradients in a flat buffer
    params, optimizers = [], []
    for k in range(a.workers):
        views = [v.detach().requires_grad_() for v in model.views(workers[k])]
        for v, d in zip(views, model.views(torch.zeros(model.n, device=dev))):
            v.grad = d
        params.append(views)
        optimizers.append(torch.optim.AdamW(views, lr=3e-3, betas=(0.9, 0.95), weight_decay=0.1))
    plan = iso.IsoLoCoPlan(model.layout, model.n, a.workers, iso.ISOLOCO_F32)
    held_out = source.batch(4096, g)
    losses = []

    def validate(r):
        with torch.no_grad():
            out = iso.token_logprobs(model.logits(model.views(theta), held_out[0]), held_out[1], top_k=1)
        losses.append(-out.logprob.mean().item())
        hit = (out.top_index[:, 0] == held_out[1]).float().mean().item()
        print("round %d: validation loss %.4f, entropy %.4f, best token right %.1f%%" %
              (r, losses[-1], out.entropy.mean().item(), 100 * hit), flush=True)

    validate(0)
    for r in range(1, a.rounds + 1):
        workers.copy_(theta.expand(a.workers, -1))
        for k in range(a.workers):
            for _ in range(a.inner_steps):
                for p in params[k]:
                    p.grad.zero_()
                ids, targets = source.batch(a.tokens, g)
                token_loss(model.logits(params[k], ids), targets).backward()
                norm = iso.clip_grads([p.grad for p in params[k]], a.max_norm)
                optimizers[k].step()
            print("round %d, worker %d: gradient norm %.3f, scaled by %.3f" % (r, k, *norm.tolist()), flush=True)
        plan.aggregate(theta, workers, momentum, alpha=1.0, outer_lr=0.7, mu=0.9)
        validate(r)
    plan.close()
    return losses


if __name__ == "__main__":
    main()
