"""A small mixture of experts over an embedding, trained with the library end to end on one GPU: where tokens go, and what comes back.

    python examples/train_experts.py [--steps 40] [--tokens 2048] [--words 5000] [--width 256] [--hidden 512] [--experts 8]

    x0 = dropout(sqrt(width) E[word]),   n = rms(x0) w,   experts of a token: the best two of n R^T, weighted by their softmax
    u = n[token] W1_g^T + b1_g,   a = max(u, 0)^2,   o = a W2_g^T,   y = x0 + dropout(sum over a token's experts of weight o)
Tokens are sorted by word once and by expert once.  The embedding's gradient goes by the first order; dispatch and return are lookups that are each other's
gradients, the experts' products and weight gradients go by the second one's offsets.  The weight gradients find n and a in 8 bits, in the experts'
order, and no dropout mask is stored.  Words and experts that a step does not touch get zero gradients, whose pages the update
skips.  The router's product and softmax, and the activation function, are torch's.  The task: another random network's output.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2303_02868_amd as apm  # noqa: E402
from train_blocks import BF16, DEV, EPS, kept_like  # noqa: E402

PICKED = 2      # experts of a token


def whole(n, dtype=torch.int32):
    return torch.empty(n, dtype=dtype, device=DEV)


class Order:
    """Positions sorted by id, and everything that is asked of such an order."""

    def __init__(self, ids, rows):
        n = ids.numel()
        self.ids, self.offsets, self.place, self.token = ids, whole(rows + 1, torch.int64), whole(n), whole(n)
        self.order = whole(n)
        self.sorted = apm.make_token_order(ids, rows, self.order, offsets=self.offsets, place=self.place, token=self.token)
        self.room = torch.empty(max(16, apm.apm_sort_tokens_workspace_bytes(self.sorted)), dtype=torch.uint8, device=DEV)

    def sort(self):
        apm.apm_sort_tokens(self.sorted, self.room)


class Parameters:
    """bf16 parameters and gradients as tensors; fp32 masters and moments in the pages of a pool, small ones, so that few words share one."""

    def __init__(self, shapes, generator, page_elems=1 << 12):
        self.names, self.numels = list(shapes), [int(torch.Size(s).numel()) for s in shapes.values()]
        masters = [torch.ones(s, device=DEV) if n == "norm" else torch.zeros(s, device=DEV) if n == "b1" else
                   torch.randn(s, device=DEV, generator=generator) * s[-1] ** -0.5 for n, s in shapes.items()]
        self.value = {n: m.to(BF16) for n, m in zip(self.names, masters)}
        self.grad = {n: torch.zeros_like(v) for n, v in self.value.items()}
        plan = apm.apm_pack_plan(page_elems, self.numels)
        self.pool, self.pages = apm.apm_pool_create(apm.APM_DEV_GPU, page_elems, plan.n_pages), plan.n_pages
        apm.apm_pack_tensors(self.pool, apm.APM_P32, apm.make_tensors(self.numels, apm.APM_F32, masters), len(masters))
        self.skipped = torch.zeros(self.pages, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        self.steps = 0

    def step(self, lr):
        self.steps += 1
        lists = [apm.make_tensors(self.numels, apm.APM_BF16, [d[n] for n in self.names]) for d in (self.grad, self.value)]
        hyper = apm.make_hyper(lr=lr, weight_decay=0.0, skip_mode=apm.APM_SKIP_UNTOUCHED)
        apm.apm_page_adamw_step_fused(self.pool, None, self.pages, self.steps, hyper, *lists, len(self.names), skip_mask=self.skipped)


class Network:
    def __init__(self, tokens, words, width, hidden, experts, drop=0.1, form=apm.APM_CKPT_I8, seed=0):
        self.tokens, self.width, self.hidden, self.experts, self.drop, self.seed = tokens, width, hidden, experts, drop, seed
        n = tokens * PICKED
        self.p = Parameters({"E": (words, width), "norm": (width,), "R": (experts, width), "W1": (experts, hidden, width), "b1": (experts, hidden),
                             "W2": (experts, width, hidden)}, torch.Generator(device=DEV).manual_seed(seed))

        def make(rows, cols, dtype=BF16):
            return torch.empty(rows, cols, dtype=dtype, device=DEV)

        self.step_word = torch.zeros(1, dtype=torch.int64, device=DEV)      # added to the dropout's seed: another mask each step
        self.by_word = Order(whole(tokens, torch.int64), words)
        self.by_expert = Order(whole(n).view(tokens, PICKED), experts)
        self.x0, self.x, self.n = make(tokens, width, torch.float32), make(tokens, width, torch.float32), make(tokens, width)
        self.hat, self.rstd = kept_like(tokens, width, form), torch.empty(tokens, device=DEV)
        self.n_sorted, self.u, self.o = make(n, width), make(n, hidden), make(n, width)
        self.n_kept, self.a_kept = kept_like(n, width, form), kept_like(n, hidden, form)
        self.back, self.y = make(tokens, width), make(tokens, width, torch.float32)
        self.join = apm.make_norm_join(tokens, width, x=self.x, n=self.n, pre_norm=apm.APM_NORM_RMS, pre_eps=EPS, pre_weight=self.p.value["norm"],
                                       pre_ckpt=self.hat, pre_rstd=self.rstd)
        self.room = torch.empty(apm.apm_norm_join_workspace_bytes(tokens, width), dtype=torch.uint8, device=DEV)

    def dropout(self, x, y, layer, residual=None):
        apm.apm_dropout_apply(apm.make_dropout(x, y, p=self.drop, seed=self.seed, seed_at=self.step_word, layer=layer, residual=residual))

    def product(self, x, name, y, bias=None, transposed=False):
        p = apm.make_grouped_product(x, self.p.value[name], y, offsets=self.by_expert.offsets, bias=bias, transposed=transposed)
        size = apm.apm_grouped_product_workspace_bytes(p)
        apm.apm_grouped_product(p, torch.empty(size, dtype=torch.uint8, device=DEV) if size else None)

    def weight_gradient(self, dy, kept, name, db=None):
        grad = apm.make_weight_grad(dy, kept, self.p.grad[name], db=db, offsets=self.by_expert.offsets)
        size = apm.apm_ckpt_weight_grad_workspace_bytes(grad)
        apm.apm_ckpt_weight_grad(grad, torch.empty(size, dtype=torch.uint8, device=DEV) if size else None)

    def forward(self, words):
        v = self.p.value
        self.by_word.ids.copy_(words)
        self.by_word.sort()
        apm.apm_lookup_forward(apm.make_lookup(self.by_word.ids, v["E"], self.x0, scale=self.width ** 0.5))
        self.dropout(self.x0, self.x, layer=0)
        apm.apm_norm_join_forward(self.join)
        scores = self.n.float() @ v["R"].float().T
        self.scores, picked = torch.topk(scores, PICKED, dim=1)
        self.weights = torch.softmax(self.scores, 1)
        self.by_expert.ids.copy_(picked)
        self.by_expert.sort()
        apm.apm_lookup_forward(apm.make_lookup(self.by_expert.token, self.n, self.n_sorted))
        apm.apm_ckpt_write(self.n_sorted, self.n_kept)
        self.product(self.n_sorted, "W1", self.u, bias=v["b1"])
        a = self.u.relu().square()
        apm.apm_ckpt_write(a, self.a_kept)
        self.product(a, "W2", self.o)
        self.returned = apm.make_lookup(self.by_expert.place.view(self.tokens, PICKED), self.o, self.back, weights=self.weights)
        apm.apm_lookup_forward(self.returned)
        self.dropout(self.back, self.y, layer=1, residual=self.x)
        return self.y

    def backward(self, dy):
        v, g = self.p.value, self.p.grad
        dy = dy.contiguous()
        dback, do, dn_sorted = torch.empty_like(self.back), torch.empty_like(self.o), torch.empty_like(self.n_sorted)
        dweights, dn, dx, dx0 = torch.empty_like(self.weights), torch.empty_like(self.n), torch.empty_like(self.x), torch.empty_like(self.x)
        self.dropout(dy, dback, layer=1)
        # back to the experts: row i of their outputs belongs to one position, whose weight it gets
        apm.apm_lookup_backward(self.returned, apm.make_lookup_grads(self.returned, dback, dweights=dweights))
        apm.apm_lookup_forward(apm.make_lookup(self.by_expert.token, dback, do, weights=self.weights.flatten()[self.by_expert.order.long()]))
        self.weight_gradient(do, self.a_kept, "W2")
        du = torch.empty_like(self.u)
        self.product(do, "W2", du, transposed=True)
        du *= 2 * self.u.relu()
        self.weight_gradient(du, self.n_kept, "W1", db=g["b1"])
        self.product(du, "W1", dn_sorted, transposed=True)
        apm.apm_lookup_forward(apm.make_lookup(self.by_expert.place.view(self.tokens, PICKED), dn_sorted, dn))
        # the router
        dpicked = self.weights * (dweights - (self.weights * dweights).sum(1, keepdim=True))
        dscores = torch.zeros(self.tokens, self.experts, device=DEV).scatter_(1, self.by_expert.ids.long(), dpicked)
        g["R"].copy_(dscores.T @ self.n.float())
        dn += (dscores @ v["R"].float()).to(BF16)
        apm.apm_norm_join_backward(self.join, apm.make_norm_join_grads(self.join, dn=dn, dy=dy, dx=dx, dpre_weight=g["norm"]), self.room)
        self.dropout(dx, dx0, layer=0)
        looked = apm.make_lookup(self.by_word.ids, None, scale=self.width ** 0.5, rows=v["E"].shape[0], cols=self.width)
        room = torch.empty(max(16, apm.apm_lookup_workspace_bytes(looked)), dtype=torch.uint8, device=DEV)
        apm.apm_lookup_backward(looked, apm.make_lookup_grads(looked, dx0, order=self.by_word.sorted, dtable=g["E"]), room)


def train(steps=40, tokens=2048, words=5000, width=256, hidden=512, experts=8, lr=2e-3, seed=0, say=print):
    net, teacher = Network(tokens, words, width, hidden, experts, seed=seed), Network(tokens, words, width, hidden, experts, drop=0.0, seed=seed + 1)
    g = torch.Generator(device=DEV).manual_seed(seed + 2)
    share = 1.0 / (torch.arange(words, device=DEV) + 2.7)
    losses = []
    for step in range(steps):
        batch = torch.multinomial(share, tokens, replacement=True, generator=g)
        net.step_word.fill_(step)
        error = net.forward(batch) - teacher.forward(batch)
        losses.append(error.square().mean())
        net.backward(error * (2.0 / tokens))
        net.p.step(lr)
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step}: loss {float(losses[-1]):.4f}, {int(net.p.skipped.sum())} of {net.p.pages} pages untouched")
    return [float(v) for v in losses]


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("steps", 40), ("tokens", 2048), ("words", 5000), ("width", 256), ("hidden", 512), ("experts", 8)):
        parser.add_argument("--" + name, type=int, default=default)
    train(**vars(parser.parse_args()))
