"""From ratings to rankings, on one MI355X.

1. Learn factors U, V from ratings with the blocked SGD sweep (bgmf.Model).
2. Train them further on choices: the softmax over the catalogue of the items
   that users rated highly, its gradient, clipped by the global norm.
3. Answer requests: the item factors in 8-bit integers, laid out once; per
   request the user's scores over the whole catalogue, and the best items among
   those the user has not rated, with their log probabilities.

    python examples/rank_items.py [--epochs 3] [--steps 300] [--batch 4096]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2304_13724_amd import bgmf, ranking  # before torch: one HIP runtime in the process

import numpy as np
import torch

from workloads import make_config


def learn(w, epochs):
    """Factors of the workload's ratings, as PyTorch tensors that the sweep updates."""
    U, V = torch.from_numpy(w.U0).cuda(), torch.from_numpy(w.V0).cuda()
    with bgmf.Model(w.n, w.m, w.k, w.p) as model:
        ws = torch.empty(model.query_sizes(len(w.rows))["incore_ws_bytes"], dtype=torch.uint8,
                         device="cuda")
        model.bind_tensors(U, V, ws, stream=torch.cuda.current_stream().cuda_stream)
        model.load_coo(w.rows, w.cols, w.vals)
        for _ in range(epochs):
            model.epoch(w.alpha, w.beta)
            print(f"sweep: rmse {model.rmse():.4f}", flush=True)
    return U, V


def train_on_choices(U, V, users, items, steps, batch, rate, max_norm, temperature, seed):
    """SGD on -log p(item | user), with a little entropy kept, in place."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    losses = []
    for _ in range(steps):
        pick = torch.randint(0, len(users), (batch,), generator=g, device="cuda")
        u = U[users[pick]].requires_grad_()
        v = V.detach().requires_grad_()
        r = ranking.log_probs(u @ v.t(), items[pick], temperature=temperature)
        loss = -(r.log_prob + 0.01 * r.entropy).mean()
        loss.backward()
        ranking.clip_grad_norm([u.grad, v.grad], max_norm)
        U.index_add_(0, users[pick], u.grad, alpha=-rate)
        V.add_(v.grad, alpha=-rate)
        losses.append(loss.detach())
    return torch.stack(losses).tolist()


def rated(w, users):
    """excluded[i, j]: user users[i] has rated item j."""
    out = np.zeros((len(users), w.m), dtype=bool)
    for i, u in enumerate(users):
        out[i, w.cols[w.rows == u]] = True
    return torch.from_numpy(out).cuda()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--config", default="tiny")
    ap.add_argument("--epochs", type=int, default=3)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--batch", type=int, default=4096)
    ap.add_argument("--rate", type=float, default=200.0)
    ap.add_argument("--max-norm", type=float, default=0.05)
    ap.add_argument("--temperature", type=float, default=1.0)
    ap.add_argument("--top", type=int, default=5)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)

    w = make_config(a.config)
    U, V = learn(w, a.epochs)
    liked = w.vals >= np.quantile(w.vals, 0.8)
    users = torch.from_numpy(w.rows[liked].astype(np.int64)).cuda()
    items = torch.from_numpy(w.cols[liked].astype(np.int32)).cuda()
    losses = train_on_choices(U, V, users, items, a.steps, a.batch, a.rate, a.max_norm,
                              a.temperature, a.seed)
    print(f"choices: loss {losses[0]:.4f} -> {losses[-1]:.4f}", flush=True)

    catalogue = ranking.Catalogue(V)
    who = np.arange(min(8, w.n))
    answer = catalogue.rank(U[torch.from_numpy(who).cuda()], top=a.top,
                            temperature=a.temperature, excluded=rated(w, who))
    for i, u in enumerate(who):
        best = ", ".join(f"{j} ({p:.3f})" for j, p in zip(answer.top_item[i].tolist(),
                                                          answer.top_log_prob[i].exp().tolist()))
        print(f"user {u}: entropy {answer.entropy[i].item():.3f}, best items {best}", flush=True)
    return {"losses": losses, "U": U, "V": V, "answer": answer, "who": who, "workload": w}


if __name__ == "__main__":
    main()
