"""From ratings to rankings, on one MI355X.

1. Learn factors U, V from ratings with the blocked SGD sweep (bgmf.Model).
2. Train them further on choices: the softmax over the catalogue of the items
   that users rated highly, its gradient, clipped by the global norm.
3. Optionally, learn from feedback: the policy that a 4-bit catalogue serves
   shows items, users accept or reject them, and the factors are trained on the
   clipped policy loss of the shown items, held near where they started, with
   dropout on the users' factors.
4. Answer requests: the item factors in 8-bit integers (or 4 bits), laid out
   once; per request the user's scores over the whole catalogue, and the best
   items among those the user has not rated, with their log probabilities.

    python examples/rank_items.py [--epochs 3] [--steps 300] [--batch 4096]
                                  [--feedback 20] [--dropout 0.1] [--bits 4]
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


def show(catalogue, users, temperature, generator):
    """One item for each user, drawn from the policy that the catalogue serves, and
    its log probability."""
    scores = catalogue.scores(users)
    noise = -torch.empty_like(scores).exponential_(generator=generator).log()
    items = (scores / temperature + noise).argmax(1).int()
    return items, ranking.log_probs(scores, items, temperature=temperature).log_prob


def feedback_step(u, v, frozen, shown, old_log_prob, advantage, kl_weight, temperature, dropout,
                  seed, offset):
    """The clipped policy loss of shown items and its gradients with respect to the
    users' and the items' factors; frozen: both sides' factors before training."""
    u, v = u.detach().requires_grad_(), v.detach().requires_grad_()
    scores = ranking.dropout(u, dropout, seed, offset) @ v.t()
    reference = frozen[0] @ frozen[1].t()
    r = ranking.policy_loss(scores, shown, advantage, old_log_prob, reference=reference,
                            kl_weight=kl_weight, temperature=temperature)
    r.loss.mean().backward()
    return r, u.grad, v.grad


def train_on_feedback(U, V, taste, steps, batch, rate, max_norm, temperature, dropout, seed):
    """Rounds of showing items and learning from what users did with them, in place.
    taste(users, items) -> how much each liked what it was shown."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    U0, V0 = U.clone(), V.clone()
    rewards = []
    for step in range(steps):
        catalogue = ranking.Catalogue(V, bits=4)
        who = torch.randint(0, U.shape[0], (batch,), generator=g, device="cuda")
        shown, old = show(catalogue, U[who], temperature, g)
        reward = taste(who, shown)
        _, gu, gv = feedback_step(U[who], V, (U0[who], V0), shown, old, reward - reward.mean(),
                                  0.05, temperature, dropout, seed, step * batch * U.shape[1])
        ranking.clip_grad_norm([gu, gv], max_norm)
        U.index_add_(0, who, gu, alpha=-rate)
        V.add_(gv, alpha=-rate)
        rewards.append(reward.mean())
    return torch.stack(rewards).tolist() if rewards else []


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
    ap.add_argument("--feedback", type=int, default=0, help="rounds of feedback")
    ap.add_argument("--dropout", type=float, default=0.1, help="during feedback")
    ap.add_argument("--bits", type=int, default=8, choices=(4, 8), help="of the catalogue served")
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

    rewards = []
    if a.feedback:
        u_liked, v_liked = U.clone(), V.clone()  # users keep the taste learned so far
        rewards = train_on_feedback(U, V, lambda u, j: (u_liked[u] * v_liked[j.long()]).sum(1),
                                    a.feedback, a.batch, a.rate, a.max_norm, a.temperature,
                                    a.dropout, a.seed)
        print(f"feedback: mean reward {rewards[0]:.4f} -> {rewards[-1]:.4f}", flush=True)

    catalogue = ranking.Catalogue(V, bits=a.bits)
    who = np.arange(min(8, w.n))
    answer = catalogue.rank(U[torch.from_numpy(who).cuda()], top=a.top,
                            temperature=a.temperature, excluded=rated(w, who))
    for i, u in enumerate(who):
        best = ", ".join(f"{j} ({p:.3f})" for j, p in zip(answer.top_item[i].tolist(),
                                                          answer.top_log_prob[i].exp().tolist()))
        print(f"user {u}: entropy {answer.entropy[i].item():.3f}, best items {best}", flush=True)
    return {"losses": losses, "rewards": rewards, "U": U, "V": V, "answer": answer, "who": who,
            "workload": w}


if __name__ == "__main__":
    main()
