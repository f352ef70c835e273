"""From ratings to recommendations in one run: ALS iterations on a synthetic workload (driver.run), the items'
factors to 8 bits, then batches of users who are each drawn one item that they have not rated.

    python -m paper_1603_03820_amd.recommend [--workload tiny] [--iters 5] [--batch 256] [--temperature 0.2]
        [--top-k 50] [--top-p 0.9] [--evaluate [--steps 20]]

With --evaluate a tenth of the ratings is held out of the training instead, and the model says how probable it finds those
items: the mean log probability of a held-out item among those that its user has not rated, the entropy of the user's
distribution, and how many of the items are among its best 20; before and after the items' offsets are fitted to half of
the users.

Run it from the repository's root, as the workloads are those of its ``synth`` package."""
from __future__ import annotations

import argparse
import time

import torch

from . import als, driver, serve


def run(workload: str = "tiny", iters: int = 5, batch: int = 256, temperature: float = 0.2, top_k: int = 50,
        top_p: float = 0.9, seed: int = 1, device: int = 0):
    """(training RMSE per iteration, items int32 [m], log probabilities [m], seconds of the draws): one item for
    every user of the workload."""
    import synth
    p = synth.config(workload)
    ctx = als.Context(device, p.f)
    dp = driver.DeviceProblem.from_host_csr(ctx, p.m, p.n, p.f, p.lam, p.rowptr, p.colidx, p.vals)
    x, theta, rmse = driver.train(ctx, dp, torch.from_numpy(p.theta0).to(ctx.device), iters)
    answers = serve.Recommender(serve.Context(device), x, theta, rated=(dp.rowptr, dp.colidx))
    gen = torch.Generator(device=ctx.device).manual_seed(seed)
    u = torch.rand(p.m, device=ctx.device, generator=gen)
    users = torch.arange(p.m, dtype=torch.int32, device=ctx.device)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    drawn = [answers.recommend(users[k:k + batch], u[k:k + batch], temperature, top_k, top_p)
             for k in range(0, p.m, batch)]
    items, log = (torch.cat(part) for part in zip(*drawn))
    torch.cuda.synchronize()
    return rmse, items, log, time.perf_counter() - t0


def evaluate(workload: str = "tiny", iters: int = 5, batch: int = 256, temperature: float = 0.2, top: int = 20,
             steps: int = 20, held: float = 0.1, device: int = 0):
    """(before, after, means): of the held-out items of every second user, a dict of their mean log probability
    ("log_prob"), their users' mean entropy ("entropy") and the share of them among their users' `top` best ("hits"), before
    and after `steps` steps of fitting the items' offsets to the other users' held-out items, and the mean log probability
    of those before each step."""
    import synth
    from . import predict
    p = synth.config(workload)
    train, test = synth.split(p.rowptr, p.colidx, p.vals, held, p.recipe["seed"])
    ctx = als.Context(device, p.f)
    dp = driver.DeviceProblem.from_host_csr(ctx, p.m, p.n, p.f, p.lam, *train)
    x, theta, _ = driver.train(ctx, dp, torch.from_numpy(p.theta0).to(ctx.device), iters)
    model = predict.Predictor(predict.Context(device), x, theta, rated=(dp.rowptr, dp.colidx))
    ptr, items = (torch.from_numpy(a).to(ctx.device) for a in test[:2])
    users = torch.arange(p.m, dtype=torch.int32, device=ctx.device)
    of = torch.repeat_interleave(users, torch.diff(ptr))
    second = of % 2 == 1

    def measure():
        log, entropy, hits = torch.empty(items.numel(), device=ctx.device), [], []
        for k in range(0, p.m, batch):
            some = users[k:k + batch]
            r = model.log_prob(some, (ptr[k:k + some.numel() + 1].contiguous(), items), temperature, top, log=log)
            entropy.append(r.entropy)
            first, end = int(ptr[k]), int(ptr[k + some.numel()])
            best = r.top_index[(of[first:end] - k).long()]
            hits.append((best == items[first:end, None]).any(1))
        counted = second & (log > float("-inf"))
        return dict(log_prob=log[counted].double().mean().item(), entropy=torch.cat(entropy)[1::2].double().mean().item(),
                    hits=torch.cat(hits)[counted].double().mean().item())
    before = measure()
    means = model.fit_offsets(of[~second].contiguous(), items[~second].contiguous(), temperature, steps, batch=max(batch, 1024))
    return before, measure(), means


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workload", default="tiny")
    ap.add_argument("--iters", type=int, default=5)
    ap.add_argument("--batch", type=int, default=256)
    ap.add_argument("--temperature", type=float, default=0.2)
    ap.add_argument("--top-k", type=int, default=50)
    ap.add_argument("--top-p", type=float, default=0.9)
    ap.add_argument("--evaluate", action="store_true", help="how probable held-out items are, in place of drawing any")
    ap.add_argument("--steps", type=int, default=20, help="of fitting the items' offsets (with --evaluate)")
    args = ap.parse_args()
    if args.evaluate:
        before, after, means = evaluate(args.workload, args.iters, args.batch, args.temperature, steps=args.steps)
        for name, r in (("before", before), ("after", after)):
            print(f"{name} fitting the offsets: held-out items' mean log probability {r['log_prob']:.3f}, entropy "
                  f"{r['entropy']:.3f}, among the best 20 {100 * r['hits']:.1f}%")
        if means:
            print(f"of those fitted to: {means[0]:.3f} before the first step, {means[-1]:.3f} before the last")
        return
    rmse, items, log, seconds = run(args.workload, args.iters, args.batch, args.temperature, args.top_k, args.top_p)
    print(f"training RMSE {', '.join(f'{r:.4f}' for r in rmse)}")
    print(f"{items.numel()} users in {seconds * 1e3:.2f} ms, {items.unique().numel()} items, "
          f"mean log probability {log.mean().item():.3f}")
    for user in range(min(5, items.numel())):
        print(f"user {user}: item {items[user].item()}")


if __name__ == "__main__":
    main()
