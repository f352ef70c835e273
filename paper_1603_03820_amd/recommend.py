"""From ratings to recommendations in one run: ALS iterations on a synthetic workload (driver.run), the items'
factors to 8 bits, then batches of users who are each drawn one item that they have not rated.

    python -m paper_1603_03820_amd.recommend [--workload tiny] [--iters 5] [--batch 256] [--temperature 0.2]
        [--top-k 50] [--top-p 0.9]

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


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workload", default="tiny")
    ap.add_argument("--iters", type=int, default=5)
    ap.add_argument("--batch", type=int, default=256)
    ap.add_argument("--temperature", type=float, default=0.2)
    ap.add_argument("--top-k", type=int, default=50)
    ap.add_argument("--top-p", type=float, default=0.9)
    args = ap.parse_args()
    rmse, items, log, seconds = run(args.workload, args.iters, args.batch, args.temperature, args.top_k, args.top_p)
    print(f"training RMSE {', '.join(f'{r:.4f}' for r in rmse)}")
    print(f"{items.numel()} users in {seconds * 1e3:.2f} ms, {items.unique().numel()} items, "
          f"mean log probability {log.mean().item():.3f}")
    for user in range(min(5, items.numel())):
        print(f"user {user}: item {items[user].item()}")


if __name__ == "__main__":
    main()
