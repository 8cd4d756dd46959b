"""Several tenants' policies trained at once on one adapted output projection, with the library's calls alone between the
hidden states and the committed adapters (Algorithm 1: rollout, policy update, commit; Experimental setup: GRPO).

Every tenant's task is a toy with a verifiable reward: of `vocabulary` tokens, those congruent to the tenant's number are
right.  The policy is softmax(x (W + s A_t B_t)) over features x of the prompt, an eighth of them the same for all prompts
(what a tenant's task has in common); the base weight W is frozen and shared, each tenant's adapter starts at B = 0.  One
iteration:

    rollout    logits of the mixed batch (marlaas_lora_forward), sampled tokens, their log-probabilities under the behaviour
               policy (marlaas_token_logprobs), rewards of each answer
    training   group-relative advantages and token weights (marlaas_group_advantages); per epoch: the logits of the current
               policy, the clipped loss whose gradient replaces the logits in place (marlaas_policy_loss), dA and dB
               (marlaas_lora_backward), AdamW with 8-bit moments and commit (marlaas_adapter_pool_adamw_compact_commit)

    python examples/policy_update.py [iterations]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_08527_b200 import binding as B  # noqa: E402


def run(iterations=12, tenants=4, prompts=8, answers=8, length=6, width=256, vocabulary=256, rank=8, epochs=2, seed=0,
        verbose=True):
    """Mean reward per tenant and iteration, [iterations][tenants], and the last iteration's stats of the loss."""
    dev = "cuda:0"
    torch.manual_seed(seed)
    pool = B.AdapterPool(width, vocabulary, rank, tenants)
    W = (0.5 / width ** 0.5 * torch.randn(width, vocabulary, device=dev)).bfloat16()
    A = [torch.randn(width, rank, device=dev) / width ** 0.5 for _ in range(tenants)]
    Bm = [torch.zeros(rank, vocabulary, device=dev) for _ in range(tenants)]
    dA, dB = [torch.empty_like(a) for a in A], [torch.empty_like(b) for b in Bm]
    for t in range(tenants):
        B.marlaas_adapter_pool_register(pool, t, 0, rank, 2.0 * rank, A[t].bfloat16(), Bm[t].bfloat16())
    states = [B.compact_state(pool, rank) for _ in range(tenants)]
    tables = B.CompactAdamWTables(pool, range(tenants), dA, dB, A, Bm, [s[0] for s in states], [s[1] for s in states])

    # a sequence per answer, the answers to one prompt side by side, a tenant's prompts side by side
    S = tenants * prompts * answers
    T = S * length
    i32 = dict(dtype=torch.int32, device=dev)
    slot = torch.arange(tenants, **i32).repeat_interleave(prompts * answers)
    seg = B.Segments(torch.arange(0, T + 1, length, **i32), slot)
    groups = torch.arange(0, S + 1, answers, **i32)
    wanted = slot.repeat_interleave(length)
    common = torch.randn(width // 8, device=dev)
    history, step, stats = [], 0, None
    for it in range(iterations):
        prompt = torch.randn(S // answers, width, device=dev).repeat_interleave(answers * length, 0)
        x = prompt + 0.5 * torch.randn(T, width, device=dev)
        x[:, :width // 8] = common
        x = x.bfloat16()
        # ---- rollout ----
        logits = B.marlaas_lora_forward(pool, x, W, seg)
        tokens = torch.multinomial(torch.softmax(logits.float(), 1), 1)[:, 0].int()
        old = B.marlaas_token_logprobs(pool, logits, tokens)
        rewards = (tokens % tenants == wanted).float().view(S, length).mean(1)
        history.append(rewards.view(tenants, -1).mean(1).tolist())
        # ---- policy update ----
        targets = tokens.clone()
        targets.view(S, length)[:, 0] = -1          # the first position stands for the prompt: nothing to learn there
        _, adv, weight = B.marlaas_group_advantages(pool, seg, rewards, groups, targets)
        for _ in range(epochs):
            step += 1
            h = torch.empty(T, pool.rank_stride, device=dev)
            logits = B.marlaas_lora_forward(pool, x, W, seg, h_save=h)
            stats = B.marlaas_policy_loss(pool, logits, targets, seg, old, adv, weight, ref_logp=old, dlogits=logits,
                                          clip_low=0.2, clip_high=0.28, kl_coef=0.02)
            B.marlaas_lora_backward(pool, x, W, logits, seg, dA=dA, dB=dB, h_saved=h)
            B.marlaas_adapter_pool_adamw_compact_commit(pool, tables, lr=2e-2, beta2=0.99, step=step, seed=seed)
        if verbose:
            s = stats.cpu()
            print(f"iteration {it:2d}  reward " + " ".join(f"{r:.3f}" for r in history[-1]) +
                  f"  loss {s[:tenants, 0].mean():+.4f}  kl {s[:tenants, 2].mean():.4f}  clipped {s[:tenants, 5].mean():.3f}")
    B.marlaas_check_status(pool)
    return history, stats, pool


if __name__ == "__main__":
    run(int(sys.argv[1]) if len(sys.argv) > 1 else 12)
