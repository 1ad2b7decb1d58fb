"""The small model learns from the large one (host control flow over the ABI, like joint.py).

What the routing loop asks the large model for is what the small model could not do: the tokens it emitted instead, and its logits around them. `collect` runs both models
over sequences that `joint.generate` produced and keeps, for every generated position, the small model's exposed hidden row (Section 3.3) and the large model's
top logits; `adapt_head` fits the small model's LM head to them with the losses of `losses.py`: distillation from the top logits and cross entropy of the emitted tokens.
The head that comes back replaces `lm_head` of the small model's weights in a new context (tie_lm_head = 0: the embedding stays as it is).
"""
from __future__ import annotations

import numpy as np
import torch

from . import losses
from .tokroute import POST_FINAL_NORM


def collect(slm, llm, prompts, tokens, top: int = 16):
    """One row for every generated position of every sequence: (hidden float32 [n][d], ids int32 [n][top], teacher float32 [n][top], targets int32 [n]).

    prompts: the sequences' prompts; tokens: int32 [B][max_new], what they emitted. ids at or past the small model's vocabulary (a large model's padding) are no entries of
    the losses. slm exposes the rows that its LM head multiplies (hidden_tap POST_FINAL_NORM): others are refused. Both models' slots 0 .. B - 1 are used, and hold the sequences afterwards.
    """
    if slm.cfg.hidden_tap != POST_FINAL_NORM:
        raise ValueError("the small model exposes hidden rows before the final norm: its LM head does not multiply them")
    slots = list(range(len(prompts)))
    keep = ([], [], [], [])

    def take(small, large, targets):
        value, index = large.logits.topk(top, 1)
        for to, x in zip(keep, (small.hidden, index.int(), value, torch.from_numpy(np.ascontiguousarray(targets, dtype=np.int32)).to(value.device))):
            to.append(x)

    take(slm.prefill(slots, prompts), llm.prefill(slots, prompts, want_logits=True), tokens[:, 0])
    for t in range(1, tokens.shape[1]):
        take(slm.decode_step(slots, tokens[:, t - 1]), llm.decode_step(slots, tokens[:, t - 1], want_logits=True), tokens[:, t])
    return tuple(torch.cat(x) for x in keep)


def adapt_head(head, hidden, ids, teacher, targets, steps: int = 20, rate: float = None, share: float = 0.5, temperature: float = 2.0):
    """Gradient descent on the LM head [vocab][d] (float32 or bfloat16): `share` of the loss is distillation, the rest cross entropy, both means over the rows that count.

    hidden: float32 as `collect` gives them, or bfloat16, with which the gradients over a bfloat16 head run on bf16 matrix instructions, several times as fast.
    rate: None takes 1 / (mean |hidden|^2 / 2), each loss's mean over its own rows that count, by its share: the inverse of a bound on the curvature of the loss in the head (a softmax's second
    derivative is at most 1/2; T^2 makes up for 1/T twice), with which every step of a float32 head goes down (a bfloat16 head's too, but for its rounding). Rows that do not count for a loss (as
    the losses have it) have no part in any of this, whatever they hold; nor have targets past the head's vocabulary, tokens that only the large model has. Returns (new head in the head's type, losses of the steps as a list of floats). Updates are kept in fp32.
    """
    head, hidden = head.detach(), hidden.detach()          # (steps of its own, whatever graph they come from)
    plan = losses.VocabLoss(hidden.shape[0], head.shape[1], head.shape[0], hidden.dtype, head.dtype, max_entries=ids.shape[1], device=head.device)
    master, value = head.float().clone(), []
    targets = targets.where(targets < head.shape[0], torch.full_like(targets, -1))
    count_ce, count_kd = targets >= 0, ((ids >= 0) & (ids < head.shape[0]) & (teacher != float("-inf"))).any(1)
    n_ce, n_kd = max(1, int(count_ce.sum())), max(1, int(count_kd.sum()))
    if rate is None:
        square = hidden.float().square().sum(1)
        mean_ce, mean_kd = (float(square.where(on, torch.zeros_like(square)).sum()) / n for on, n in ((count_ce, n_ce), (count_kd, n_kd)))
        curvature = (share * mean_kd + (1 - share) * mean_ce) / 2
        rate = 1.0 / curvature if curvature else 0.0        # (no row that counts, or rows of zeros: no gradient either)
    for _ in range(steps):
        w = master.to(head.dtype, copy=True).requires_grad_()
        with torch.enable_grad():
            loss = share / n_kd * losses.distill(plan, hidden, w, ids, teacher, temperature).sum() + (1 - share) / n_ce * losses.cross_entropy(plan, hidden, w, targets).sum()
        loss.backward()
        master -= rate * w.grad.float()
        value.append(loss.detach())
    return master.to(head.dtype), torch.stack(value).tolist() if value else []
