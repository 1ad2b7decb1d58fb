"""The small model learns from the large one: rows of a routed run, then the head, then the small model with that head; and what the losses say of a token that the routing tail
emitted is what the tail's confidence says."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
SEED, B, NEW = 7878, 4, 12


@pytest.fixture(scope="module")
def run():
    from paper_2504_07878_amd import adapt, joint, synth, tokroute
    s = synth.TINY.with_(threshold=0.5)
    big = synth.TINY.with_(name="tiny-large", vocab=s.vocab + 64, router_hidden=0)      # the large model's vocabulary is padded further
    w = synth.make_weights(s, SEED)
    slm = tokroute.Model(s.asdict(), w, B, 64)
    llm = tokroute.Model(big.asdict(), synth.make_weights(big, SEED + 1, std=0.05), B, 64)
    prompts = [synth.prompt_tokens(SEED, f"adapt{b}", 9 + 5 * b, s.vocab) for b in range(B)]
    tokens, routed = joint.generate(slm, llm, prompts, NEW)
    # a large model's padding is never emitted by the small one; here it would have to be
    tokens = np.minimum(tokens, s.vocab - 1)
    rows = adapt.collect(slm, llm, prompts, tokens, top=8)
    return dict(s=s, w=w, slm=slm, llm=llm, prompts=prompts, tokens=tokens, rows=rows)


def test_rows_of_a_routed_run(run):
    hidden, ids, teacher, targets = run["rows"]
    n = B * NEW
    assert hidden.shape == (n, run["s"].d_model) and ids.shape == teacher.shape == (n, 8) and targets.shape == (n,)
    assert np.array_equal(targets.cpu().numpy().reshape(NEW, B).T, run["tokens"])
    assert (teacher[:, :-1] >= teacher[:, 1:]).all() and run["slm"].seq_len(0) == run["llm"].seq_len(0) == len(run["prompts"][0]) + NEW - 1


def test_the_head_learns_the_large_models_answers(run):
    from paper_2504_07878_amd import adapt, tokroute
    hidden, ids, teacher, targets = run["rows"]
    head = run["slm"].dev["tok_emb"]
    new, losses = adapt.adapt_head(head, hidden, ids, teacher, targets, steps=200)
    assert new.shape == head.shape and new.dtype == head.dtype and len(losses) == 200
    assert all(b < a for a, b in zip(losses, losses[1:])), losses       # steps within the losses' curvature only go down
    assert adapt.adapt_head(head, hidden, ids, teacher, targets, steps=0)[1] == []
    # the small model with that head: more of its greedy tokens are the large model's favourites
    weights = {k: v for k, v in run["slm"].dev.items()} | {"lm_head": new}
    model = tokroute.Model(run["s"].with_(tie_lm_head=0).asdict(), weights, B, 64)
    slots, best = list(range(B)), ids[:, 0].cpu().numpy().reshape(NEW, B)

    def agreement(m):
        got = [m.prefill(slots, run["prompts"]).cpu().token] + [m.decode_step(slots, run["tokens"][:, t - 1]).cpu().token for t in range(1, NEW)]
        return float((np.stack(got) == best).mean())

    before, after = agreement(run["slm"]), agreement(model)
    assert after > before, (before, after)


def test_the_tails_confidence_is_the_losses_probability(run):
    """conf = exp(-loss) of the emitted token, on the hidden rows and the head of the tail: both sum 4096 exponentials of 256-term products in fp32, 1e-5 apart at most."""
    from paper_2504_07878_amd import losses
    s, slm = run["s"], run["slm"]
    x = torch.randn((B, s.d_model), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    out = slm.tail(x)
    plan = losses.VocabLoss(B, s.d_model, s.vocab, torch.float32, torch.float32)
    loss, lse = plan.cross_entropy(out.hidden, slm.dev["tok_emb"], out.token)
    assert torch.allclose(torch.exp(-loss), out.conf, rtol=1e-5, atol=0)


def some_rows(n=48, d=256, vocab=500, top=4, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    hidden = torch.randn((n, d), device="cuda", generator=g)
    head = torch.randn((vocab, d), device="cuda", generator=g) * 0.05
    ids = torch.randint(0, vocab, (n, top), device="cuda", generator=g).int()
    teacher = torch.randn((n, top), device="cuda", generator=g)
    return head, hidden, ids, teacher, ids[:, 0].contiguous()


@pytest.mark.parametrize("junk", [0.0, float("nan"), float("inf")])
def test_rows_that_do_not_count_have_no_part_in_the_steps(junk):
    """Three rows of four count for neither loss: the losses of the steps are those of the others alone (the same sums over the same rows, in blocks of other sizes: fp32 roundings of
    losses of about 6, 100 u of them, over steps that bring them closer together)."""
    from paper_2504_07878_amd import adapt
    head, hidden, ids, teacher, targets = some_rows()
    off = torch.arange(48, device="cuda") % 4 > 0
    want = adapt.adapt_head(head, hidden[~off], ids[~off], teacher[~off], targets[~off], steps=30)
    hidden[off], ids[off], targets[off] = junk, -1, -1
    got = adapt.adapt_head(head, hidden, ids, teacher, targets, steps=30)
    assert np.allclose(got[1], want[1], rtol=1e-5, atol=0), (got[1], want[1])
    assert all(b < a for a, b in zip(got[1], got[1][1:])) and torch.allclose(got[0], want[0], rtol=1e-4, atol=1e-6)


def test_rows_without_a_teachers_logits_do_not_count():
    """Logits of -inf are no entries: a row of nothing else counts like one without ids, and each loss is a mean over its own rows."""
    from paper_2504_07878_amd import adapt
    head, hidden, ids, teacher, targets = some_rows()
    none = ids.clone()
    none[::3] = -1
    want = adapt.adapt_head(head, hidden, none, teacher, targets, steps=10)
    teacher[::3] = float("-inf")
    got = adapt.adapt_head(head, hidden, ids, teacher, targets, steps=10)
    assert torch.equal(got[0], want[0]) and got[1] == want[1]


def test_no_row_counts():
    from paper_2504_07878_amd import adapt
    head, hidden, ids, teacher, targets = some_rows()
    new, losses = adapt.adapt_head(head, hidden, ids.fill_(-1), teacher, targets.fill_(-1), steps=3)
    assert torch.equal(new, head) and losses == [0.0] * 3


def test_targets_past_the_vocabulary_do_not_count():
    """Tokens of the large model's longer vocabulary: no target for this head, and no NaN in the steps' losses."""
    from paper_2504_07878_amd import adapt
    head, hidden, ids, teacher, targets = some_rows()
    targets[::5] = -1
    want = adapt.adapt_head(head, hidden, ids, teacher, targets, steps=10)
    targets[::5] = torch.tensor([500, 501, 2 ** 31 - 1, 500, 563, 500, 500, 777, 500, 500], dtype=torch.int32, device="cuda")
    given = targets.clone()
    got = adapt.adapt_head(head, hidden, ids, teacher, targets, steps=10)
    assert torch.equal(got[0], want[0]) and got[1] == want[1] and torch.equal(targets, given)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_parameter_as_the_head_and_no_grad_around_it(dtype):
    """The head may be a parameter of the caller's, the rows part of a graph, gradients switched off: the same steps, and no gradient left with the caller."""
    from paper_2504_07878_amd import adapt
    head, hidden, ids, teacher, targets = some_rows()
    head = head.to(dtype)
    want = adapt.adapt_head(head, hidden, ids, teacher, targets, steps=5)
    p, rows = torch.nn.Parameter(head.clone()), hidden.clone().requires_grad_()
    for mode in (torch.enable_grad, torch.no_grad):
        with mode():
            got = adapt.adapt_head(p, rows, ids, teacher, targets, steps=5)
        assert torch.equal(got[0], want[0]) and got[1] == want[1] and not got[0].requires_grad
        assert p.grad is None and rows.grad is None and torch.equal(p.detach(), head)


def test_a_bf16_models_head_learns():
    """The rows that a bf16 model exposes are fp32, over a bf16 head."""
    from paper_2504_07878_amd import adapt, joint, synth, tokroute
    s = synth.TINY.with_(name="tiny-bf16", dtype=synth.BF16, kv_dtype=synth.BF16, threshold=0.5)
    slm = tokroute.Model(s.asdict(), synth.make_weights(s, SEED), B, 64)
    llm = tokroute.Model(s.with_(router_hidden=0).asdict(), synth.make_weights(s.with_(router_hidden=0), SEED + 1, std=0.05), B, 64)
    prompts = [synth.prompt_tokens(SEED, f"adapt{b}", 9 + 5 * b, s.vocab) for b in range(B)]
    tokens, _ = joint.generate(slm, llm, prompts, NEW)
    hidden, ids, teacher, targets = adapt.collect(slm, llm, prompts, tokens, top=8)
    head = slm.dev["tok_emb"]
    assert hidden.dtype == torch.float32 and head.dtype == torch.bfloat16
    new, losses = adapt.adapt_head(head, hidden, ids, teacher, targets, steps=100)
    _, same = adapt.adapt_head(head.float(), hidden, ids, teacher, targets, steps=1)
    assert abs(losses[0] - same[0]) < 1e-5 * same[0]            # the same head, and losses of the same precision
    assert new.dtype == torch.bfloat16 and losses[-1] < losses[50] < losses[0]
