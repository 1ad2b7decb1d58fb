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
