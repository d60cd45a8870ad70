"""The serving loop of the example against its model in 64 bits: with a temperature near 0 every token of an answer is
the model's first choice after the tokens before it, whatever was drafted.

Margin.  An attention output of bf16 is off by at most u |out| + (u + 2 e + 2^-18) sum p|v| <= 3 u sum p|v|, with
u = 2^-8 and e the scores' error, of which 2 e + 2^-18 < u is asserted; a logit is then off by at most M = (3 u +
512 2^-23) sum p|v| |proj|, and the chosen token is below the first by at most both tokens' M and 60 temperatures,
which a race of 500 exponential numbers bridges with a probability below 1e-20."""
import numpy as np
import pytest

from tests import decode_ref as ref

pytestmark = pytest.mark.gpu


def _below_first(model, prompt, answer):
    """How far each answered token's logit is below the largest, and the margin, in 64 bits."""
    q, k, v, proj = (x.double().cpu().numpy() for x in (model.q, model.k, model.v, model.proj))
    tokens = np.array(prompt + answer[:-1])
    kk, vv = ref.dequantise(*ref.quantise(k[tokens])), ref.dequantise(*ref.quantise(v[tokens]))
    G, gaps = q.shape[1] // k.shape[1], []
    for i, x in enumerate(answer):
        n = len(prompt) + i
        out, mag = [], []
        for hq in range(q.shape[1]):
            x_q, keys = q[tokens[n - 1], hq], kk[:n, hq // G]
            e = model.scale * (64 * 2.0 ** -23 * (np.abs(keys) @ np.abs(x_q)).max() +
                               2.0 ** -20 * np.abs(x_q).max() * np.abs(keys).sum(1).max())
            assert 2 * e + 2.0 ** -18 < 2.0 ** -8
            s = keys @ x_q * model.scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out.append(p @ vv[:n, hq // G])
            mag.append(p @ np.abs(vv[:n, hq // G]))
        logits = np.concatenate(out) @ proj
        M = (3 * 2.0 ** -8 + 512 * 2.0 ** -23) * (np.concatenate(mag) @ np.abs(proj))
        first = logits.argmax()
        gaps.append((logits[first] - logits[x], M[first] + M[x] + 60 * model.temperature))
    return np.array(gaps)


@pytest.mark.parametrize("drafts", [0, 1, 4])
def test_answers_are_the_models_first_choices(drafts):
    from examples.decode_loop import Model, serve
    model = Model.random(vocab=500, temperature=1e-3, seed=3)
    rng = np.random.RandomState(8)
    prompts = [rng.randint(0, 500, n).tolist() for n in (1, 17, 70, 3)]
    answers, steps = serve(model, prompts, 40, drafts, 1 << 19)
    assert [len(a) for a in answers] == [40] * 4
    assert steps <= 40
    for prompt, answer in zip(prompts, answers):
        gaps = _below_first(model, prompt, answer)
        assert (gaps[:, 0] <= gaps[:, 1]).all(), gaps[gaps[:, 0] > gaps[:, 1]]


def test_a_cache_that_is_too_small_is_refused():
    from examples.decode_loop import Model, serve
    with pytest.raises(ValueError, match="too small"):
        serve(Model.random(), [[1, 2, 3]], 40, 2, 1 << 10)


@pytest.mark.parametrize("drafts", [0, 1, 4])
def test_accepted_drafts_save_steps(drafts):
    """A model whose token x is always followed by x + 1 mod 5: a query is twice its token's key (entries of 1 and -1), so
    that attention gives that token's value, and the projection takes it to the next token.  Once the drafter has seen the
    five pairs, after at most five steps, every draft is accepted and a step gives drafts + 1 tokens."""
    import torch

    from examples.decode_loop import Model, serve
    V, H, G, D = 5, 2, 2, 64
    g = torch.Generator().manual_seed(5)
    def signs():
        return 2.0 * torch.randint(0, 2, (V, H, D), generator=g) - 1.0
    k, v = signs(), signs()
    proj = v.roll(1, 0).repeat_interleave(G, 1).flatten(1).T                  # column y: the value of token y - 1
    bf16 = dict(device="cuda", dtype=torch.bfloat16)
    model = Model(q=(2 * k).repeat_interleave(G, 1).to(**bf16), k=k.to(**bf16), v=v.to(**bf16),
                  proj=proj.contiguous().cuda(), temperature=1.0)
    prompts = [[0], [3, 1, 1, 4], [2] * 33]
    answers, steps = serve(model, prompts, 40, drafts, 1 << 19)
    assert answers == [[(p[-1] + 1 + i) % V for i in range(40)] for p in prompts]
    if drafts:
        assert steps <= 1 + V + -(-39 // (drafts + 1))
    else:
        assert steps == 40
