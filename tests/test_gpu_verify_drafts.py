"""Verification of drafted tokens against the request-by-request reference:
tokens and counts equal."""
import numpy as np
import pytest

from tests import decode_ref as ref

pytestmark = pytest.mark.gpu


def _softmax(x):
    e = np.exp(x - x.max(-1, keepdims=True))
    return e / e.sum(-1, keepdims=True)


def _inputs(seed, B, K, V, dtype, near=0.7):
    """Probabilities rounded to the type, held as 32-bit numbers; a draft is drawn from its own distribution."""
    import torch
    rng = np.random.RandomState(seed)
    logits = 2.0 * rng.standard_normal((B, K + 1, V))
    ty = getattr(torch, dtype)
    def held(x):
        return torch.from_numpy(x.astype(np.float32)).to(ty).float().numpy()
    target = held(_softmax(logits))
    draft = held(_softmax(logits[:, :K] + near * rng.standard_normal((B, K, V))))
    tokens = (draft / rng.exponential(1, draft.shape)).argmax(-1).astype(np.int32) if K else np.zeros((B, 0), np.int32)
    n = rng.randint(-1, K + 1, B).astype(np.int32)
    u = rng.rand(B, K).astype(np.float32)
    noise = rng.exponential(1, (B, V)).astype(np.float32)
    return target, draft, tokens, n, u, noise, ty


def _run(target, draft, tokens, n, u, noise, ty):
    import torch

    import paper_2609_15359_amd as maps
    c = lambda x, t=None: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(t).cuda()  # noqa: E731
    err = maps.new_error_word()
    out, accepted = maps.verify_drafts(c(target, ty), c(tokens), c(n), c(u), c(noise), draft=c(draft, ty), dev_err=err)
    torch.cuda.synchronize()
    return out.cpu().numpy(), accepted.cpu().numpy(), maps.error_names(int(err.item()))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("B,K,V", [(1, 1, 1), (3, 0, 50), (9, 3, 1), (40, 4, 333), (5, 2, 8192), (5, 2, 8193), (3, 64, 100),
                                   (33, 5, 20001), (300, 3, 1000)])
@pytest.mark.parametrize("with_draft", [True, False])
def test_matches_the_reference(B, K, V, dtype, with_draft):
    *x, ty = _inputs(B * 7 + K, B, K, V, dtype)
    if not with_draft:
        x[1] = None
    tokens, accepted, err = _run(*x, ty)
    want, want_accepted = ref.verify(*x)
    assert err == []
    assert np.array_equal(accepted, want_accepted) and np.array_equal(tokens, want)


def test_equal_distributions_accept_everything():
    *x, ty = _inputs(1, 50, 6, 500, "float32", near=0.0)
    x[1] = x[0][:, :6].copy()
    tokens, accepted, err = _run(*x, ty)
    assert err == [] and np.array_equal(accepted, x[3])


def test_ties_go_to_the_lowest_token():
    B, K, V = 4, 1, 30000
    target = np.full((B, K + 1, V), 1 / V, np.float32)
    draft = np.zeros((B, K, V), np.float32)
    draft[:, :, 0] = 1.0
    x = [target, draft, np.zeros((B, K), np.int32), np.array([0, 1, 1, 0], np.int32), np.full((B, K), 0.9, np.float32),
         np.ones((B, V), np.float32)]
    import torch
    tokens, accepted, err = _run(*x, torch.float32)
    assert err == [] and accepted.tolist() == [0, 0, 0, 0]
    assert tokens.tolist() == [[0, -1], [1, -1], [1, -1], [0, -1]]      # refused: token 0 has nothing left


def test_nothing_left_falls_back_to_the_target():
    """A draft that is above the target everywhere (as rounded probabilities can be) leaves the target's own race."""
    *x, ty = _inputs(2, 20, 2, 400, "float32")
    x[1] = np.maximum(x[1], x[0][:, :2]) * np.float32(1.5)
    x[4][:] = 0.999
    tokens, accepted, err = _run(*x, ty)
    want, want_accepted = ref.verify(*x)
    assert err == [] and np.array_equal(tokens, want) and np.array_equal(accepted, want_accepted)


def test_special_numbers():
    """No noise, zero, subnormal and NaN probabilities."""
    *x, ty = _inputs(3, 12, 1, 700, "float32")
    x[3][:] = 0
    x[0][0] = 0.0
    x[0][0, :, 37] = 1e-42
    x[0][1, :, ::2] = np.nan
    x[5][2, 5:9] = 0.0                       # an infinite score: the first of them
    tokens, accepted, err = _run(*x, ty)
    assert err == [] and tokens[0, 0] == 37 and tokens[1, 0] % 2 == 1 and tokens[2, 0] == 5
    want, _ = ref.verify(*[None if a is None else a[3:] for a in x])
    assert np.array_equal(tokens[3:], want)


def test_frequencies_follow_the_target():
    """One drafted token, 20,000 independent requests over 6 tokens: the first output token has the target's
    distribution.  Each count is binomial: 5 standard deviations."""
    import torch
    rng = np.random.RandomState(8)
    B, V = 20000, 6
    p, q = np.array([.3, .25, .2, .15, .07, .03], np.float32), np.array([.05, .1, .15, .2, .2, .3], np.float32)
    tokens = rng.choice(V, (B, 1), p=q / q.sum(dtype=np.float64)).astype(np.int32)
    out, accepted, err = _run(np.broadcast_to(p, (B, 2, V)), np.broadcast_to(q, (B, 1, V)), tokens, np.ones(B, np.int32),
                              rng.rand(B, 1).astype(np.float32), rng.exponential(1, (B, V)).astype(np.float32),
                              torch.float32)
    assert err == []
    count = np.bincount(out[:, 0], minlength=V)
    assert (np.abs(count - B * p) < 5 * np.sqrt(B * p * (1 - p))).all(), count


def test_views():
    import torch

    import paper_2609_15359_amd as maps
    target, draft, tokens, n, u, noise, ty = _inputs(5, 10, 3, 999, "bfloat16")
    want, want_accepted = ref.verify(target, draft, tokens, n, u, noise)
    c = lambda x, t=None: torch.from_numpy(np.ascontiguousarray(x)).to(t).cuda()  # noqa: E731
    wide = torch.full((4, 10, 1024), 9.0, dtype=ty, device="cuda")               # drafts before requests, padded rows
    wide[:, :, 3:1002] = c(target, ty).transpose(0, 1)
    wide_draft = torch.full((10, 3, 1001), 9.0, dtype=ty, device="cuda")
    wide_draft[:, :, :999] = c(draft, ty)
    wide_noise = torch.full((10, 1111), 9.0, device="cuda")
    wide_noise[:, 1:1000] = c(noise)
    out, accepted = maps.verify_drafts(wide[:, :, 3:1002].transpose(0, 1), c(tokens), c(n), c(u), wide_noise[:, 1:1000],
                                       draft=wide_draft[:, :, :999])
    assert np.array_equal(out.cpu().numpy(), want) and np.array_equal(accepted.cpu().numpy(), want_accepted)


@pytest.mark.parametrize("with_draft", [True, False])
def test_no_requests(with_draft):
    import torch

    import paper_2609_15359_amd as maps
    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")
    tokens, accepted = maps.verify_drafts(empty(0, 4, 50), empty(0, 3, dtype=torch.int32), empty(0, dtype=torch.int32),
                                          empty(0, 3), empty(0, 50), draft=empty(0, 3, 50) if with_draft else None)
    assert tokens.shape == (0, 4) and accepted.shape == (0,) and tokens.dtype == accepted.dtype == torch.int32


def test_value_errors():
    *x, ty = _inputs(6, 6, 2, 50, "float32")
    x[3][:] = 2
    for name, at, value in (("token", 2, 50), ("token", 2, -1), ("count", 3, 3), ("count", 3, -2)):
        y = [a.copy() for a in x]
        y[at][1] = value
        assert _run(*y, ty)[2] == ["DRAFT"], (name, value)
    y = [a.copy() for a in x]
    y[0][3] = 0.0
    tokens, accepted, err = _run(*y, ty)
    assert err == ["DRAFT"] and tokens[3].tolist() == [-1, -1, -1]
