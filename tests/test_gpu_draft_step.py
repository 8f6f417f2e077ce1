"""The example of a step with drafted tokens: its decisions against whole-number arithmetic, its probabilities against the
model computed anew over the whole text in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import step_oracle as S

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "draft_step.py")


def _example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("draft_step", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _logits(X, model, text):
    """Of every token of a text, without a cache."""
    w = {k: v.double().cpu().numpy() for k, v in vars(model).items()}
    n = len(text)
    x, pos, hidden = w["embedding"][text], np.arange(n), np.triu(np.ones((n, n), bool), 1)

    def mix(q, k, v, scale):  # [heads, n, d]
        s = np.where(hidden, -np.inf, q @ k.transpose(0, 2, 1) * scale)
        p = np.exp(s - s.max(-1, keepdims=True))
        return (p / p.sum(-1, keepdims=True)) @ v

    def heads(y, count):
        return y.reshape(n, count, -1)

    q = S.rotate(S.rms_norm(heads(x @ w["wq"], X.Q_HEADS), w["q_norm"], X.EPS), pos, X.FREQ, 0)
    k = S.rotate(S.rms_norm(heads(x @ w["wk"], X.KV_HEADS), w["k_norm"], X.EPS), pos, X.FREQ, 0)
    v = heads(x @ w["wv"], X.KV_HEADS)
    k, v = (np.repeat(y, X.Q_HEADS // X.KV_HEADS, 1).transpose(1, 0, 2) for y in (k, v))
    x = x + mix(q.transpose(1, 0, 2), k, v, X.DIM ** -0.5).transpose(1, 0, 2).reshape(n, -1) @ w["wo"]
    q, kv = heads(x @ w["wq_latent"], X.HEADS), x @ w["wkv_latent"]
    q = np.concatenate([q[..., :X.NOPE], S.rotate(q[..., X.NOPE:], pos, X.FREQ, 0)], -1)
    c = S.rms_norm(kv[:, :X.LATENT], w["latent_norm"], X.EPS)
    r = S.rotate(kv[:, None, X.LATENT:], pos, X.FREQ, 0)
    both = np.matmul(c[None], w["w_kv"].transpose(0, 2, 1))
    k = np.concatenate([both[..., :X.NOPE], np.repeat(r, X.HEADS, 1).transpose(1, 0, 2)], -1)
    out = mix(q.transpose(1, 0, 2), k, both[..., X.NOPE:], X.SCALE)
    return (x + out.transpose(1, 0, 2).reshape(n, -1) @ w["wo_latent"]) @ w["head"]


@pytest.mark.parametrize("users,longest", [(1, 20), (5, 300)])
def test_served_steps(users, longest):
    X = _example()
    service, texts, records = X.serve(users, 4, 5, longest)
    lengths = [len(t) - 1 for t in texts]
    assert service.cached.tolist() == lengths, "all but the last token are cached"
    for r in records:
        want = S.verify(r["counts"].tolist(), r["target"].cpu().numpy(), r["draft"].cpu().numpy(), r["drafted"].tolist(), r["uniforms"].cpu().numpy())
        assert r["tokens"].tolist() == list(want[0]) and r["accepted"].tolist() == list(want[1])
    # The last step's first row of each user stands behind the text as it was.  Some twenty values of size one are rounded to
    # bf16 on the way from a token to its logits, each by at most 2^-8.
    first, last = 0, records[-1]
    for u, text in enumerate(texts):
        at = lengths[u] - int(last["accepted"][u]) - 1
        want = _logits(X, service.model, np.array(text[:at + 1]))[-1]
        got = np.log(last["target"][first].double().cpu().numpy())
        diff = (got - got.mean()) - (want - want.mean())
        assert np.abs(diff).max() <= 20 * 2.0 ** -8, np.abs(diff).max()
        first += int(last["counts"][u]) + 1
