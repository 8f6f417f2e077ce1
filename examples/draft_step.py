"""A small model's serving loop with drafted tokens: prompts, then steps in which every user has some.

The model is random and has two layers, one of each kind of cache:

  heads   queries and keys normed per head and rotated on their way into the paged cache (efim_norm_rope_append),
          attention of the new tokens (efim_extend_attention);
  latent  one row a token for all heads: normed and rotated on its way into the paged cache (efim_latent_append), attention
          over the rows themselves (efim_latent_attention) in a short step, over keys and values expanded from them
          (efim_latent_attention_expanded) where a step has many new tokens.

A step computes a user's last token and its drafted ones together.  efim_verify_drafts says how many of these stay and
which token follows; what the others left in the caches lies behind the user's length and is written again.

  python3 examples/draft_step.py [users] [steps]
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2505_21889_amd import binding as E  # noqa: E402

HIDDEN, VOCAB, PAGE, EPS = 256, 997, 16, 1e-6
Q_HEADS, KV_HEADS, DIM = 4, 2, 64
HEADS, NOPE, ROPE, VALUE, LATENT = 4, 128, 64, 128, 512
SCALE = (NOPE + ROPE) ** -0.5
EXPAND_FROM = 170  # new tokens of a request from which on the expanded form costs less
FREQ = 1e4 ** (-2.0 * np.arange(DIM // 2) / DIM)  # (both layers rotate 64 elements)


class Model:
    def __init__(self, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, scale=1.0):
            return torch.randn(shape, dtype=torch.bfloat16, device="cuda", generator=gen).mul_(scale)

        self.embedding = normal(VOCAB, HIDDEN)
        self.head = normal(HIDDEN, VOCAB, scale=HIDDEN ** -0.5)
        self.wq, self.wo = normal(HIDDEN, Q_HEADS * DIM, scale=HIDDEN ** -0.5), normal(Q_HEADS * DIM, HIDDEN, scale=HIDDEN ** -0.5)
        self.wk, self.wv = (normal(HIDDEN, KV_HEADS * DIM, scale=HIDDEN ** -0.5) for _ in range(2))
        self.q_norm, self.k_norm = normal(DIM, scale=0.2) + 1.0, normal(DIM, scale=0.2) + 1.0
        self.wq_latent = normal(HIDDEN, HEADS * (NOPE + ROPE), scale=HIDDEN ** -0.5)
        self.wkv_latent = normal(HIDDEN, LATENT + ROPE, scale=HIDDEN ** -0.5)
        self.latent_norm = normal(LATENT, scale=0.2) + 1.0
        self.w_kv = normal(HEADS, NOPE + VALUE, LATENT, scale=LATENT ** -0.5)  # expands a latent: keys, then values
        self.w_uk = self.w_kv[:, :NOPE].contiguous()
        self.w_uv = self.w_kv[:, NOPE:].transpose(1, 2).contiguous()
        self.wo_latent = normal(HEADS * VALUE, HIDDEN, scale=(HEADS * VALUE) ** -0.5)


class Service:
    """The caches of all users and their lengths."""

    def __init__(self, model, users, longest, seed=1):
        self.model, self.users = model, users
        per_user = -(-longest // PAGE)
        self.pages = users * per_user
        order = np.random.default_rng(seed).permutation(self.pages).astype(np.int32)
        self.table = torch.from_numpy(order.reshape(users, per_user)).cuda()
        bf16 = {"dtype": torch.bfloat16, "device": "cuda"}
        self.k_cache, self.v_cache = (torch.empty(self.pages, KV_HEADS, PAGE, DIM, **bf16) for _ in range(2))
        self.rows = torch.empty(self.pages, PAGE, LATENT + ROPE, **bf16)
        self.cached = np.zeros(users, np.int32)

    def _workspace(self, nbytes):
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device="cuda"), nbytes

    def _heads_layer(self, x, new):
        m, tokens = self.model, len(x)
        q, k, v = (x @ m.wq).view(tokens, Q_HEADS, DIM), (x @ m.wk).view(tokens, KV_HEADS, DIM), (x @ m.wv).view(tokens, KV_HEADS, DIM)
        batch = E.BatchDesc(self.cached, new, self.table, Q_HEADS, KV_HEADS, DIM, PAGE, self.pages)
        E.efim_norm_rope_append(batch, q, q, k, v, m.q_norm, m.k_norm, EPS, self.k_cache, self.v_cache, FREQ, DIM)
        out = torch.empty_like(q)
        ws, nbytes = self._workspace(E.efim_extend_workspace_bytes(batch))
        E.efim_extend_attention(batch, q, self.k_cache, self.v_cache, out, DIM ** -0.5, ws, nbytes)
        return x + out.view(tokens, -1) @ m.wo

    def _latent_layer(self, x, new):
        m, tokens = self.model, len(x)
        q, kv = (x @ m.wq_latent).view(tokens, HEADS, NOPE + ROPE), x @ m.wkv_latent
        batch = E.BatchDesc(self.cached, new, self.table, HEADS, 1, LATENT + ROPE, PAGE, self.pages)
        if new.max() >= EXPAND_FROM:
            E.efim_latent_append(batch, q[:, :, NOPE:], NOPE + ROPE, q[:, :, NOPE:], NOPE + ROPE, kv, LATENT + ROPE, m.latent_norm, EPS,
                                 self.rows, FREQ)
            out = torch.empty(tokens, HEADS, VALUE, dtype=torch.bfloat16, device="cuda")
            ws, nbytes = self._workspace(E.efim_latent_expanded_workspace_bytes(batch))
            E.efim_latent_attention_expanded(batch, q, self.rows, m.w_kv, out, SCALE, ws, nbytes)
        else:
            absorbed = torch.empty(tokens, HEADS, LATENT + ROPE, dtype=torch.bfloat16, device="cuda")
            E.efim_latent_append(batch, q[:, :, NOPE:], NOPE + ROPE, absorbed[:, :, LATENT:], LATENT + ROPE, kv, LATENT + ROPE, m.latent_norm,
                                 EPS, self.rows, FREQ)
            absorbed[:, :, :LATENT] = torch.bmm(q[:, :, :NOPE].transpose(0, 1).contiguous(), m.w_uk).transpose(0, 1)
            mixed = torch.empty(tokens, HEADS, LATENT, dtype=torch.bfloat16, device="cuda")
            ws, nbytes = self._workspace(E.efim_latent_workspace_bytes(batch))
            E.efim_latent_attention(batch, absorbed, self.rows, mixed, SCALE, ws, nbytes)
            out = torch.bmm(mixed.transpose(0, 1).contiguous(), m.w_uv).transpose(0, 1)
        return x + out.reshape(tokens, -1) @ m.wo_latent

    def logits(self, tokens, new):
        """Of `new[r]` tokens of every user, packed; they lie in the caches afterwards."""
        x = self._latent_layer(self._heads_layer(self.model.embedding[tokens.long()], new), new)
        return x.float() @ self.model.head.float()

    def step(self, last, drafts, draft_probs, uniforms):
        """last [users]: each user's last token, not in the caches yet.  drafts: a list of each user's drafted tokens (host), drawn
        from the rows of draft_probs.  Returns the users' tokens from here on and what the step was decided by."""
        counts = np.array([len(d) for d in drafts], np.int32)
        new = counts + 1
        tokens = torch.tensor([t for l, d in zip(last, drafts) for t in [l] + list(d)], dtype=torch.int32, device="cuda")
        drafted = torch.tensor([t for d in drafts for t in d], dtype=torch.int32, device="cuda")
        target = torch.softmax(self.logits(tokens, new), -1)
        out = torch.empty(len(tokens), dtype=torch.int32, device="cuda")
        accepted = torch.empty(self.users, dtype=torch.int32, device="cuda")
        ws, nbytes = self._workspace(E.efim_verify_workspace_bytes(self.users, VOCAB))
        E.efim_verify_drafts(counts, VOCAB, target, VOCAB, draft_probs, VOCAB, drafted, uniforms, out, accepted, ws, nbytes)
        stay, out = accepted.cpu().numpy(), out.cpu().numpy()
        first = np.concatenate([[0], np.cumsum(new)])
        self.cached = self.cached + stay + 1
        got = [out[first[r]:first[r] + stay[r] + 1].tolist() for r in range(self.users)]
        return got, {"counts": counts, "target": target, "draft": draft_probs, "drafted": drafted, "uniforms": uniforms, "tokens": out,
                     "accepted": stay}


def serve(users=4, steps=4, most_drafts=5, longest_prompt=300, seed=3):
    """Serves `users` random prompts; returns the service, every user's tokens and the steps' records."""
    rng, gen = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    prompts = [rng.integers(0, VOCAB, rng.integers(1, longest_prompt + 1)).tolist() for _ in range(users)]
    service = Service(Model(seed), users, longest_prompt + steps * (most_drafts + 1) + most_drafts + 1)
    # the prompts but for their last tokens, which begin the first step
    new = np.array([len(p) - 1 for p in prompts], np.int32)
    service.logits(torch.tensor([t for p in prompts for t in p[:-1]], dtype=torch.int32, device="cuda"), new)
    service.cached = service.cached + new
    records = []
    for _ in range(steps):
        counts = rng.integers(0, most_drafts + 1, users)
        draft_probs = torch.softmax(torch.randn(int(counts.sum()), VOCAB, device="cuda", generator=gen), -1)
        drawn = torch.multinomial(draft_probs, 1, generator=gen)[:, 0].tolist() if len(draft_probs) else []
        ends = np.cumsum(counts)
        drafts = [drawn[e - n:e] for e, n in zip(ends, counts)]
        uniforms = torch.rand(int(counts.sum()) + users, device="cuda", generator=gen)
        got, record = service.step([p[-1] for p in prompts], drafts, draft_probs, uniforms)
        for p, g in zip(prompts, got):
            p += g
        records.append(record)
    return service, prompts, records


if __name__ == "__main__":
    numbers = [int(a) for a in sys.argv[1:]]
    _, texts, records = serve(*numbers)
    for i, r in enumerate(records):
        print("step %d: drafted %s, stayed %s" % (i, r["counts"].tolist(), r["accepted"].tolist()))
    print("last tokens:", [t[-6:] for t in texts])
