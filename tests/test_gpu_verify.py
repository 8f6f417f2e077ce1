"""efim_verify_drafts against whole-number arithmetic in Python: tokens and counts equal, for every answer there is."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_21889_amd import binding
    return binding


def _rows(rng, n, vocab, spread):
    x = np.exp(rng.standard_normal((n, vocab)) * spread).astype(np.float32)
    return (x / x.sum(-1, keepdims=True)).astype(np.float32)


def _draw(seed, drafts, vocab, given=True, spread=2.0):
    rng = np.random.default_rng(seed)
    total = int(np.sum(drafts))
    target = _rows(rng, total + len(drafts), vocab, spread)
    # near the target, so that some tokens stay
    where = np.concatenate([np.arange(n) + t for n, t in zip(drafts, np.cumsum([0] + [n + 1 for n in drafts[:-1]]))]).astype(int)
    near = target[where] * np.exp(rng.standard_normal((total, vocab)) * 0.3)
    draft = (near / near.sum(-1, keepdims=True)).astype(np.float32)
    if given:
        tokens = np.array([rng.choice(vocab, p=row.astype(np.float64) / row.astype(np.float64).sum()) for row in draft], np.int32)
    else:
        tokens = draft.argmax(-1).astype(np.int32) if total else np.zeros(0, np.int32)
    uniforms = rng.random(total + len(drafts), dtype=np.float32)
    return target, draft if given else None, tokens.astype(np.int32), uniforms


def _run(E, drafts, target, draft, tokens, uniforms, pad=0, shift=0):
    """pad: elements behind each row; shift: elements in front of the first, so that rows start at any multiple of 4 bytes."""
    vocab = target.shape[1]

    def dev(x):
        wide = np.full((len(x), vocab + pad), np.nan, np.float32)
        wide[:, :vocab] = x
        flat = torch.full((wide.size + shift,), float("nan"), device="cuda")
        flat[shift:] = torch.from_numpy(wide.reshape(-1)).cuda()
        return flat[shift:]

    td, dd = dev(target), None if draft is None else dev(draft)
    tok, u = torch.from_numpy(tokens).cuda(), torch.from_numpy(uniforms).cuda()
    out = torch.full((len(uniforms),), 12345, dtype=torch.int32, device="cuda")
    accepted = torch.full((len(drafts),), 12345, dtype=torch.int32, device="cuda")
    nbytes = E.efim_verify_workspace_bytes(len(drafts), vocab)
    ws = torch.full((max(nbytes, 256),), 0xFF, dtype=torch.uint8, device="cuda")
    E.efim_verify_drafts(np.asarray(drafts, np.int32), vocab, td, vocab + pad, dd, vocab + pad, tok, u, out, accepted, ws, nbytes)
    torch.cuda.synchronize()
    return out.cpu().numpy(), accepted.cpu().numpy()


def _check(E, drafts, target, draft, tokens, uniforms, **more):
    got = _run(E, drafts, target, draft, tokens, uniforms, **more)
    want = S.verify(drafts, target, draft, tokens, uniforms)
    assert np.array_equal(got[1], want[1])
    assert np.array_equal(got[0], want[0])
    return want


@pytest.mark.parametrize("vocab", [1, 2, 7, 255, 2047, 2048, 2049, 4099, 32004])
@pytest.mark.parametrize("given", [True, False])
def test_against_whole_numbers(E, vocab, given):
    for k, drafts in enumerate(([0], [1], [5, 0, 15, 3], [63, 1])):
        if sum(drafts) * vocab > 300000:
            drafts = [3, 0, 2]
        _check(E, drafts, *_draw(vocab + k, drafts, vocab, given))


@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 2), (60, 3)])
def test_strides_and_unaligned_rows(E, pad, shift):
    drafts = [4, 0, 7]
    _check(E, drafts, *_draw(5, drafts, 5001), pad=pad, shift=shift)


def test_a_row_of_several_blocks_a_chunk(E):
    """A vocabulary above 256 * 2048: a workgroup's chunk is more than one block."""
    vocab = 256 * 2048 + 777
    rng = np.random.default_rng(2)
    target, draft = _rows(rng, 3, vocab, 1.0), _rows(rng, 2, vocab, 1.0)
    for u in (0.0, 0.37, 0.999999):
        uniforms = np.array([0.999, 0.999, u], np.float32)
        _check(E, [2], target, draft, np.array([vocab - 1, 5], np.int32), uniforms)


def test_the_first_and_the_last_of_the_weights(E):
    vocab = 3000
    target = np.zeros((1, vocab), np.float32)
    target[0, 17], target[0, 2999] = 0.25, 0.75
    for u, token in ((0.0, 17), (0.2499999, 17), (0.25, 2999), (1.0 - 2.0 ** -24, 2999), (float("nan"), 17), (-1.0, 17), (2.0, 2999)):
        got, accepted = _run(E, [0], target, None, np.zeros(0, np.int32), np.array([u], np.float32))
        assert got.tolist() == [token] and accepted.tolist() == [0], u


def test_rows_that_leave_nothing(E):
    vocab = 2500
    p = _rows(np.random.default_rng(4), 2, vocab, 1.0)
    u = np.array([1.0 - 2.0 ** -24, 0.5], np.float32)
    # p = q: u q < p holds for every u below one, so a refusal is forced by a token outside the vocabulary; nothing is left
    # of p - q and the token is drawn from p
    for token in (-1, vocab, 2 ** 31 - 1, -2 ** 31):
        want = _check(E, [1], p, p[:1].copy(), np.array([token], np.int32), u)
        assert want[1][0] == 0 and want[0][0] >= 0
        _check(E, [1], p, None, np.array([token], np.int32), u)
    # the target holds nothing at all
    zero = np.zeros_like(p)
    want = _check(E, [1], zero, p[:1].copy(), np.array([3], np.int32), u)
    assert want[0].tolist() == [-1, -1] and want[1].tolist() == [0]
    # a certain draft whose token is all that the target holds, refused by a target below one
    only = np.zeros_like(p)
    only[:, 9] = 0.5
    want = _check(E, [1], only, None, np.array([9], np.int32), np.array([0.9, 0.1], np.float32))
    assert want[0].tolist() == [9, -1] and want[1].tolist() == [0]


def test_values_that_are_no_probabilities(E):
    vocab = 2600
    rng = np.random.default_rng(6)
    target, draft = _rows(rng, 4, vocab, 1.0), _rows(rng, 3, vocab, 1.0)
    for row, bits in ((target[0], [np.nan, -1.0, np.inf, 3.0]), (target[1], [-np.inf, 1e-45, 1e-13, 1.0]), (draft[0], [np.nan, np.inf, -2.0, 1e-40])):
        row[rng.choice(vocab, 40, replace=False)] = np.resize(np.array(bits, np.float32), 40)
    for seed in range(6):
        tokens = np.random.default_rng(seed).integers(0, vocab, 3).astype(np.int32)
        _check(E, [3], target, draft, tokens, np.random.default_rng(seed + 9).random(4, dtype=np.float32))


def test_more_requests_than_a_launch_takes_and_the_target_s_distribution(E):
    """4000 requests with one draft each of a vocabulary of five: the first token is distributed as the target says,
    however far the draft is from it (within five standard deviations)."""
    requests, vocab = 4000, 5
    rng = np.random.default_rng(8)
    p, q = np.array([0.1, 0.4, 0.05, 0.25, 0.2], np.float32), np.array([0.3, 0.1, 0.3, 0.1, 0.2], np.float32)
    target, draft = np.tile(p, (2 * requests, 1)), np.tile(q, (requests, 1))
    tokens = rng.choice(vocab, requests, p=q.astype(np.float64) / q.astype(np.float64).sum()).astype(np.int32)
    uniforms = rng.random(2 * requests, dtype=np.float32)
    out, _ = _check(E, [1] * requests, target, draft, tokens, uniforms)
    counts = np.bincount(out[::2], minlength=vocab)
    assert np.all(np.abs(counts - requests * p) <= 5 * np.sqrt(requests * p * (1 - p)))


def test_graph_replays(E):
    drafts = [3, 2]
    target, draft, tokens, uniforms = _draw(3, drafts, 9001)
    want = S.verify(drafts, target, draft, tokens, uniforms)
    td, dd, tok, u = (torch.from_numpy(x).cuda() for x in (target, draft, tokens, uniforms))
    out, accepted = torch.zeros(len(uniforms), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    nbytes = E.efim_verify_workspace_bytes(2, 9001)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        E.efim_verify_drafts(drafts, 9001, td, 9001, dd, 9001, tok, u, out, accepted, ws, nbytes, torch.cuda.current_stream())
    for k in range(4):
        for x in (out, accepted, ws):
            x.fill_(k + 7)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out.cpu().numpy(), want[0]) and np.array_equal(accepted.cpu().numpy(), want[1])
        (td * 2).sum().item()
