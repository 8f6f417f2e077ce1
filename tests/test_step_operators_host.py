"""CPU tests of the normed append, the latent cache's calls and the verification: refusals before a device is touched, sizes
of workspaces, plans under sanitizers, and pins of their oracle."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import step_oracle as S
from oracle.efim_oracle import f64_to_bf16
from paper_2505_21889_amd import binding as E

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_21889_amd", "csrc")
FAKE = 0x7F0000001000  # never dereferenced by the host-only paths exercised here
FREQ = (ctypes.c_double * 64)(*[1.0 / (j + 1) for j in range(64)])
BAD, UNSUPPORTED, SPACE = E.EFIM_ERR_INVALID_ARG, E.EFIM_ERR_UNSUPPORTED, E.EFIM_ERR_WORKSPACE


def _desc(c, n, hq=4, hkv=1, d=576, page=16, table=FAKE, max_pages=None, num_pages=None):
    need = [-(-(int(a) + int(b)) // 16) for a, b in zip(c, n)]
    return E.BatchDesc(np.asarray(c, np.int32), np.asarray(n, np.int32), table, hq, hkv, d, page,
                       sum(need) + 2 if num_pages is None else num_pages, max(need + [1]) if max_pages is None else max_pages)


def _norm(desc, q=FAKE, q_out=FAKE, k=FAKE, v=FAKE, wq=FAKE, wk=FAKE, eps=1e-6, kc=FAKE, vc=FAKE, freq=FREQ, rotary=128, inter=0, scales=None):
    lib, args = E.raw_library(), (ctypes.byref(desc.c), q, q_out, k, v, wq, wk, eps, kc, vc, freq, rotary, inter)
    if scales:
        return lib.efim_norm_rope_append_fp8(*args, *scales, None)
    return lib.efim_norm_rope_append(*args, None)


def test_norm_append_refusals():
    heads = dict(hq=4, hkv=2, d=128)
    ok = _desc([10], [5], **heads)
    assert _norm(_desc([10], [5], 4, 2, 96)) == UNSUPPORTED
    assert _norm(_desc([10], [5], page=24, max_pages=9, **heads)) == UNSUPPORTED
    assert _norm(_desc([10], [5], 5, 2, 128)) == BAD
    assert _norm(_desc([100], [5], max_pages=3, **heads)) == BAD
    for eps in (-1e-6, float("nan"), float("inf")):
        assert _norm(ok, eps=eps) == BAD
    for rotary in (0, 8, 24, 144):
        assert _norm(ok, rotary=rotary) == BAD
    assert _norm(ok, freq=None) == BAD and _norm(ok, inter=2) == BAD
    assert _norm(ok, freq=(ctypes.c_double * 64)(*([1.0] * 63 + [float("nan")]))) == BAD
    assert _norm(ok, q_out=None) == BAD and _norm(ok, q=None) == BAD
    for name in ("k", "v", "kc", "vc"):
        assert _norm(ok, **{name: None}) == BAD
    for name in ("q", "q_out", "k", "v", "wq", "wk", "kc", "vc"):
        assert _norm(ok, **{name: FAKE + 8}) == BAD
    assert _norm(_desc([10], [5], table=FAKE + 2, **heads)) == BAD
    for scales in ((0.0, 1.0), (1.0, -1.0), (float("inf"), 1.0), (1.0, float("nan"))):
        assert _norm(ok, scales=scales) == BAD
    assert _norm(_desc([0], [1 << 26], 1, 1, 64, page=256, max_pages=1 << 18, num_pages=1 << 18), rotary=64) == UNSUPPORTED
    assert E.raw_library().efim_norm_rope_append(None, *[None] * 6, 0.0, None, None, None, 0, 0, None) == BAD
    assert _norm(_desc([10, 3], [0, 0], **heads), None, None, None, None, None, None, 1e-6, None, None) == E.EFIM_OK
    assert _norm(_desc([], [], table=None, **heads), None, None, None, None, None, None, 1e-6, None, None) == E.EFIM_OK


def _append(desc, q=FAKE, qs=192, qo=FAKE + 0x1000, qos=64, kv=FAKE, kvs=576, w=FAKE, eps=1e-6, cache=FAKE, freq=FREQ, inter=0):
    return E.raw_library().efim_latent_append(ctypes.byref(desc.c), q, qs, qo, qos, kv, kvs, w, eps, cache, freq, inter, None)


def _attend(desc, q=FAKE, cache=FAKE + 0x1000, out=FAKE + 0x2000, scale=0.07, ws=FAKE + 0xFFF000, nbytes=1 << 40):
    return E.raw_library().efim_latent_attention(ctypes.byref(desc.c), q, cache, out, scale, ws, nbytes, None)


def _expand(desc, q=FAKE, cache=FAKE + 0x1000, w=FAKE + 0x3000, out=FAKE + 0x2000, scale=0.07, ws=FAKE + 0xFFF000, nbytes=1 << 40):
    return E.raw_library().efim_latent_attention_expanded(ctypes.byref(desc.c), q, cache, w, out, scale, ws, nbytes, None)


def test_latent_refusals():
    ok = _desc([10], [5])
    for call in (_append, _attend, _expand):
        assert call(_desc([10], [5], d=512)) == UNSUPPORTED
        assert call(_desc([10], [5], hq=4, hkv=2)) == UNSUPPORTED
        assert call(_desc([10], [5], hq=257)) == UNSUPPORTED
        for page in (4, 24, 512):
            assert call(_desc([10], [5], page=page, max_pages=9, num_pages=9)) == UNSUPPORTED
        assert call(_desc([-1], [5])) == BAD and call(_desc([1], [-5])) == BAD
        assert call(_desc([100], [5], max_pages=3)) == BAD and call(_desc([100], [5], num_pages=2)) == BAD
        assert call(_desc([10], [5], table=None)) == BAD and call(_desc([10], [5], table=FAKE + 1)) == BAD
        assert call(_desc([4], [0]), None) == E.EFIM_OK or call is _append
    for eps in (-1.0, float("nan"), float("inf")):
        assert _append(ok, eps=eps) == BAD
    assert _append(ok, q=None) == BAD and _append(ok, qo=None) == BAD and _append(ok, kv=None) == BAD and _append(ok, cache=None) == BAD
    for name in ("q", "qo", "kv", "w", "cache"):
        assert _append(ok, **{name: FAKE + 4}) == BAD
    for name, values in (("qs", (0, 60, 68, -64)), ("qos", (32, 65)), ("kvs", (512, 577, 580))):
        for value in values:
            assert _append(ok, **{name: value}) == BAD
    assert _append(ok, qo=FAKE, qos=64) == BAD          # in place needs the same stride
    assert _append(ok, freq=None) == BAD and _append(ok, inter=-1) == BAD
    assert _append(_desc([4], [0]), None, 0, None, 0, None, 576, None, 1e-6, None) == E.EFIM_OK
    assert _append(_desc([0], [1 << 26], 1, page=256, max_pages=1 << 18, num_pages=1 << 18)) == UNSUPPORTED
    for call in (_attend, _expand):
        for scale in (0.0, -1.0, float("nan"), float("inf")):
            assert call(ok, scale=scale) == BAD
        for name in ("q", "cache", "out"):
            assert call(ok, **{name: None}) == BAD and call(ok, **{name: FAKE + 0x8008}) == BAD
        assert call(ok, out=FAKE) == BAD and call(ok, out=FAKE + 0x1000) == BAD
        assert call(ok, ws=None) == SPACE and call(ok, ws=FAKE + 0xFFF010) == SPACE
    assert _expand(ok, w=None) == BAD and _expand(ok, w=FAKE + 8) == BAD and _expand(ok, out=FAKE + 0x3000) == BAD
    need = E.efim_latent_expanded_workspace_bytes(ok)
    assert need == 2 * 64 * 640 * 4 and _expand(ok, nbytes=need - 1) == SPACE
    split = _desc([60000], [1])
    need = E.efim_latent_workspace_bytes(split)
    assert need > 256 and _attend(split, nbytes=need - 1) == SPACE
    assert E.efim_latent_workspace_bytes(_desc([], [], table=None)) == 256
    for size in (E.efim_latent_workspace_bytes, E.efim_latent_expanded_workspace_bytes):
        assert size(_desc([10], [5], d=128)) == 0 and size(_desc([3], [0])) == 256
    # a request alone whose expanded tiles pass a launch's reach
    assert E.efim_latent_expanded_workspace_bytes(_desc([1 << 29], [1], 256, page=256, max_pages=1 << 22, num_pages=1 << 22)) == 0
    assert _expand(_desc([1 << 29], [1], 256, page=256, max_pages=1 << 22, num_pages=1 << 22)) == UNSUPPORTED


def test_latent_rows_are_counted_in_32_bits():
    def rows(new, heads):
        return _desc([0] * len(new), new, heads, page=256, max_pages=1 << 22, num_pages=1 << 22)

    for new, heads in (([1 << 23], 256), ([1 << 22] * 2, 256), ([(1 << 22) + 1], 256)):
        for call in (_attend, _expand):
            assert call(rows(new, heads)) == UNSUPPORTED
        assert E.efim_latent_workspace_bytes(rows(new, heads)) == 0 == E.efim_latent_expanded_workspace_bytes(rows(new, heads))
    assert E.efim_latent_workspace_bytes(rows([1 << 22], 256)) > 256


def _verify(counts=(2, 1), batch=None, vocab=100, t=FAKE, ts=100, d=FAKE, ds=100, tok=FAKE, u=FAKE, out=FAKE, acc=FAKE, ws=FAKE, nbytes=1 << 30, drafts=True):
    arr = np.asarray(counts, np.int32)
    return E.raw_library().efim_verify_drafts(len(counts) if batch is None else batch, arr.ctypes.data if drafts else None, vocab,
                                              t, ts, d, ds, tok, u, out, acc, ws, nbytes, None)


def test_verify_refusals():
    assert _verify(batch=-1) == BAD and _verify(vocab=0) == BAD and _verify(vocab=-5) == BAD
    assert _verify(ts=99) == BAD and _verify(ds=99) == BAD
    assert _verify((1, -1)) == BAD and _verify((64,)) == UNSUPPORTED and _verify(vocab=(1 << 22) + 1, ts=1 << 23, ds=1 << 23) == UNSUPPORTED
    assert _verify(drafts=False) == BAD
    for name in ("t", "tok", "u", "out", "acc"):
        assert _verify(**{name: None}) == BAD
    for name in ("t", "d", "tok", "u", "out", "acc"):
        assert _verify(**{name: FAKE + 2}) == BAD
    need = E.efim_verify_workspace_bytes(2, 100)
    assert need >= 256 and _verify(nbytes=need - 1) == SPACE and _verify(ws=None) == SPACE and _verify(ws=FAKE + 16) == SPACE
    assert _verify((), drafts=False) == E.EFIM_OK
    assert E.efim_verify_workspace_bytes(-1, 10) == 0 and E.efim_verify_workspace_bytes(1, 0) == 0
    assert E.efim_verify_workspace_bytes(3, (1 << 22) + 1) == 0 and E.efim_verify_workspace_bytes(0, 10) == 256


def test_plans_under_sanitizers(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("g++ or the HIP headers are not available")
    exe = str(tmp_path / "fuzz_latent_plan")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
           "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(ROOT, "tests", "native", "fuzz_latent_plan.cpp"), os.path.join(CSRC, "latent_plan.cpp"),
           os.path.join(CSRC, "planner.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0 and "latent plan ok" in run.stdout, (run.stdout + run.stderr)[-4000:]


# --- pins of the oracle --------------------------------------------------------------------------------------------------------


def test_oracle_norm_and_rotation():
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])
    assert np.allclose(S.rms_norm(x, None, 0.0), x / 2.5)
    assert np.allclose(S.rms_norm(x, np.array([1.0, 2.0, 3.0, 4.0]), 0.0), [[[1.2, 3.2, 0, 0]]])
    quarter = np.array([np.pi / 2])
    assert np.allclose(S.rotate(x, [1], quarter, 1), [[[-4.0, 3.0, 0, 0]]])
    assert np.allclose(S.rotate(x, [2], quarter, 0), [[[-3.0, -4.0, 0, 0]]])
    y = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    assert np.allclose(S.rotate(y, [1], np.array([np.pi / 2, np.pi]), 0), [[[-3.0, -2.0, 1.0, -4.0]]])


def test_oracle_attention_forms_against_torch():
    rng = np.random.default_rng(5)
    cached, new, page, heads = [3], [4], 8, 2
    table, cache = np.array([[1]]), np.zeros((2, 8, 576), np.uint16)
    cache[1, :7] = f64_to_bf16(rng.standard_normal((7, 576)))
    rows = S.latent_rows(cache, table[0], page, 7)
    q, w = rng.standard_normal((4, heads, 192)), rng.standard_normal((heads, 256, 512)) / 23
    got, _ = S.latent_attention_expanded(cached, new, table, page, q, cache, w, 0.1, round_expanded=False)
    keys = np.concatenate([np.einsum("hjc,kc->hkj", w[:, :128], rows[:, :512]), np.broadcast_to(rows[:, 512:], (heads, 7, 64))], -1)
    values = np.einsum("hjc,kc->hkj", w[:, 128:], rows[:, :512])
    mask = torch.ones(4, 7, dtype=torch.bool).tril(3)
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x))
    want = torch.nn.functional.scaled_dot_product_attention(t(q.transpose(1, 0, 2)), t(keys), t(values), attn_mask=mask, scale=0.1)
    assert np.allclose(got, want.numpy().transpose(1, 0, 2))
    absorbed = np.concatenate([np.einsum("thj,hjc->thc", q[..., :128], w[:, :128]), q[..., 128:]], -1)
    latent, _ = S.latent_attention(cached, new, table, page, absorbed, cache, 0.1)
    assert np.allclose(np.einsum("thc,hjc->thj", latent, w[:, 128:]), got)


def test_oracle_verification_by_hand():
    target = np.array([[0.5, 0.25, 0.25], [0.0, 0.5, 0.5], [0.25, 0.25, 0.5]], np.float32)
    draft = np.array([[0.25, 0.5, 0.25], [0.5, 0.25, 0.25]], np.float32)
    run = lambda tokens, u, q=draft: tuple(x.tolist() for x in S.verify([2], target, q, np.array(tokens, np.int32), np.array(u, np.float32)))
    assert run([0, 2], [0.99, 0.99, 0.5]) == ([0, 2, 2], [2])     # both stay; u = 0.5 passes the first two quarters
    assert run([1, 2], [0.5, 0.0, 0.5]) == ([0, -1, -1], [0])     # 0.5 * 0.5 is not below 0.25; all that is left is token 0
    assert run([1, 2], [0.49, 0.0, 0.49]) == ([1, 2, 1], [2])
    assert run([0, 0], [0.0, 0.0, 0.3]) == ([0, 1, -1], [1])      # the target holds nothing for token 0 in row 1; 0.25 of each left
    assert run([0, 1], [0.4, 0.6, 0.0], None) == ([0, 2, -1], [1])
