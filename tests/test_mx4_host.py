"""CPU tests of the operators of a step over a 4-bit cache: refusals before a device is touched, sizes, and pins of their oracle."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import mx4_oracle as M
from oracle.efim_oracle import bf16_to_f64, f64_to_bf16
from paper_2505_21889_amd import binding as E

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_21889_amd", "csrc")
FAKE = 0x7F0000001000  # never dereferenced by the host-only paths exercised here
FREQ = (ctypes.c_double * 64)(*[1.0 / (j + 1) for j in range(64)])
BAD, UNSUPPORTED, SPACE = E.EFIM_ERR_INVALID_ARG, E.EFIM_ERR_UNSUPPORTED, E.EFIM_ERR_WORKSPACE


def _desc(c, n, hq=4, hkv=2, d=128, page=16, table=FAKE, max_pages=None, num_pages=None):
    need = [-(-(int(a) + int(b)) // 16) for a, b in zip(c, n)]
    return E.BatchDesc(np.asarray(c, np.int32), np.asarray(n, np.int32), table, hq, hkv, d, page,
                       sum(need) + 2 if num_pages is None else num_pages, max(need + [1]) if max_pages is None else max_pages)


def _append(desc, q=FAKE, qo=FAKE + 0x1000, k=FAKE, v=FAKE, kc=FAKE, vc=FAKE, ks=None, vs=None, freq=FREQ, rotary=128, inter=0):
    return E.raw_library().efim_rope_append_mx4(ctypes.byref(desc.c), q, qo, k, v, kc, vc, ks, vs, freq, rotary, inter, None)


def _attend(desc, q=FAKE, kc=FAKE, vc=FAKE, out=FAKE + 0x2000, scale=0.0, ws=FAKE + 0xFFF000, size=1 << 40):
    return E.raw_library().efim_extend_attention_mx4(ctypes.byref(desc.c), q, kc, vc, out, scale, ws, size, None)


def test_cache_calls_refuse():
    for call in (_append, _attend):
        assert call(_desc([10], [5], d=96)) == UNSUPPORTED and call(_desc([10], [5], hq=5)) == BAD
        assert call(_desc([10], [5], hq=130, hkv=2)) == UNSUPPORTED
        for page in (4, 24, 512):
            assert call(_desc([10], [5], page=page, max_pages=9, num_pages=9)) == UNSUPPORTED
        assert call(_desc([-1], [5])) == BAD and call(_desc([1], [-5])) == BAD
        assert call(_desc([100], [5], max_pages=3)) == BAD and call(_desc([100], [5], num_pages=2)) == BAD
        assert call(_desc([10], [5], table=None)) == BAD and call(_desc([10], [5], table=FAKE + 2)) == BAD
        for name in ("q", "kc", "vc"):
            assert call(_desc([10], [5]), **{name: None}) == BAD and call(_desc([10], [5]), **{name: FAKE + 8}) == BAD
    ok = _desc([10], [5])
    for name in ("k", "v", "qo"):
        assert _append(ok, **{name: None}) == BAD and _append(ok, **{name: FAKE + 8}) == BAD
    assert _append(ok, ks=FAKE + 8) == BAD and _append(ok, vs=FAKE + 8) == BAD
    for rotary in (0, 8, 24, 144):
        assert _append(ok, rotary=rotary) == BAD
    assert _append(ok, freq=None) == BAD and _append(ok, inter=2) == BAD
    assert _append(ok, freq=(ctypes.c_double * 64)(*([1.0] * 63 + [float("nan")]))) == BAD
    assert _append(_desc([0], [1 << 26], 1, 1, page=256, max_pages=1 << 18, num_pages=1 << 18)) == UNSUPPORTED
    assert _append(_desc([10, 3], [0, 0]), None, None, None, None, None, None) == E.EFIM_OK
    assert _append(_desc([], [], table=None), None, None, None, None, None, None) == E.EFIM_OK

    for scale in (-1.0, float("nan"), float("inf")):
        assert _attend(ok, scale=scale) == BAD
    assert _attend(ok, out=None) == BAD and _attend(ok, out=FAKE + 8) == BAD
    need = E.efim_mx4_workspace_bytes(ok)
    assert need >= 256
    assert _attend(ok, ws=None) == SPACE and _attend(ok, ws=FAKE + 0xFFF080) == SPACE and _attend(ok, size=need - 1) == SPACE
    long = _desc([0], [1 << 25], 64, 1, page=256, max_pages=1 << 17, num_pages=1 << 17)
    assert _attend(long) == UNSUPPORTED and E.efim_mx4_workspace_bytes(long) == 0
    assert _attend(_desc([4], [0]), None, None, None, None, 0.0, None, 0) == E.EFIM_OK
    assert E.efim_mx4_workspace_bytes(_desc([4], [0])) == 256 and E.efim_mx4_workspace_bytes(_desc([4], [1], d=32)) == 0
    assert E.raw_library().efim_extend_attention_mx4(None, *[None] * 4, 0.0, None, 0, None) == BAD


def test_cache_sizes():
    assert E.efim_mx4_cache_bytes(10, 8, 16, 128) == 10 * 8 * 16 * 68 == int(np.prod(M.cache_shape(10, 8, 16, 128)))
    assert E.efim_mx4_cache_bytes(3, 2, 8, 64) == 3 * 2 * 8 * 34
    assert E.efim_mx4_cache_bytes(1 << 31, 64, 256, 128) == (1 << 31) * 64 * 256 * 68
    for wrong in ((-1, 8, 16, 128), (1, 0, 16, 128), (1, 8, 24, 128), (1, 8, 4, 128), (1, 8, 512, 128), (1, 8, 16, 96), (1 << 62, 64, 256, 128)):
        assert E.efim_mx4_cache_bytes(*wrong) == 0


def _tables(batch=2, h=FAKE, c=FAKE, n=FAKE, page=16, table=FAKE, wide=5, free=FAKE, capacity=9, count=FAKE, after=FAKE, slots=FAKE, room=7,
            start=FAKE, status=FAKE, ws=FAKE + 0xFFF000, size=1 << 30):
    return E.raw_library().efim_block_tables(batch, h, c, n, page, table, wide, free, capacity, count, after, slots, room, start, status, ws, size, None)


def test_block_tables_refuse():
    for wrong in ({"batch": -1}, {"wide": -1}, {"capacity": -1}, {"capacity": 1 << 31}, {"room": -1}, {"slots": FAKE + 4}):
        assert _tables(**wrong) == BAD, wrong
    for name in ("h", "c", "n", "table", "free", "count", "after", "start", "status"):
        assert _tables(**{name: None}) == BAD and _tables(**{name: FAKE + 2}) == BAD, name
    for page in (0, 4, 24, 512, -16):
        assert _tables(page=page) == UNSUPPORTED
    assert _tables(batch=(1 << 20) + 1) == UNSUPPORTED
    assert _tables(ws=None) == SPACE and _tables(ws=FAKE + 0xFFF010) == SPACE
    assert _tables(size=E.efim_block_tables_workspace_bytes(2) - 1) == SPACE
    assert E.efim_block_tables_workspace_bytes(-1) == 0 and E.efim_block_tables_workspace_bytes(0) == 256


def _logits(drafts=(2, 0), vocab=100, stride=100, out=FAKE, out_stride=100, ws=FAKE + 0xFFF000, size=1 << 40, bf16=0, **fields):
    arrays = dict(logits=FAKE, params=FAKE, history=FAKE, history_stride=4, draft_tokens=FAKE, bias_tokens=FAKE, bias_values=FAKE, bias_stride=3,
                  masks=FAKE, mask_stride=4, num_masks=2, mask_rows=FAKE)
    arrays.update(fields)
    desc = E.LogitsDesc(drafts, vocab, arrays.pop("logits"), stride, bf16=bf16, **arrays)
    return E.raw_library().efim_logit_probs(ctypes.byref(desc.c), out, out_stride, ws, size, None), desc


def test_logit_probs_refuse():
    code = lambda *a, **k: _logits(*a, **k)[0]
    assert code((2, -1)) == BAD and code((2, 64)) == UNSUPPORTED
    assert code(vocab=0) == BAD and code(vocab=-3) == BAD and code(vocab=(1 << 22) + 1, stride=1 << 23, out_stride=1 << 23) == UNSUPPORTED
    assert code(stride=99) == BAD and code(out_stride=99) == BAD and code(bf16=2) == BAD
    assert code(logits=None) == BAD and code(out=None) == BAD and code(draft_tokens=None) == BAD
    assert code(logits=FAKE + 2) == BAD and code(logits=FAKE + 1, bf16=1) == BAD and code(out=FAKE + 2) == BAD
    for name in ("params", "history", "draft_tokens", "bias_tokens", "bias_values", "masks", "mask_rows"):
        assert code(**{name: FAKE + 2}) == BAD, name
    assert code(history_stride=-1) == BAD and code(bias_stride=-1) == BAD
    assert code(bias_tokens=None) == BAD and code(bias_values=None) == BAD
    assert code(mask_stride=3) == BAD and code(num_masks=-1) == BAD
    _, desc = _logits()
    need = E.efim_logit_workspace_bytes(desc)
    assert need >= 256
    assert code(ws=None) == SPACE and code(ws=FAKE + 0xFFF008) == SPACE and code(size=need - 1) == SPACE
    assert code(()) == E.EFIM_OK and code((), logits=None, out=None, ws=None) == E.EFIM_OK
    assert E.raw_library().efim_logit_probs(None, None, 0, None, 0, None) == BAD
    assert E.raw_library().efim_logit_workspace_bytes(None) == 0
    assert E.efim_logit_workspace_bytes(_logits((2, 64))[1]) == 0
    # rows of a launch decide: two launches of 512 requests take what one does
    assert E.efim_logit_workspace_bytes(_logits((1,) * 1024, draft_tokens=FAKE)[1]) == E.efim_logit_workspace_bytes(_logits((1,) * 512)[1])
    assert E.SAMPLING_DTYPE.itemsize == 32


def test_sizes_beyond_the_calls_limits():
    limit = (1 << 30) - 64
    assert _logits(history_stride=limit + 1)[0] == UNSUPPORTED and _logits(history_stride=limit, size=0)[0] == SPACE
    heads = (1 << 16) + 1
    wide = _desc([10], [1], heads, heads)
    assert _attend(wide) == UNSUPPORTED and E.efim_mx4_workspace_bytes(wide) == 0
    assert _attend(_desc([10], [1], 1 << 16, 1 << 16), size=0) == SPACE


# --- pins of the oracle --------------------------------------------------------------------------------------------------------


def test_oracle_format_by_hand():
    row = np.zeros(64)
    row[:8] = [7.0, -6.0, 5.0, 2.5, 0.25, -0.75, 1.25, 0.26]
    row[32:36] = [7.0625, 1.0, -3.5, -0.0]
    codes, scales = M.quantise(f64_to_bf16(row))
    assert scales.tolist() == [127, 128]
    # 7 saturates to 6; 5 is half way between 4 and 6, 2.5 between 2 and 3, 0.25 between 0 and 0.5: the even codes
    assert codes[:8].tolist() == [7, 15, 6, 4, 0, 8 + 2, 2, 1]
    assert codes[32:36].tolist() == [6, 1, 8 + 4, 8]  # over 2: 3.53, 0.5, -1.75 (between 1.5 and 2), -0
    assert M.values(codes, scales)[:4].tolist() == [6.0, -6.0, 4.0, 2.0] and M.values(codes, scales)[32:35].tolist() == [8.0, 1.0, -4.0]
    assert M.quantise(np.full(32, 0x7F80, np.uint16))[1].tolist() == [255]


def test_oracle_rounding_is_within_half_a_step():
    rng = np.random.default_rng(0)
    bits = f64_to_bf16(rng.standard_normal((2000, 64)) * np.exp2(rng.integers(-120, 120, (2000, 1))))
    x, (codes, scales) = bf16_to_f64(bits), M.quantise(bits)
    y, step = M.values(codes, scales), np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, -1)
    size = np.abs(x) / step
    assert (np.abs(x - y) <= step * np.where(size < 2, 0.25, np.where(size < 4, 0.5, 1.0))).all()
    again = M.quantise(f64_to_bf16(y))  # what codes stand for comes back as it is
    assert np.array_equal(M.values(*again), y)


def test_oracle_places_in_a_page():
    shape = M.cache_shape(3, 2, 8, 64)
    assert shape == (3, 2, 8 * 34)
    cache = np.zeros(shape, np.uint8)
    codes, scales = np.arange(2 * 64).reshape(1, 2, 64).astype(np.uint8) % 16, np.array([[[1, 2], [3, 4]]], np.uint8)
    M.put(cache, 8, 64, [2], [5], codes, scales)
    assert cache[2, 1, 5 * 32] == 0x10 and cache[2, 1, 5 * 32 + 31] == 0xFE and cache[2, 0, 256 + 10:256 + 12].tolist() == [1, 2]
    assert np.count_nonzero(cache) == 2 * 32 + 4  # (every byte has a code that is not zero)
    got = M.get(cache, 8, 64, [2], [5])
    assert np.array_equal(got[0], codes) and np.array_equal(got[1], scales)


def test_oracle_block_tables_by_hand():
    table = np.array([[7, 8, 9], [5, 0, 0]], np.int32)
    free = np.array([1, 2, 3, -1, -1, -1], np.int32)
    got = M.block_tables([40, 16], [16, 16], [1, 20], 16, table, free, 3, 30)
    # request 0 gives its third page back, request 1 takes it and the one below it
    assert got[0].tolist() == [[7, 8, 9], [5, 9, 3]] and got[1].tolist() == [1, 2, 3, 9, -1, -1] and got[2] == 2
    assert got[3][:3].tolist() == [8 * 16, 9 * 16, 9 * 16 + 1] and got[3][21:].tolist() == [-1] * 9 and got[4].tolist() == [0, 1, 21] and got[5] == 0


def test_oracle_probabilities_by_hand():
    p = np.zeros(1, E.SAMPLING_DTYPE)
    p["temperature"], p["repetition"], p["presence"], p["frequency"], p["prompt_len"], p["history_len"], p["num_biases"] = 2, 2, 0.5, 0.25, 1, 3, 2
    logits = np.array([[1.0, -1.0, 2.0, 0.0]] * 2, np.float32)
    got, _ = M.probs([1], logits, p, np.array([[1, 2, 2]]), np.array([3], np.int32), np.array([[0, 0]]), np.array([[9.0, 1.0]]), None, None)
    soft = lambda z: np.exp(np.array(z) / 2) / np.exp(np.array(z) / 2).sum()
    # token 1 is the prompt's, token 2 was made twice, token 0 has a bias; the second row has seen token 3 too
    assert np.allclose(got[0], soft([2.0, -2.0, 1.0 - 1.0, 0.0])) and np.allclose(got[1], soft([2.0, -2.0, 0.0, -0.75]))
    mask = np.array([[0b0101]], np.uint32)
    got, _ = M.probs([0], logits[:1], np.zeros(1, E.SAMPLING_DTYPE), np.zeros((1, 0), int), [], np.zeros((1, 0), int), np.zeros((1, 0)), mask, [0])
    assert got.tolist() == [[0, 0, 1, 0]]


def test_plans_under_sanitizers(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("g++ or the HIP headers are not available")
    exe = str(tmp_path / "fuzz_mx4_plan")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
           "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(ROOT, "tests", "native", "fuzz_mx4_plan.cpp"), os.path.join(CSRC, "mx4_plan.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0 and "4-bit plan ok" in run.stdout, (run.stdout + run.stderr)[-4000:]
