"""What the library's host side checks and does before a launch, on a CPU: its objects are linked with a stand-in for the CUDA
runtime (fake_cudart.cpp) that counts launches instead of making them."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2605_23163_b200 import build, fdd

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def host_library(tmp_path_factory):
    build.build_library()
    objects = [os.path.join(build.OBJ, os.path.basename(s)[:-3] + ".o") for s in build.sources()]
    if not all(os.path.exists(o) for o in objects):
        build.build_library(force=True)
    out = str(tmp_path_factory.mktemp("host") / "libfdd_host.so")
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    cmd = ["g++", "-shared", "-fPIC", "-std=c++17", "-O1", "-I", os.path.join(cuda, "include"), os.path.join(HERE, "fake_cudart.cpp")] + objects + \
          ["-Wl,-Bsymbolic", "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    return out


@pytest.fixture
def host(host_library, monkeypatch):
    monkeypatch.setattr(fdd, "LIB_PATH", host_library)
    monkeypatch.setattr(fdd, "_lib_handle", None)
    L = fdd.lib()
    L.fake_launches.restype = ctypes.c_ulonglong
    L.fake_set_device(0)
    yield L
    L.fake_set_device(0)


class Buffers:
    """Host arrays whose addresses stand for device memory, 256-byte aligned, zeroed."""

    def __init__(self):
        self.kept = []

    def __call__(self, n):
        raw = np.zeros(n + 256, dtype=np.uint8)
        self.kept.append(raw)
        return raw.ctypes.data + (-raw.ctypes.data) % 256


HQ, HKV, DIM, BLOCK, VOCAB, CAP = 4, 2, 64, 16, 64, 256
GROUPS = CAP // 64


@pytest.fixture
def ctx(host):
    c = fdd.fdd_create(HQ, HKV, DIM, VOCAB, 1, 0, BLOCK, 8, fdd.FDD_LOGITS_F32)
    yield c
    fdd.fdd_destroy(c)


@pytest.fixture
def buf():
    return Buffers()


def _quantized(ctx, buf, n=1, length=64, cap=CAP, k=None, v=None, ek=None, ev=None):
    k, v = (p or buf(HKV * CAP * DIM) for p in (k, v))
    ek, ev = (p or buf(HKV * GROUPS) for p in (ek, ev))
    return fdd.fdd_fork_quantized(ctx, [k], [v], [ek], [ev], None, length, cap, n, range(n), [None], [None], 0)


def _plain(ctx, buf, n=1, length=64):
    return fdd.fdd_fork(ctx, [buf(2 * HKV * CAP * DIM)], [buf(2 * HKV * CAP * DIM)], None, length, CAP, n, range(n), [None], [None], 0)


def _refused(status, fn, *args, **kw):
    with pytest.raises(fdd.FddError) as e:
        fn(*args, **kw)
    assert e.value.status == status, e.value


@pytest.mark.parametrize("first", ["bits8", "bf16"])
@pytest.mark.parametrize("callback", [False, True])
def test_a_block_loop_over_prefixes_of_both_types_is_refused_before_anything_happens(host, ctx, buf, first, callback):
    sets = [_quantized(ctx, buf), _plain(ctx, buf)]
    if first == "bf16":
        sets.reverse()
    rows = 2 * BLOCK
    q, k, v, out = buf(rows * HQ * DIM * 2), buf(rows * HKV * DIM * 2), buf(rows * HKV * DIM * 2), buf(rows * HQ * DIM * 2)
    called = []
    step_fn = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p)(lambda user, t, stream: called.append(t))
    steps, left = ctypes.c_int(), ctypes.c_int()
    launched = host.fake_launches()
    status = host.fdd_decode_block(
        ctx, fdd.ptr_array(sets), 2, 1, 4, 1, *(fdd.ptr_array([x]) for x in (q, k, v, out, buf(rows * VOCAB * 4))), buf(rows * 4), buf(rows),
        fdd.i32_array([BLOCK, BLOCK]), 0.125, 0, 0.9, 1.0, 0, 0, buf(8), buf(8), ctypes.byref(steps), ctypes.byref(left),
        step_fn if callback else None, None, None)
    assert status == fdd.FDD_ERR_STATE
    assert host.fake_launches() == launched and not called


@pytest.mark.parametrize("shape,pitch,fits", [
    ((6, 2, 64), 128, True), ((6, 2, 64), 384, False), ((6, 2, 64), 256, False),     # rows as they lie, and as they do not
    ((1, 2, 64), 384, True),                                                         # one row has no pitch
    ((2, 3, 2, 64), 128, True), ((2, 3, 2, 64), 384, True), ((2, 3, 2, 64), 256, False),
    ((1, 6, 2, 64), 384, False), ((6, 128), 128, True), ((768,), 384, False),
])
def test_the_stated_pitch_of_contiguous_rows_is_theirs(shape, pitch, fits):
    import torch
    t = torch.zeros(shape, dtype=torch.bfloat16)
    if fits:
        assert fdd._rows_ptr(t, pitch).value == t.data_ptr()
        return
    beside = t.as_strided((1, *shape), (pitch, *t.stride()))       # (the stride of a dimension of one entry says nothing)
    assert beside.is_contiguous()
    with pytest.raises(ValueError):
        fdd._rows_ptr(beside, pitch)
    with pytest.raises(ValueError):
        fdd._rows_ptr(t, pitch)
    for call in (lambda: fdd.fdd_prefix_write(None, [], 0, t, t, [1], pitch, 0, stream=0),
                 lambda: fdd.fdd_prefix_read(None, None, 0, 0, 1, t, t, pitch, stream=0)):
        with pytest.raises(ValueError):
            call()


def test_calls_on_8_bit_prefixes_and_scores_want_the_contexts_device_to_be_current(host, ctx, buf):
    fs = _quantized(ctx, buf)
    rows = buf(8 * HKV * DIM * 2)
    calls = (
        lambda: fdd.fdd_prefix_write(ctx, [fs], 0, rows, rows, [8], HKV * DIM, 1, stream=0),
        lambda: fdd.fdd_prefix_extend(ctx, [fs], 0, rows, rows, [8], 1, stream=0),
        lambda: fdd.fdd_prefix_read(ctx, fs, 0, 0, 8, rows, rows, HKV * DIM, stream=0),
        lambda: host.fdd_score_tokens(ctx, buf(VOCAB * 4), buf(4), None, 1, 0, buf(4), None, None, None, None),
    )
    host.fake_set_device(1)
    launched = host.fake_launches()
    for call in calls[:3]:
        _refused(fdd.FDD_ERR_STATE, call)
    assert calls[3]() == fdd.FDD_ERR_STATE
    assert host.fake_launches() == launched and fdd.fdd_forkset_prefix_len(fs) == 64
    host.fake_set_device(0)
    for call in calls:
        assert call() == fdd.FDD_OK
    assert host.fake_launches() == launched + 4 and fdd.fdd_forkset_prefix_len(fs) == 80


@pytest.mark.parametrize("shared", ["k", "v", "ek", "ev", "k of one, v of the other", "ek of one, ev of the other"])
def test_sets_that_share_any_array_of_a_contiguous_cache_are_not_written_in_one_call(host, ctx, buf, shared):
    arrays = [dict(k=buf(HKV * CAP * DIM), v=buf(HKV * CAP * DIM), ek=buf(HKV * GROUPS), ev=buf(HKV * GROUPS)) for _ in range(2)]
    if " of one" in shared:
        arrays[1][shared.split(", ")[1].split()[0]] = arrays[0][shared.split()[0]]
    else:
        arrays[1][shared] = arrays[0][shared]
    sets = [_quantized(ctx, buf, **a) for a in arrays]
    rows = buf(16 * HKV * DIM * 2)
    launched = host.fake_launches()
    _refused(fdd.FDD_ERR_STATE, fdd.fdd_prefix_write, ctx, sets, 0, rows, rows, [8, 8], HKV * DIM, 1, stream=0)
    _refused(fdd.FDD_ERR_STATE, fdd.fdd_prefix_extend, ctx, sets, 0, rows, rows, [8, 8], 1, stream=0)
    assert host.fake_launches() == launched
    fdd.fdd_prefix_write(ctx, sets, 0, rows, rows, [8, 0], HKV * DIM, 1, stream=0)       # one of them alone
    assert host.fake_launches() == launched + 1


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("shared", [("k", "v"), ("ek", "ev")])
def test_a_set_whose_k_and_v_are_one_array_is_not_written(host, buf, page, shared):
    c = fdd.fdd_create(HQ, HKV, DIM, VOCAB, 1, page, BLOCK, 8, fdd.FDD_LOGITS_F32)
    try:
        a = dict(k=buf(HKV * CAP * DIM), v=buf(HKV * CAP * DIM), ek=buf(HKV * GROUPS), ev=buf(HKV * GROUPS))
        a[shared[1]] = a[shared[0]]
        table = buf(4 * GROUPS) if page else None
        fs = fdd.fdd_fork_quantized(c, [a["k"]], [a["v"]], [a["ek"]], [a["ev"]], table, 64, GROUPS if page else CAP, 1, [0], [None], [None], 0)
        rows = buf(8 * HKV * DIM * 2)
        launched = host.fake_launches()
        _refused(fdd.FDD_ERR_STATE, fdd.fdd_prefix_write, c, [fs], 0, rows, rows, [8], HKV * DIM, 1, stream=0)
        _refused(fdd.FDD_ERR_STATE, fdd.fdd_prefix_extend, c, [fs], 0, rows, rows, [8], 1, stream=0)
        assert host.fake_launches() == launched
        fdd.fdd_prefix_read(c, fs, 0, 0, 8, rows, rows, HKV * DIM, stream=0)             # reading is no matter
    finally:
        fdd.fdd_destroy(c)


def test_paged_sets_may_share_a_pool(host, buf):
    c = fdd.fdd_create(HQ, HKV, DIM, VOCAB, 1, 64, BLOCK, 8, fdd.FDD_LOGITS_F32)
    try:
        k, v, ek, ev = buf(HKV * CAP * DIM), buf(HKV * CAP * DIM), buf(HKV * GROUPS), buf(HKV * GROUPS)
        sets = [fdd.fdd_fork_quantized(c, [k], [v], [ek], [ev], buf(4 * GROUPS), 64, GROUPS, 1, [0], [None], [None], 0) for _ in range(2)]
        rows = buf(16 * HKV * DIM * 2)
        fdd.fdd_prefix_write(c, sets, 0, rows, rows, [8, 8], HKV * DIM, 1, stream=0)
        assert [fdd.fdd_forkset_prefix_len(fs) for fs in sets] == [72, 72]
    finally:
        fdd.fdd_destroy(c)


MOST = 2 ** 31 - 128             # tokens of a prefix


def test_prefixes_end_where_their_tiles_can_still_be_counted(host, buf):
    for page in (0, 64):
        c = fdd.fdd_create(HQ, 1, DIM, VOCAB, 1, page, BLOCK, 8, fdd.FDD_LOGITS_F32)
        try:
            k, v, ek, ev, table, rows = (buf(4096) for _ in range(6))
            caps = [2 ** 25, 2 ** 31 - 1] if page else [2 ** 31 - 1]

            def fork8(length, cap):
                return fdd.fdd_fork_quantized(c, [k], [v], [ek], [ev], table if page else None, length, cap, 1, [0], [None], [None], 0)

            def fork16(length, cap):
                return fdd.fdd_fork(c, [k], [v], table if page else None, length, cap, 1, [0], [None], [None], 0)

            for fork in (fork8, fork16):
                for cap in caps + [4]:
                    for length in (MOST + 1, 2 ** 31 - 64, 2 ** 31 - 1):
                        _refused(fdd.FDD_ERR_CAPACITY, fork, length, cap)
                for cap in caps:
                    fs = fork(MOST - 8, cap)
                    launched = host.fake_launches()
                    _refused(fdd.FDD_ERR_CAPACITY, fdd.fdd_prefix_extend, c, [fs], 0, rows, rows, [9], 1, stream=0)
                    if fork is fork8:
                        _refused(fdd.FDD_ERR_CAPACITY, fdd.fdd_prefix_write, c, [fs], 0, rows, rows, [9], DIM, 1, stream=0)
                    assert host.fake_launches() == launched
                    fdd.fdd_prefix_extend(c, [fs], 0, rows, rows, [8], 1, stream=0)
                    assert fdd.fdd_forkset_prefix_len(fs) == MOST and host.fake_launches() == launched + 1
        finally:
            fdd.fdd_destroy(c)
