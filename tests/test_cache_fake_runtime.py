"""The cache's entry points over a stand-in for the CUDA runtime (fake_cudart.cpp): what they set
up on which device, and what they do when that fails.  No GPU; each case is a process of its own,
since the library keeps its set-up for the life of one."""
import os
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))

PRELUDE = """
import ctypes
lib, fake = ctypes.CDLL(%r), ctypes.CDLL(%r)
A16 = 0x10000  # a device pointer that nothing reads
class Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_codes", "v_codes", "k_affine", "v_affine")] + \
               [(n, ctypes.c_int) for n in ("pages", "heads", "page_size", "head_dim")]
def strides(*s):
    return (ctypes.c_int64 * len(s))(*s)
p, i, d, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_double, ctypes.c_size_t
lib.fdllm_cache_attention.argtypes = [p, p, i, i, i, i, p, p, i, p, p, p, p, p, i, p, i, d, p, p, p, sz, p]
lib.fdllm_cache_key_weights.argtypes = [p, p, i, i, i, i, p, p, i, p, p, d, p, p, i, p]
lib.fdllm_cache_evict.argtypes = [p, p, i, i, p, p, i, i, i, i, p, i, p, p, p, p]
fake.fake_map.restype = ctypes.c_ulonglong
def cache(**kw):
    f = dict(k_codes=A16, v_codes=A16, k_affine=A16, v_affine=A16, pages=4, heads=2, page_size=64, head_dim=128)
    f.update(kw)
    return Cache(**f)
def attend(c, Lq, Ln=0):
    D, h = c.head_dim, c.heads
    q, k = strides(Lq * h * D, h * D, D), strides(max(Ln, 1) * h * D, h * D, D)
    new = A16 if Ln else None
    return lib.fdllm_cache_attention(A16, q, 0, 1, Lq, h, ctypes.byref(c), A16, 4, A16, new, k, new, k, Ln,
                                     None, 0, 1.0, A16, None, A16, 1 << 40, None)
def weigh(c, Lq):
    D, h = c.head_dim, c.heads
    return lib.fdllm_cache_key_weights(A16, strides(Lq * h * D, h * D, D), 0, 1, Lq, h, ctypes.byref(c), A16, 4,
                                       A16, A16, 1.0, None, A16, 64, None)
def evict(c, max_len):
    return lib.fdllm_cache_evict(ctypes.byref(c), A16, 1, 4, A16, A16, max_len, 8, 0, 0, A16, 1, A16, A16, A16, None)
def maps():
    return [tuple([int(fake.fake_map(m, 0, 0))] + [[int(fake.fake_map(m, w, a)) for a in range(int(fake.fake_map(m, 0, 0)))]
                                                  for w in (1, 2, 3)]) for m in range(fake.fake_maps())]
"""


@pytest.fixture(scope="module")
def run(cuda_lib_path, tmp_path_factory):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    fake = str(tmp_path_factory.mktemp("fake") / "libfake_cudart.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", include,
                    os.path.join(HERE, "fake_cudart.cpp"), "-o", fake], check=True)

    def go(body):
        code = PRELUDE % (cuda_lib_path, fake) + body
        r = subprocess.run([sys.executable, "-S", "-c", code], env={**os.environ, "LD_PRELOAD": fake},
                           capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stdout + r.stderr

    return go


CALLS = ["attend(cache(), 1)", "attend(cache(), 20)", "attend(cache(), 40)", "attend(cache(head_dim=64), 40, 40)",
         "weigh(cache(), 1)", "weigh(cache(), 40)", "evict(cache(), 1000)", "evict(cache(), 20000)"]


@pytest.mark.parametrize("call", CALLS)
def test_every_device_is_set_up(run, call):
    run("""
for device in (0, 1, 0, 3):
    fake.fake_set_device(device)
    before = fake.fake_launches()
    assert %s == 0, device
    assert fake.fake_launches() > before
""" % call)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("which", [1, 2, 3, 4])
def test_a_failed_set_up_is_tried_again(run, call, which):
    """The first, second ... of a first call's set-up steps fails, once (a call that has fewer
    steps is told nothing)."""
    run("""
fake.fake_fail(%d)
first = %s
failed = fake.fake_failed()
assert first == (4 if failed else 0), first
fake.fake_fail(0)
assert [%s for _ in range(2)] == [0, 0]
""" % (which, call, call))


@pytest.mark.parametrize("page,D,pages,heads", [
    (32, 128, (1 << 20) + 1, 16),   # 73 GB: as many rows of channels as 31 bits count
    (64, 128, (1 << 20) + 1, 16), (32, 64, 1 << 25, 1), (256, 64, 1 << 20, 8), (32, 64, (1 << 31) - 1, 1),
])
def test_maps_of_large_pools(run, page, D, pages, heads):
    """Every axis of a tensor map is within 32-bit coordinates, whatever the pool's size."""
    run("""
c = cache(pages=%d, heads=%d, page_size=%d, head_dim=%d)
assert attend(c, 3) == 0 and weigh(c, 3) == 0
pages, heads, page, D = %d, %d, %d, %d
k, v, k2 = maps()
span = min(page, 128)
assert k == k2 == (3, [D // 2, page, pages * heads], [D // 2, page * D // 2, 0], [D // 2, span, 1]), k
assert v == (3, [page // 2, D, pages * heads], [page // 2, page * D // 2, 0], [span // 2, D, 1]), v
""" % ((pages, heads, page, D) * 2))


def test_more_page_heads_than_a_map_counts_are_refused(run):
    run("""
c = cache(pages=1 << 28, heads=8)
assert attend(c, 3) == 1 and weigh(c, 3) == 1 and evict(c, 100) == 1 and fake.fake_launches() == 0
""")


@pytest.mark.parametrize("rejects", [0, 1])
def test_the_decode_loops_second_capture_has_no_programmatic_edges(run, rejects):
    """Where a driver rejects programmatic edges in the loop's body, the body is captured again
    without: the forward pass's operators have to do without them too."""
    run("""
FORWARD = ctypes.CFUNCTYPE(ctypes.c_int, p, p, p, p, p)
lib.fdllm_cache_append.argtypes = [p, p, i, i, p, p, p, p, p, p, i, i, p]
lib.fdllm_cache_read.argtypes = [p, p, i, i, p, p, p, p, i, i, p]
lib.fdllm_qk_norm_rope.argtypes = [p, p, p, p, i, i, i, i, i, p, p, d, p, i, p, p, i, i, p, p, p]
lib.fdllm_decode_loop.argtypes = [i, i, i, i, i, d, i, FORWARD, p, p, p, p, i, p, p]
used = []
def forward(user, state, mask, logits, stream):
    before = fake.fake_programmatic()
    c, s = cache(), strides(256, 256, 128)
    st = [attend(c, 3), weigh(c, 3), evict(c, 1000), evict(c, 20000),
          lib.fdllm_cache_append(ctypes.byref(c), A16, 1, 4, None, None, A16, s, A16, s, 0, 3, stream),
          lib.fdllm_cache_read(ctypes.byref(c), A16, 1, 4, None, None, A16, A16, 0, 3, stream),
          lib.fdllm_qk_norm_rope(A16, strides(128, 128), None, None, 0, 4, 1, 0, 128, None, None, 0.0, A16, 1, None,
                                 (ctypes.c_double * 64)(), 64, 0, A16, None, stream)]
    used.append(fake.fake_programmatic() - before)
    return max(st)
steps = ctypes.c_int(0)
fake.fake_reject_programmatic(%d)
st = lib.fdllm_decode_loop(1, 8, 8, 512, 0, 0.75, 0, FORWARD(forward), None, A16, A16, A16, 9, ctypes.byref(steps), None)
assert st == 0 and fake.fake_instantiated() == 1, (st, used)
assert used[0] > 0 and used[1:] == [0] * %d, used
# and outside the loop they have them again
before = fake.fake_programmatic()
assert attend(cache(), 3) == 0 and fake.fake_programmatic() > before
""" % (rejects, rejects))
