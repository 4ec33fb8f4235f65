"""Drafting's entry points on the host (no GPU): refusals before anything touches the device, sizes
of workspaces, and set-up on each device over a stand-in for the CUDA runtime."""
import ctypes
import math

import pytest

from test_cache_fake_runtime import run  # noqa: F401  (a fixture)
from test_cache_host import cache, strides

OK, ERR_ARG, ERR_ALIGN, ERR_WORKSPACE = 0, 1, 2, 5
A16, A2 = 0x10000, 0x10002  # fake, never dereferenced
P, I, D, SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_double, ctypes.c_size_t


@pytest.fixture(scope="module")
def lib(cuda_lib_path):
    lib = ctypes.CDLL(cuda_lib_path)
    lib.fdllm_tree_mask.argtypes = [P, P, I, I, P, P, P]
    lib.fdllm_cache_tree_attention.argtypes = [P, P, I, I, I, I, P, P, I, P, P, P, P, P, I, P, P, D, P, P, P, SZ, P]
    lib.fdllm_verify_draft.argtypes = [P, P, P, P, I, I, I, I, P, P, P, D, D, P, P, P, P, P, P, SZ, P]
    lib.fdllm_verify_draft_workspace_bytes.argtypes = [I, I, I, I]
    lib.fdllm_verify_draft_workspace_bytes.restype = SZ
    lib.fdllm_distill_loss.argtypes = [P, I, I, I, I, P, P, P, I, I, P, D, P, P, P]
    lib.fdllm_distill_grad.argtypes = [P, I, I, I, I, P, P, P, I, I, P, D, P, P, P, P]
    lib.fdllm_distill_step.argtypes = [P, I, I, I, I, P, P, P, I, I, P, D, P, P, P, P]
    return lib


@pytest.mark.parametrize("change", [dict(parents=None), dict(out=None), dict(B=0), dict(B=65536), dict(M=0),
                                    dict(M=1025)])
def test_tree_mask_refuses(lib, change):
    a = {**dict(parents=A16, B=2, M=3, out=A16), **change}
    assert lib.fdllm_tree_mask(a["parents"], None, a["B"], a["M"], a["out"], None, None) == ERR_ARG


def verify(lib, **change):
    a = {**dict(target=A16, draft=A16, dtype=0, B=2, M=3, V=100, tokens=A16, parents=None, t=1.0, td=1.0, u=A16,
                e=A16, out=A16, nodes=A16, n=A16, ws=A16, size=1 << 20, ts=strides(300, 100),
                ds=strides(200, 100)), **change}
    return lib.fdllm_verify_draft(a["target"], a["ts"], a["draft"], a["ds"], a["dtype"], a["B"], a["M"], a["V"], a["tokens"],
                                  a["parents"], None, a["t"], a["td"], a["u"], a["e"], a["out"], a["nodes"],
                                  a["n"], a["ws"], a["size"], None)


@pytest.mark.parametrize("change,want", [
    (dict(target=None), ERR_ARG), (dict(dtype=3), ERR_ARG), (dict(B=0), ERR_ARG), (dict(B=65536), ERR_ARG),
    (dict(M=0), ERR_ARG), (dict(M=1025), ERR_ARG), (dict(V=0), ERR_ARG), (dict(V=(1 << 20) + 1), ERR_ARG),
    (dict(tokens=None), ERR_ARG), (dict(parents=A16), ERR_ARG), (dict(t=0.0), ERR_ARG), (dict(t=-1.0), ERR_ARG),
    (dict(t=math.nan), ERR_ARG), (dict(t=math.inf), ERR_ARG), (dict(t=1e-7), ERR_ARG), (dict(td=0.0), ERR_ARG),
    (dict(td=math.nan), ERR_ARG), (dict(u=None), ERR_ARG), (dict(e=None), ERR_ARG), (dict(out=None), ERR_ARG),
    (dict(nodes=None), ERR_ARG), (dict(n=None), ERR_ARG), (dict(target=A16 + 1), ERR_ALIGN), (dict(draft=A16 + 1), ERR_ALIGN),
    (dict(target=A2, dtype=1), ERR_ALIGN), (dict(ts=None), ERR_ARG), (dict(ds=None), ERR_ARG), (dict(ws=None), ERR_WORKSPACE), (dict(ws=A16 + 16), ERR_WORKSPACE),
    (dict(size=8), ERR_WORKSPACE)])
def test_verify_refuses(lib, change, want):
    assert verify(lib, **change) == want


def test_verify_workspace(lib):
    size = lib.fdllm_verify_draft_workspace_bytes
    assert 0 < size(1, 1, 1, 0) <= size(64, 9, 126464, 0) and size(64, 9, 126464, 0) % 256 == 0
    for bad in ((0, 1, 1, 0), (1, 1025, 1, 0), (1, 1, (1 << 20) + 1, 0), (1, 1, 1, 7)):
        assert size(*bad) == 0
    need = size(2, 3, 100, 0)
    assert verify(lib, size=need - 1) == ERR_WORKSPACE


def distill(lib, which, **change):
    a = {**dict(x=A16, dtype=0, B=2, L=3, V=100, mask=A16, index=A16, top=A16, td=1, K=4, t=1.0, loss=A16,
                stats=A16, g=A16, dx=A16), **change}
    head = (a["x"], a["dtype"], a["B"], a["L"], a["V"], a["mask"], a["index"], a["top"], a["td"], a["K"], None, a["t"])
    if which == "loss":
        return lib.fdllm_distill_loss(*head, a["loss"], a["stats"], None)
    if which == "grad":
        return lib.fdllm_distill_grad(*head, a["stats"], a["g"], a["dx"], None)
    return lib.fdllm_distill_step(*head, a["g"], a["loss"], a["dx"], None)


@pytest.mark.parametrize("which", ["loss", "grad", "step"])
@pytest.mark.parametrize("change,want", [
    (dict(x=None), ERR_ARG), (dict(dtype=-1), ERR_ARG), (dict(td=5), ERR_ARG), (dict(B=0), ERR_ARG),
    (dict(L=0), ERR_ARG), (dict(B=1 << 16, L=1 << 15), ERR_ARG), (dict(V=0), ERR_ARG),
    (dict(V=(1 << 20) + 1), ERR_ARG), (dict(K=0), ERR_ARG), (dict(K=1025), ERR_ARG), (dict(mask=None), ERR_ARG),
    (dict(index=None), ERR_ARG), (dict(top=None), ERR_ARG), (dict(t=0.0), ERR_ARG), (dict(t=math.nan), ERR_ARG),
    (dict(t=1e7), ERR_ARG), (dict(x=A2), ERR_ALIGN)])
def test_distill_refuses(lib, which, change, want):
    assert distill(lib, which, **change) == want


@pytest.mark.parametrize("which,change,want", [
    ("loss", dict(loss=None), ERR_ARG), ("loss", dict(stats=A16 + 4), ERR_ALIGN), ("grad", dict(stats=None), ERR_ARG),
    ("grad", dict(stats=A16 + 4), ERR_ALIGN), ("grad", dict(g=None), ERR_ARG), ("grad", dict(dx=None), ERR_ARG),
    ("grad", dict(dx=A2), ERR_ALIGN), ("step", dict(g=None), ERR_ARG), ("step", dict(loss=None), ERR_ARG),
    ("step", dict(dx=None), ERR_ARG), ("step", dict(dx=A2), ERR_ALIGN)])
def test_distill_refuses_its_outputs(lib, which, change, want):
    assert distill(lib, which, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(q=None), ERR_ARG), (dict(mask=None), ERR_ARG), (dict(dtype=1), ERR_ARG), (dict(Hq=3), ERR_ARG),
    (dict(scale=math.nan), ERR_ARG), (dict(k=None), ERR_ARG), (dict(Ln=-1), ERR_ARG), (dict(q=A2), ERR_ALIGN),
    (dict(k=A2), ERR_ALIGN), (dict(ws=None), ERR_WORKSPACE), (dict(size=64), ERR_WORKSPACE)])
def test_tree_attention_refuses(lib, change, want):
    a = {**dict(q=A16, dtype=0, Hq=4, mask=A16, k=A16, Ln=3, scale=1.0, ws=A16, size=1 << 30), **change}
    s, own = strides(3 * 512, 512, 128), strides(3 * 256, 256, 128)
    assert lib.fdllm_cache_tree_attention(
        a["q"], s, a["dtype"], 1, 3, a["Hq"], ctypes.byref(cache()), A16, 4, A16, a["k"], own, A16, own, a["Ln"],
        None, a["mask"], a["scale"], A16, None, a["ws"], a["size"], None) == want


MORE = """
lib.fdllm_tree_mask.argtypes = [p, p, i, i, p, p, p]
lib.fdllm_cache_tree_attention.argtypes = [p, p, i, i, i, i, p, p, i, p, p, p, p, p, i, p, p, d, p, p, p, sz, p]
lib.fdllm_verify_draft.argtypes = [p, p, p, p, i, i, i, i, p, p, p, d, d, p, p, p, p, p, p, sz, p]
lib.fdllm_distill_loss.argtypes = [p, i, i, i, i, p, p, p, i, i, p, d, p, p, p]
lib.fdllm_distill_step.argtypes = [p, i, i, i, i, p, p, p, i, i, p, d, p, p, p, p]
def mask(M):
    return lib.fdllm_tree_mask(A16, None, 1, M, A16, A16, None)
def tree(M, D):
    c, h = cache(head_dim=D), 2
    s = strides(M * h * D, h * D, D)
    return lib.fdllm_cache_tree_attention(A16, s, 0, 1, M, h, ctypes.byref(c), A16, 4, A16, A16, s, A16, s, M, None,
                                          A16, 1.0, A16, None, A16, 1 << 40, None)
def verify(M, V, dtype, t=1.0):
    return lib.fdllm_verify_draft(A16, strides(M * V, V), None, None, dtype, 2, M, V, A16, None, None, t, 1.0, A16, A16, A16, A16, A16, A16,
                                  1 << 40, None)
def loss(V, dtype):
    return lib.fdllm_distill_loss(A16, dtype, 2, 3, V, A16, A16, A16, 1, 4, None, 1.0, A16, A16, None)
def step(V, dtype):
    return lib.fdllm_distill_step(A16, dtype, 2, 3, V, A16, A16, A16, 1, 4, None, 1.0, A16, A16, A16, None)
"""
CALLS = ["mask(3)", "mask(1024)", "tree(1, 128)", "tree(20, 64)", "tree(40, 128)", "verify(1, 100, 0)",
         "verify(5, 126464, 1)", "verify(5, 126464, 2, 0.0)", "loss(126464, 0)", "step(101, 1)", "step(126464, 2)"]


@pytest.mark.parametrize("call", CALLS)
def test_every_device_is_set_up(run, call):  # noqa: F811
    run(MORE + """
for device in (0, 1, 0, 3):
    fake.fake_set_device(device)
    before = fake.fake_launches()
    assert %s == 0, device
    assert fake.fake_launches() > before
""" % call)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("which", [1, 2, 3, 4])
def test_a_failed_set_up_is_tried_again(run, call, which):  # noqa: F811
    run(MORE + """
fake.fake_fail(%d)
first = %s
failed = fake.fake_failed()
assert first == (4 if failed else 0), first
fake.fake_fail(0)
assert [%s for _ in range(2)] == [0, 0]
""" % (which, call, call))
