"""The cache's operators called from other host threads than the first."""
import threading

import pytest
import torch

import cache_ref as ref
from test_gpu_cache_attention import gaussian, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["attention", "key_weights", "append", "read", "evict", "norm", "status"])
def test_a_thread_whose_first_call_it_is(fd, name):
    """All memory is there: nothing but the operator itself makes the device's context current
    in the new thread."""
    cache, table = ref.make_cache(fd, [40], 2, 64, 32, seed=3)
    q, n = gaussian((1, 2, 4, 64), 5, torch.bfloat16), ints([40])
    k = gaussian((1, 3, 2, 64), 6, torch.bfloat16)
    out, lse = fd.fdllm_cache_attention(q, cache, table, n, return_lse=True)
    ws = torch.empty(fd.fdllm_cache_attention_workspace_bytes(1, 2, 4, 2, 64), dtype=torch.uint8,
                     device="cuda")
    w = fd.fdllm_cache_key_weights(q, lse, cache, table, n)
    rk, rv = torch.empty_like(k), torch.empty_like(k)
    pool, dst = fd.KvCache.empty(8, 2, 32, 64), torch.tensor([[7]], dtype=torch.int32).cuda()
    source = torch.tensor([[0, 1]], dtype=torch.int32).cuda()
    fd.fdllm_cache_append(pool, source, None, gaussian((1, 40, 2, 64), 7, torch.bfloat16),
                          gaussian((1, 40, 2, 64), 8, torch.bfloat16))
    kept = fd.fdllm_cache_evict(pool, source, n, w, 8, dst)
    got, got_lse, got_w, got_q = (torch.zeros_like(x) for x in (out, lse, w, q[0]))
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    freq = torch.ones(32, dtype=torch.float64)
    calls = {
        "attention": lambda: fd.fdllm_cache_attention(q, cache, table, n, out=got, out_lse=got_lse, workspace=ws),
        "key_weights": lambda: fd.fdllm_cache_key_weights(q, lse, cache, table, n, out=got_w),
        "append": lambda: fd.fdllm_cache_append(cache, table, None, k, k),
        "read": lambda: fd.fdllm_cache_read(cache, table, None, 3, out_k=rk, out_v=rv),
        "evict": lambda: fd.fdllm_cache_evict(pool, source, n, w, 8, dst, out_lens=kept[0],
                                              out_weights=kept[1], out_index=kept[2]),
        "norm": lambda: fd.fdllm_qk_norm_rope(q[0], None, pos, freq, out_q=got_q),
        "status": lambda: fd.fdllm_cache_status(),
    }
    errors = []

    def call():
        try:
            calls[name]()
        except Exception as e:  # a thread's exception is the test's
            errors.append(e)

    thread = threading.Thread(target=call)
    thread.start()
    thread.join()
    torch.cuda.synchronize()
    assert not errors, errors
    if name == "attention":
        assert torch.equal(got, out) and torch.equal(got_lse, lse)
    if name == "key_weights":
        assert torch.equal(got_w, w)
    if name == "norm":
        assert torch.equal(got_q, q[0])


def test_a_call_inside_another_has_a_workspace_of_its_own(fd, monkeypatch):
    """What two threads do at the worst, in one: while a call is in the library, another is made
    on the same stream.  Neither may be given the other's workspace."""
    cache, table = ref.make_cache(fd, [40], 2, 64, 32, seed=3)
    q = gaussian((1, 2, 4, 64), 5, torch.bfloat16)
    lib, seen = fd._load(), []

    class Library:
        fdllm_cache_attention_workspace_bytes = lib.fdllm_cache_attention_workspace_bytes

        def fdllm_cache_attention(self, *args):
            seen.append(args[-3])
            if len(seen) == 1:
                fd.fdllm_cache_attention(q, cache, table, ints([40]))
            return lib.fdllm_cache_attention(*args)

    monkeypatch.setattr(fd, "_load", lambda: Library())
    fd.fdllm_cache_attention(q, cache, table, ints([40]))
    assert len(seen) == 2 and seen[0] and seen[1] and seen[0] != seen[1]


def test_threads_on_one_stream(fd):
    """Four threads, each with a batch of its own whose units are cut between thread blocks."""
    work = []
    for i, (B, n) in enumerate([(1, 3000), (3, 900), (2, 1500), (5, 333)]):
        cache, table = ref.make_cache(fd, [n] * B, 2, 128, 64, seed=i)
        q = gaussian((B, 32, 4, 128), i, torch.bfloat16)
        work.append((q, cache, table, ints([n] * B)))
    want = [fd.fdllm_cache_attention(*w, return_lse=True) for w in work]
    got, errors = [[] for _ in work], []

    def many(i):
        try:
            for _ in range(200):
                got[i].append(fd.fdllm_cache_attention(*work[i], return_lse=True))
        except Exception as e:  # a thread's exception is the test's
            errors.append(e)

    threads = [threading.Thread(target=many, args=(i,)) for i in range(len(work))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for i, results in enumerate(got):
        assert len(results) == 200
        assert all(torch.equal(a, b) for r in results for a, b in zip(r, want[i]))
