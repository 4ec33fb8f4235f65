"""The cache's operators as part of the forward pass of fdllm_decode_loop: captured into the
loop's graph and replayed at every step."""
import numpy as np
import pytest
import torch

import cache_ref as ref
import fdllm_synth as syn
import oracle
from test_gpu_cache_attention import gaussian, ints
from test_gpu_decode_loop import clean_seed

pytestmark = pytest.mark.gpu


def test_operators_in_the_decode_loops_forward_pass(fd, orc):
    B, gen, Lb, V, heads, D = 2, 32, 8, 512, 2, 64
    seed, want = clean_seed(orc, B, gen, Lb, V, oracle.PROFILE, 1.0, 16.0)
    lens = [300, 45]
    cache, table = ref.make_cache(fd, lens, heads, D, 32, seed=9, min_pages=12)
    n, width = ints(lens), table.shape[1] * 32
    qkv = gaussian((B * Lb, 3 * heads, D), 1, torch.bfloat16)
    pos = torch.arange(B * Lb, dtype=torch.int32, device="cuda")
    freq = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))
    q, k = (torch.empty(B * Lb, heads, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    v = qkv[:, 2 * heads:].unflatten(0, (B, Lb))
    out, lse = torch.empty(B, Lb, heads, D, dtype=torch.bfloat16, device="cuda"), torch.empty(B, Lb, heads, device="cuda")
    ws = torch.empty(fd.fdllm_cache_attention_workspace_bytes(B, Lb, heads, heads, D), dtype=torch.uint8,
                     device="cuda")
    weights = torch.zeros(B, heads, width, device="cuda")
    pool, kept_table = fd.KvCache.empty(64, heads, 32, D), (40 + torch.arange(4, dtype=torch.int32)).view(2, 2).cuda()
    pool_table = torch.arange(4, dtype=torch.int32).view(2, 2).cuda()
    back = [torch.empty(B, Lb, heads, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kept = [torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, heads, 4, device="cuda"),
            torch.empty(B, heads, 4, dtype=torch.int32, device="cuda")]
    eight = ints([Lb, Lb])

    def step(stream):
        fd.fdllm_qk_norm_rope(qkv[:, :heads], qkv[:, heads:2 * heads], pos, freq, out_q=q, out_k=k, stream=stream)
        q4, k4 = q.unflatten(0, (B, Lb)), k.unflatten(0, (B, Lb))
        fd.fdllm_cache_attention(q4, cache, table, n, k4, v, out=out, out_lse=lse, workspace=ws, stream=stream)
        fd.fdllm_cache_key_weights(q4, lse, cache, table, n, weights=weights, out=weights, stream=stream)
        fd.fdllm_cache_append(pool, pool_table, None, k4, v, stream=stream)
        fd.fdllm_cache_read(pool, pool_table, None, Lb, out_k=back[0], out_v=back[1], stream=stream)
        fd.fdllm_cache_evict(pool, pool_table, eight, weights, 4, kept_table, out_lens=kept[0],
                             out_weights=kept[1], out_index=kept[2], stream=stream)

    buf = torch.empty((B, Lb, V), dtype=torch.bfloat16, device="cuda")

    def forward(state, mask, logits, stream):
        step(stream)
        syn.synth_block_logits_gpu(logits, mask, B, Lb, V, seed, step_ptr=state, peak_max=16.0, stream_ptr=stream)

    results = (out, lse, weights, *back, *kept)
    for _ in range(want["steps"]):  # (also each operator's first call on the device)
        step(None)
    eager = [r.clone() for r in results]
    weights.zero_()
    for r in results:
        r.zero_()
    seq, nfe, steps = fd.fdllm_decode_loop(forward, buf, gen, 1.0, fd.PROFILE)
    assert steps == want["steps"] and np.array_equal(seq.cpu().numpy(), want["seq"])
    assert np.array_equal(nfe.cpu().numpy(), want["nfe"])
    assert bool((weights > 0).any())
    for a, b in zip(results, eager):  # the weights were added to at every step
        assert torch.equal(a, b)
    assert fd.fdllm_cache_status() == 0
