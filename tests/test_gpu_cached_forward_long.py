"""dd_denoise_forward_cached over contexts long enough that attention cuts them: pieces' partial results behind the
forward pass's own workspace, and their join."""
import numpy as np
import pytest

import workloads
from paper_2609_04010_amd import _lib as dd
from tests.gpu_util import torch_or_skip
from tests.test_gpu_cached_forward import Server

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cfg,T,passes", [
    (workloads.model_cfg(1, max_len=2304), 600, [[600, 0], [550, 50], [500, 100], [1, 1], [7, 30]]),
    (workloads.model_cfg(2, n_layers=2, vocab=300, max_len=2304), 160, [[160, 0]] * 7 + [[1, 20]])], ids=["fp32", "bf16"])
def test_cut_contexts_against_oracle(cfg, T, passes):
    """Prompts in several passes; the first request passes 1024 tokens, the second stays short and whole."""
    torch = torch_or_skip()
    rng = np.random.default_rng(21)
    sv = Server(torch, cfg, 22, S=2, T=T, n_blocks=44, P=64, ld_table=36)
    assert dd.cache_attention_workspace_bytes(sv.cc, 2, T, cfg["n_heads"], T, sv.max_kv) > 0
    for i, n_new in enumerate(passes):
        sv.plan(np.array(n_new))
        z = np.where(np.arange(T) < sum(n_new), rng.integers(0, cfg["vocab"], T), -5)
        sv.forward(z, 1.0, "bidirectional" if i == len(passes) - 1 else "causal")
        sv.length.copy_(sv.m.kv_len)
    assert int(sv.length[0].item()) > 1024
