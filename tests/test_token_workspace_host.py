"""Workspaces of the attention with a decay for each head: what they may cost, and whom they serve.  No GPU."""
import os
import random

import pytest

from paper_2605_24584_amd import binding as B

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def library():
    if not os.path.exists(B.LIB_PATH):
        from paper_2605_24584_amd import build
        build.build()


need = B.laplex_decay_attention_workspace_bytes
TYPES = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("dtype", TYPES)
def test_many_short_sequences_need_no_state_each(dtype):
    """Only sequences of several stretches have states in the workspace."""
    for tokens, sequences, heads, d in ((65536, 4096, 16, 128), (65536, 512, 32, 128), (1 << 24, 1 << 20, 16, 128), (1 << 25, 1 << 20, 8, 256), (4096, 4096, 64, 64)):
        assert need(dtype, tokens, sequences, heads, d, d) <= 1 << 30, (tokens, sequences, heads, d)
    assert need(dtype, 64, 64, 16, 128, 128) == 0
    assert need(dtype, 0, 100, 16, 128, 128) == 0


@pytest.mark.parametrize("dtype", TYPES)
def test_a_workspace_serves_every_smaller_call(dtype):
    """A program that sizes it by its longest prompt and its largest batch has enough for the others."""
    assert need(dtype, 1408, 1, 16, 128, 128) >= need(dtype, 1344, 1, 16, 128, 128)
    r = random.Random(3)
    for _ in range(3000):
        heads, dk, dv = r.choice([1, 2, 5, 16, 64]), r.choice([8, 64, 96, 128, 200]), r.choice([32, 64, 128, 256])
        tokens, sequences = int(2 ** r.uniform(0, 22)), int(2 ** r.uniform(0, 14))
        most = need(dtype, tokens, sequences, heads, dk, dv)
        assert need(dtype, r.randint(0, tokens), sequences, heads, dk, dv) <= most
        assert need(dtype, tokens, r.randint(1, sequences), heads, dk, dv) <= most
