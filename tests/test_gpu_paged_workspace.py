"""One workspace for calls over both kinds of pages, one after another: the first 32 KB of it, where parts that meet are counted, hold counters
and nothing else, whichever call comes first."""
import pytest
import torch

from e4m3 import Batch8
from paged import DEV, Batch

pytestmark = pytest.mark.gpu

COUNTERS = 2 * 2048 * 8
BATCHES = [   # calls whose parts meet
    ([1], [9000], 8, 2, 128), ([1, 1, 1], [3000, 50, 2100], 8, 8, 64), ([4], [5000], 32, 8, 128), ([60], [2000], 8, 2, 128), ([300], [2100], 4, 1, 64)]


def _counters_alone(ws):
    words = ws[:COUNTERS].view(torch.int64)
    words = words[words != 0]
    assert len(words) > 0
    assert (words & 0xffff == 0).all()                       # a counter is reset by the last part; its upper 48 bits are a call's
    return {int(w) for w in words}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", [Batch, Batch8])
@pytest.mark.parametrize("at", range(len(BATCHES)))
def test_only_counters_where_counters_are(dtype, kind, at):
    new, lens, heads, heads_kv, d = BATCHES[at]
    b = kind(new, lens, heads, heads_kv, d, dtype, 16, seed=at)
    ws = torch.zeros_like(b.workspace())
    O, _ = b.attend(lse=False, workspace=ws)
    assert (ws[COUNTERS:] != 0).any()                         # (parts did meet)
    assert len(_counters_alone(ws)) == 1
    assert torch.equal(b.attend(lse=False)[0], O)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_both_calls_in_turn(dtype):
    calls = [kind(*BATCHES[at][:5], dtype, 16, seed=at) for at in range(len(BATCHES)) for kind in (Batch, Batch8)]
    want = [b.attend(lse=False)[0] for b in calls]
    ws = torch.zeros(max(b.workspace().numel() for b in calls), dtype=torch.uint8, device=DEV)
    tags = 0
    for _ in range(2):
        for b, O in zip(calls, want):
            assert torch.equal(b.attend(lse=False, workspace=ws)[0], O)
            tags = max(tags, len(_counters_alone(ws)))
    assert tags > 1
