"""The logits' choice handed over among as many workgroups of a row as a launch of
the smallest chunks has, and one chunk more, where the chunks grow fourfold."""
import pytest
import torch

from paper_2608_15383_amd import api
from tests.test_gpu_serving import ids

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,elements", [(torch.float32, 1024), (torch.bfloat16, 2048)])
@pytest.mark.parametrize("rows,chunks", [(1, 2044), (1, 2045), (4, 508), (4, 513)])
def test_most_chunks_of_a_row(kind, elements, rows, chunks):
    """Whichever chunk holds the largest logit; the id before it is the largest until a penalty."""
    vocab = elements * chunks
    x = torch.zeros(rows, vocab, device="cuda:0", dtype=kind)
    nt = torch.empty(rows, dtype=torch.int32, device="cuda:0")
    ws = torch.zeros(api.process_logits_workspace_bytes(rows, vocab), dtype=torch.uint8, device="cuda:0")
    out, half = torch.empty_like(x), torch.full((rows,), 2.0, device="cuda:0")
    for chunk in (0, 1, 255, 256, chunks // 2, chunks - 2, chunks - 1):
        at = [(chunk * elements + 77 * r + elements - 1) % vocab for r in range(rows)]
        for r, v in enumerate(at):
            x[r, v], x[r, v - 1] = 3.0, 4.0
        api.process_logits(x, out, ws, history=ids([[v - 1, -1] for v in at]), repetition=half, next_token=nt)
        torch.cuda.synchronize()
        assert nt.tolist() == at and not ws.any()
        for r, v in enumerate(at):
            assert float(out[r, v - 1]) == 2.0
        x.zero_()
