"""Workspaces that count more bytes than they hold are refused by the batched calls before anything is launched."""
import pytest
import torch

import paper_2606_02823_b200 as qift
from test_gpu_kv4_paged import D, filled, values
from test_gpu_lora import Case

pytestmark = pytest.mark.gpu


def test_expanded_and_strided_workspaces_are_refused():
    b = filled(900, [3], [40], 2, 32)
    q = values(901, (3, 4, D), "bf16")[0]
    need = qift.qift_kv4_paged_attention_workspace_bytes(3, 1, 4, 2)
    c = Case(910, [2, 3], [0, 1], 2, 16, 256, 64, "f32")
    need = max(need, qift.qift_lora_workspace_bytes(5, 16, 256))
    one = torch.zeros(16, dtype=torch.uint8, device="cuda")
    wide = torch.zeros(2 * need, dtype=torch.uint8, device="cuda")
    for ws in (one[:1].expand(need), wide[::2]):
        with pytest.raises(AssertionError):
            qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f, workspace=ws)
        with pytest.raises(AssertionError):
            c.call(workspace=ws)
    got = qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f, workspace=wide.view(torch.int32))
    assert torch.equal(got, qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f))
