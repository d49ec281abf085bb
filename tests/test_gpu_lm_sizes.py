"""The chunked delta rule at sizes that it takes token by token: no workspace."""
import sys

import pytest
import torch

from paper_2005_05758_amd import delta_recurrent
from paper_2005_05758_amd.binding import VAL_BF16, VAL_F32, csb_delta_args, lib

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


@pytest.mark.parametrize("fmt,dk", [("f32", 130), ("f32", 3), ("bf16", 7)])
def test_token_by_token_without_a_workspace(fmt, dk):
    say(f"[sizes] {fmt}, rows of {dk}, no workspace")
    typ = {"f32": torch.float32, "bf16": torch.bfloat16}[fmt]
    t = torch.Generator().manual_seed(dk)
    q, k = (torch.nn.functional.normalize(torch.randn(90, 1, dk, generator=t), dim=-1).to(typ).cuda() for _ in range(2))
    v, g, beta = torch.randn(90, 2, 8, generator=t).to(typ).cuda(), -0.1 * torch.rand(90, 2, generator=t).cuda(), torch.rand(90, 2, generator=t).cuda()
    want, out = delta_recurrent(q, k, v, g, beta, scale=0.25), torch.zeros_like(v)
    args = csb_delta_args(type=VAL_F32 if fmt == "f32" else VAL_BF16, heads_k=1, heads_v=2, dk=dk, dv=8, n_seq=1, n_tokens=90, d_q=q.data_ptr(),
                          d_k=k.data_ptr(), d_v=v.data_ptr(), ldq=dk, ldk=dk, ldv=16, d_g=g.data_ptr(), d_beta=beta.data_ptr(), ldg=2, ldbeta=2, scale=0.25,
                          d_out=out.data_ptr(), ldo=16)
    assert lib().csb_delta_workspace_bytes(args) == 0
    assert lib().csb_delta_chunked(args, None, None) == 0
    torch.cuda.synchronize()
    assert torch.equal(out, want)
