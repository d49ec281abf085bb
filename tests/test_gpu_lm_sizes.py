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


@pytest.mark.parametrize("dv", [1, 32, 33])
def test_the_limits_of_a_launch(dv):
    """The largest numbers of sequences that the header allows, none of them with a token, and one more."""
    say(f"[sizes] limits, {dv} columns")

    def args(n_seq, heads=1):
        return csb_delta_args(type=VAL_BF16, heads_k=1, heads_v=heads, dk=16, dv=dv, n_seq=n_seq, n_tokens=0, ldq=16, ldk=16, ldv=heads * dv, ldg=heads,
                              ldbeta=heads, ldo=heads * dv, scale=1.0)
    tiles, narrow = -(-dv // 32), -(-dv // 16)
    most = ((1 << 24) - 1) // tiles
    assert lib().csb_delta_recurrent(args(most), None) == 0 and lib().csb_delta_recurrent(args(most + 1), None) == -4
    assert lib().csb_delta_recurrent(args(most // 3, 3), None) == 0 and lib().csb_delta_recurrent(args(most // 3 + 1, 3), None) == -4
    most = ((1 << 22) - 1) // narrow // 8 * 8
    assert lib().csb_delta_chunked(args(most), None, None) == 0 and lib().csb_delta_chunked(args(most + 1), None, None) == -4
    torch.cuda.synchronize()
