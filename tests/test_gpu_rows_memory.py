"""Whose memory joins, dropout and log probabilities take: addresses of the host's own are refused in the places that are looked at, before anything runs; pinned memory is taken."""
import numpy as np
import pytest
import torch

from paper_2608_16308_b200 import binding as B
from rows_util import DEV, Logprobs, randn

pytestmark = pytest.mark.gpu
HOST = np.zeros(4096, np.float32)
HOST = HOST[(-HOST.ctypes.data // 4) % 16:][:2048]


def refused(f, **kw):
    with pytest.raises(B.DbSpmspvError) as e:
        f(**kw)
    torch.cuda.synchronize()
    assert e.value.status == B.ERR_INVALID_ARG


@pytest.mark.parametrize("first", ["logprob", "entropy", "stats", "top_ids", "top_logprobs"])
def test_outputs_of_log_probabilities(first):
    d = torch.zeros(4096, device=DEV)
    names = ["logprob", "entropy", "stats", "top_ids", "top_logprobs"]
    for others in (False, True):              # those behind it: not wanted, or right
        kw = {k: HOST if k == first else d if others and names.index(k) > names.index(first) else None for k in names}
        refused(B.dbspmspv_logprobs, logits=d, ldl=8, logits_f32=1, tokens=2, vocab=8, temperature=1.0, targets=d, top=1 if kw["top_ids"] is not None or kw["top_logprobs"] is not None else 0, **kw)


GRADIENTS = ["dr", "db", "dw_block", "dc_block", "dgate", "dw_next", "dc_next"]


def back(norm_block=B.NORM_RMS, norm_next=B.NORM_RMS, **change):
    d = torch.zeros(1 << 16, device=DEV)
    o = B.default_join_opts()
    o.norm_block, o.norm_next, o.stream_f32, o.block_f32, o.dblock_f32 = norm_block, norm_next, 1, 1, 1
    room = B.dbspmspv_join_workspace(o, 2, 8)
    assert room <= d.numel() * 4
    kw = dict(opts=o, tokens=2, n=8, out=d, ldo=8, b=d, ldb=8, stats=d, w_block=None, c_block=None, gate=d, ldg=0, w_next=None, random=None, dh=d, lddh=8, dout=d, lddo=8, dr=None, lddr=8, db=None, lddb=8,
              dw_block=None, dc_block=None, dgate=None, lddg=0, dw_next=None, dc_next=None, workspace=d, workspace_bytes=room)
    refused(B.dbspmspv_join_backward, **{**kw, **change})


@pytest.mark.parametrize("first", GRADIENTS)
def test_outputs_of_the_gradient_of_a_join(first):
    back(**{first: HOST})
    right = torch.zeros(4096, device=DEV)
    back(**{k: HOST if k == first else right for k in GRADIENTS[GRADIENTS.index(first):]})


def test_inputs_of_the_gradient_of_a_join():
    right = torch.zeros(4096, device=DEV)
    back(dr=right, db=right, out=HOST)
    back(dr=right, db=right, dh=HOST)
    back(dr=right, db=right, dh=None, dout=HOST)
    back(dr=right, db=right, norm_next=B.NORM_NONE, out=None, b=HOST)
    back(dr=right, dh=None, b=None, stats=HOST)


def test_pinned_memory():
    l = Logprobs(randn((3, 500), 1, 3.0), 4)
    l.forward()
    torch.cuda.synchronize()
    logits, lp, ids = l.logits.v.cpu().pin_memory(), torch.zeros(3).pin_memory(), torch.zeros(12, dtype=torch.int32).pin_memory()
    B.dbspmspv_logprobs(logits, 500, 1, 3, 500, 1.0, l.targets, lp, None, None, 4, ids, None)
    torch.cuda.synchronize()
    assert torch.equal(lp, l.logprob[:3].cpu()) and torch.equal(ids, l.ids[:12].cpu())
