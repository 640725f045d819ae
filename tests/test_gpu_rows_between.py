"""What lies between rows, in front of the first and behind the last is neither used nor written: NaN there stays there and reaches no result."""
import pytest
import torch

import rows_util
from rows_util import Join, Logprobs, Rows, order, randn

pytestmark = pytest.mark.gpu


@pytest.fixture
def nan_between(monkeypatch):
    class Between(Rows):
        def __init__(self, *args, **kw):
            super().__init__(*args, **kw)
            self.buf[~self.inside] = float("nan")

        def untouched(self):
            return bool(torch.isnan(self.buf[~self.inside]).all())

    monkeypatch.setattr(rows_util, "Rows", Between)


@pytest.mark.parametrize("pad,lead", [(1, 1), (3, 5), (8, 8), (8, 1)])
@pytest.mark.parametrize("t,n", [(1, 7), (5, 264), (40, 1037), (300, 520), (9, 4099), (4, 9001)])
@pytest.mark.parametrize("wide", [False, True])
def test_joins(nan_between, t, n, pad, lead, wide):
    j = Join(t, n, "layer", "rms", c=True, gate="shared", drop=0.1, stream=wide, blk=wide, dblk=wide, pad=pad, lead=lead, seed=n)
    j.forward()
    j.backward()
    torch.cuda.synchronize()
    j.check(), j.check_back()


@pytest.mark.parametrize("pad,lead", [(1, 1), (3, 5), (8, 8), (8, 1)])
@pytest.mark.parametrize("t,vocab", [(1, 5), (4, 519), (3, 20001), (300, 3001)])
@pytest.mark.parametrize("f32", [False, True])
def test_log_probabilities(nan_between, t, vocab, f32, pad, lead):
    l = Logprobs(randn((t, vocab), vocab, 3.0), 4, 0.7, pad=pad, lead=lead, f32=f32)
    l.forward()
    l.backward(dlogprob=randn((t,), 1).float(), dentropy=randn((t,), 2).float(), dtop=randn((t, 4), 3).float(), ids=order(l.logits.v)[:, :4].to(torch.int32).contiguous())
    torch.cuda.synchronize()
    l.check(), l.check_back()
