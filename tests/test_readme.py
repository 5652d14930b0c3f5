"""The README's decode step, run with stand-ins that check what it hands on (CPU)."""
import os
import re
from unittest import mock

import torch

from paper_2401_04829_amd import answers as A

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def test_the_decode_step_attends_with_normed_queries():
    with open(README) as f:
        step, = [b for b in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "evict_tokens" in b]
    turned = torch.ones(2, 3, 8)                              # what append_tokens gives back
    lengths, positions = torch.tensor([5, 9], dtype=torch.int32), torch.tensor([700, 9], dtype=torch.int32)
    append = mock.Mock(side_effect=lambda *a, **kw: turned if kw.get("q_out") is None else kw["q_out"])
    attend = mock.Mock(return_value=("out", "lse"))
    looked = mock.Mock()
    evict = mock.Mock(return_value=("kept", "fewer", "their weights"))
    names = dict(append_tokens=append, attend=attend, q=torch.zeros(2, 3, 8), lengths=lengths, positions=positions,
                 **{n: n for n in ("cache", "k", "v", "table", "cos", "sin", "qn", "kn", "weights", "hidden", "vocabulary",
                                   "answer", "targets")})
    with mock.patch.multiple(A, attention_weights=looked, evict_tokens=evict, linear_logprobs=mock.Mock(),
                             differentiable_linear_logprobs=mock.MagicMock()):
        exec(step, names)
    assert append.call_args.kwargs["positions"] is positions  # not by the places in the cache, which eviction moves
    for call in (attend, looked):
        assert call.call_args.args[1] is turned
    assert names["lengths"] == "fewer" and names["weights"] == "their weights"
