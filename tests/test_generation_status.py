"""The status word of the candidate generator's operators: the header's bits, the binding's, and what check_status says."""
import os
import re

import pytest

torch = pytest.importorskip("torch")

from paper_2603_02565_gb300 import binding as B, check_status  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_bits_are_the_headers():
    text = open(os.path.join(ROOT, "include", "fe.h")).read()
    bits = {n: int(v) for n, v in re.findall(r"\b(FE_ST_\w+) = (\d+)", text)}
    assert bits == {n: v for n, v in vars(B).items() if n.startswith("FE_ST_")}
    # every one of them is set by an operator
    sources = "".join(open(os.path.join(ROOT, "paper_2603_02565_gb300", "csrc", f)).read()
                      for f in ("fe_append.cu", "fe_prefix.cu", "fe_policy.cu", "fe_common.cuh"))
    for n in bits:
        assert n in sources or n[3:] in sources, n


@pytest.mark.parametrize("word,code", [(1, B.FE_ERR_INDEX), (4, B.FE_ERR_TIMEOUT), (5, B.FE_ERR_TIMEOUT)])
def test_reported(word, code):
    with pytest.raises(B.FeError) as e:
        check_status(torch.tensor([word], dtype=torch.int32))
    assert e.value.code == code


def test_nothing_reported():
    check_status(torch.zeros(1, dtype=torch.int32))
