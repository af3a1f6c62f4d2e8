"""Log probabilities of more rows than a launch has workgroups, each cut into parts."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import say
from tests.test_gpu_logprobs import Call, normal

pytestmark = pytest.mark.gpu


def test_more_rows_in_parts_than_workgroups_of_a_launch():
    """2^20 + 5 rows of the fewest words that are cut into parts where alternatives are wanted,
    77 GB in bf16: the same 1024 rows over and over, which begin alike within 16 bytes, so that
    every row's results are those of its first copy, bit for bit."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rows, vocab, each, top = (1 << 20) + 5, 36857, 1024, 3
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("needs 90 GiB of device memory")
    say(f"[gpu] log probabilities of {rows} rows of {vocab}")
    block = normal(each, vocab, torch.bfloat16, 7)
    tokens = torch.randint(0, vocab, (each,), dtype=torch.int32, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    few = Call(block, tokens, 0.0, top).check()
    whole = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda")
    for r in range(0, rows, each):
        whole[r:r + each] = block[:rows - r]
    of = torch.arange(rows, device="cuda") % each
    say("[gpu] a token a row")
    many = Call(whole, tokens[of], 0.0, top)
    for a, b in zip(many.results(), few.results()):
        assert torch.equal(a, b[of])
    say("[gpu] tokens that name the last rows")
    named = torch.arange(rows - 300, rows, dtype=torch.int32, device="cuda")
    got = Call(whole, tokens[of[rows - 300:]], 0.0, top, token_rows=named)
    assert torch.equal(got.logprob, few.logprob[of[rows - 300:]]) and torch.equal(got.ids, many.ids)
