"""A wait of a grouped product that runs out ends in REGIONE_DEV_TIMEOUT and makes the other roles give up.

In the harmless form: a self-test kernel calls the wait routines of the product's roles on a barrier that nothing arrives on, with
nothing in flight."""
import pytest

from paper_2510_25590_b200 import binding


@pytest.mark.gpu
@pytest.mark.parametrize("limit", [100_000, 1_000_000])
def test_expired_waits_report_timeout_and_return(limit):
    import torch
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((3, 3), -1, dtype=torch.int64, device="cuda")
    binding.selftest_grouped_wait(limit, st, out)
    torch.cuda.synchronize()
    assert int(st[0]) == binding.DEV_TIMEOUT
    lone, pair, told = out.cpu().tolist()
    for done, spent, aborted in (lone, pair):
        assert done == 0 and aborted == 1 and limit <= spent <= limit + 1_000_000
    assert told[0] == 0 and told[2] == 1 and told[1] <= 1_000_000          # (its own limit is a thousand times the others')
    st.zero_()
    assert int(torch.arange(1000, device="cuda").sum()) == 499500 and int(st[0]) == 0


def test_limits():
    for limit in (0, -1, 10 ** 6 + 1):
        assert binding.load().regione_selftest_grouped_wait(limit, None, None, None) == binding.INVALID_ARG
