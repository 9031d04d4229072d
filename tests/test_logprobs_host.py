"""How log-probabilities are cut, as their scratch memory shows it, without a GPU."""
from paper_2411_05894_amd import binding as sv


def test_parts_of_rows():
    """Parts leave their results in scratch memory, workgroups over whole rows need none: those from 769 rows on, since twice as many workgroups would not be on the chip at once."""
    size = sv.lib().sssd_op_logprobs_scratch_bytes
    for kind in (0, 1):
        assert all(size(kind, rows, 128256, 1, 1) > 0 for rows in (1, 9, 400, 767, 768))
        assert all(size(kind, rows, 128256, 1, 1) == 0 for rows in (769, 900, 1023, 1024, 1536, 1537, 5000))
        assert size(kind, 3, 2048, 1, 1) == 0 and size(kind, 3, 2049, 1, 1) > 0
