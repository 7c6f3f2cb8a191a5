"""The limit of the operators' bounded waits stays a limit."""
from paper_2608_15438_gb300 import neuroute as nr


def test_a_limit_past_a_minute_is_refused():
    """As nr_params.wait_limit_us is. In nanoseconds 2^62 us pass 64 bits."""
    set_limit = nr.lib().nr_ops_wait_limit
    try:
        for us in (60_000_001, 1 << 40, 1 << 62, (1 << 63) - 1):
            assert set_limit(us) == -1, us
        for us in (1, 1000, 60_000_000, -1, -(1 << 62)):
            assert set_limit(us) == 0, us
    finally:
        assert set_limit(0) == 0
