"""Calls on caches at the ends of what their lists may hold: the arithmetic on the host.  No GPU, no compute."""
import itertools

import paper_1901_06887_amd as mt
from test_lm_cache_host import sample_args
from test_lm_host import host_ctx, refused

HIGH = 2 ** 31 - 1


def test_places_of_rows_of_any_length():
    """Tokens from the first row's on, of those that the table has; none where the first row's is behind its end.  (What is walked over is rounded down to 64 and then goes on in steps of 64 up to 4096 of them: within 32
    bits only where it starts inside of the table.)"""
    ends = [0, 1, 15, 16, 63, 64, 100, 2 ** 25 - 1, 2 ** 25, 2 ** 25 + 1, 2 ** 30, HIGH - 2 ** 18, HIGH - 64, HIGH - 16, HIGH - 1, HIGH]
    for length, reach, (first, last, after) in itertools.product(ends, [16, 48, 2 ** 18, 2 ** 25],
                                                                 [(0, 1, 1), (0, 16, 16), (5, 21, 21), (0, 16, 100), (3, 40, HIGH), (HIGH - 20, HIGH - 2, HIGH), (0, HIGH, HIGH)]):
        begin, stop = max(length - (after - first), 0), min(length - (after - last), reach)
        assert mt.debug_kv_write_places(length, first, last, after, reach) == ((begin, stop) if begin < stop else (0, 0)), (length, reach, first, last, after)


def test_sampling_needs_no_scratch():
    c = host_ctx()
    for rows, classes in ((1, 1), (1, 1 << 20), (100000, 65001)):
        assert mt.sample_scratch(rows, classes) == 0
    for kw in (dict(scratch=None, scratch_bytes=0), dict(scratch=72, scratch_bytes=1)):
        refused(7, c.sample, 0, sample_args(**kw))
    c.close()
