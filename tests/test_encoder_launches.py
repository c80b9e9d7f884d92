"""CPU tests of the rules that cut the encoder's calls into launches (csrc/encoder_rules.h)."""
from test_encoder_rules import ask  # noqa: F401


def test_no_launch_has_more_threads_than_the_runtime_takes(ask):
    """The norm's and the quantizer's rows go in launches of fewer than 2^32 threads that cover them all, up to the most rows
    that there may be; a product is cut so that its launch is such a one wherever some cut is."""
    rows = [1, 2 ** 24 - 2, 2 ** 24 - 1, 2 ** 24, 2 ** 26 - 4, 2 ** 26 - 3, 2 ** 26, 2 ** 31 - 256]
    got = iter(ask("\n".join("for (int64_t done = 0, n; done < %dLL; done += n) { n = rows_of_launch(%dLL - done, %d); put((double)n); if (n < 1) break; } "
                             "put(-1);" % (n, n, per) for n in rows for per in (1, 4))))
    for n in rows:
        for per in (1, 4):
            launches = list(iter(lambda: int(next(got)), -1))
            assert all(-(-x // per) * 256 < 2 ** 32 for x in launches) and all(x % per == 0 for x in launches[:-1])
            assert len(launches) == -(-n // (per * (2 ** 24 - 1)))
    sizes = [(2 ** 31 - 256, 1, 1), (2 ** 31 - 256, 200, 64), (2 ** 30, 64, 64), (2 ** 29, 65, 1), (2 ** 22, 2 ** 22, 1)]
    got = iter(ask("\n".join("{ const int64_t m = %d, n = %d, k = %d; const Cut c = cut_of(m, n, k, false); put(launchable(c)); "
                             "const Both b = direct_both(m, n, k, false); put(direct_forward(m, n, k, false)); "
                             "put(launchable(direct_cut_of(m, n, ceil_div(k, DIRECT_STAGE), false))); put(direct_backward(m, n, k, false)); "
                             "put(grid_of(b.first) + grid_of(b.second) <= MOST_WORKGROUPS); }" % size for size in sizes)))
    for m, n, k in sizes:
        fits, forward, forward_fits, backward, backward_fits = (bool(next(got)) for _ in range(5))
        assert fits == (-(-m // 256) * -(-n // 256) <= 2 ** 24 - 8), (m, n, k)
        assert forward_fits or not forward, (m, n, k)
        assert backward_fits or not backward, (m, n, k)
