"""Which kernel scores a call's tokens: those of one request share work-groups, a batch of one token each does not, whatever padded rows
it has.  (The rule is plain C++, csrc/score_route.h, built with g++ under the sanitizers.)"""
import pytest

from test_host_sanitized import exe, run  # noqa: F401


def _grouped(exe, *cases):
    out = run(exe, "".join("scores %d %d %d %d %d\n" % c for c in cases))
    assert len(out) == len(cases)
    return [int(line.split()[1]) for line in out]


@pytest.mark.parametrize("hkv,G", [(8, 4), (4, 7), (8, 1), (2, 4), (1, 16)])
@pytest.mark.parametrize("max_blocks", [300, 700, 1600, 1700, 20000])
def test_padded_rows_are_no_suffix(exe, hkv, G, max_blocks):  # noqa: F811
    """One token a request and up to a quarter of padded rows more: as without them."""
    cases = [(n + pad, n, G, hkv, max_blocks) for n in (4, 5, 32, 64, 128, 300) for pad in (0, 1, 3, n // 4)]
    assert not any(_grouped(exe, *cases))


def test_suffixes_share(exe):  # noqa: F811
    # tokens, table rows, heads a KV head, KV heads, table entries: where each was measured faster
    assert _grouped(exe, (681, 8, 4, 8, 900), (512, 8, 4, 8, 700), (64, 1, 4, 8, 1700), (64, 4, 4, 8, 1700), (128, 16, 7, 4, 1700),
                    (64, 1, 1, 8, 1700), (512, 8, 1, 8, 700), (256, 64, 4, 8, 1700)) == [1] * 8
    assert _grouped(exe, (8, 4, 4, 8, 1700), (64, 32, 4, 8, 1700), (64, 16, 4, 8, 1700), (16, 1, 4, 8, 1700), (128, 64, 7, 4, 1700),
                    (64, 4, 1, 8, 1700), (128, 16, 1, 8, 1700), (500, 5, 17, 1, 1700), (1, 0, 4, 8, 1700)) == [0] * 9


def test_no_division_by_zero_and_no_overflow(exe):  # noqa: F811
    _grouped(exe, (0, 0, 1, 1, 0), (0, 5, 4, 8, 1 << 26), (1 << 20, 8192, 1, 1 << 20, 1 << 26), (1 << 20, 1, 16, 65536, 1 << 26))
