"""What products in MX4 launch: every tile once, in launches that the GPU takes; the kernels that the GPU tests' sizes are meant for."""
import pytest

import mx4_cases as cases
from mx4_launches import BF16, F32, MX4, build, launches


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = build(tmp_path_factory.mktemp("launches"))
    if not exe:
        pytest.skip("no HIP-aware clang++ in this image")
    return lambda sizes: launches(exe, sizes)


# (rows, experts, channels, width, gated, out); the last ones want 2^24 workgroups and more, which were one launch of 2^32 work-items and more
SIZES = [(1, 0, 4096, 4096, 0, BF16), (333, 0, 2501, 1037, 0, F32), (8192, 0, 16384, 4096, 0, BF16), (128, 64, 2048, 2048, 1, MX4), (32768, 64, 2048, 2048, 1, MX4),
         (1 << 30, 0, 2, 32, 1, MX4), (1 << 24, 0, 64, 32, 0, BF16), (1 << 30, 0, 64, 96, 0, MX4), (1 << 22, 0, 1 << 14, 64, 1, MX4), (64, 0, 1 << 24, 32, 0, F32),
         (1 << 22, 0, 1 << 17, 128, 1, MX4), ((1 << 22) + 77, 0, (1 << 17) + 2, 128, 1, MX4), (1 << 25, 1000, 1 << 13, 96, 1, MX4), (1 << 24, 1024, 1 << 16, 1024, 1, MX4),
         (1 << 20, 1024, 1 << 24, 32, 1, MX4)]


@pytest.mark.parametrize("size", SIZES)
def test_every_tile_is_launched_once(ask, size):
    rows, experts, channels, width, gated, out = size
    got = ask([size])[0]
    for l in got:
        assert 0 < l.workgroups and l.workgroups * l.threads < 1 << 32, l
        assert l[:2] == got[0][:2] and l.each == got[0].each
    per = got[0].rows
    # as many tiles as any groups can have: none is left out
    tiles = -(-rows // per) if not experts else rows // per + min(experts, rows)
    at = 0
    for l in got:
        if l.name == "mx4_few_kernel":
            assert l.first == at and l.workgroups % l.each == 0 and l.each * 16 * l.args[1] >= channels
            at += l.workgroups // l.each
        else:
            assert l.first == at and l.first % 8 == 0 and l.each * 256 >= channels
            at += l.workgroups
    assert at == (tiles if got[0].name == "mx4_few_kernel" else tiles * got[0].each)


def test_calls_of_ordinary_size_are_one_launch(ask):
    for got in ask(SIZES[:5]):
        assert len(got) == 1 and got[0].first == 0
    assert all(len(got) > 1 for got in ask([SIZES[7], SIZES[8], SIZES[10], SIZES[11]]))


def _tiles(ask, sizes):
    """Rows of the tiles that each size's one launch has, all of them tile kernels."""
    out = []
    for size, got in zip(sizes, ask(sizes)):
        assert len(got) == 1 and got[0].name == "mx4_tile_kernel", (size, got)
        out.append(got[0].rows)
    return out


@pytest.mark.parametrize("shape", sorted(cases.TILE_ROWS))
def test_grouped_sizes_take_their_tiles(ask, shape):
    for experts, entries, k, n in cases.GROUPED[shape] + [cases.GROUPED_LONG[shape]]:
        for gated in (0, 1):
            assert set(_tiles(ask, [(entries, experts, n, k, gated, out) for out in (F32, BF16, MX4)])) == {cases.TILE_ROWS[shape]}
    rows, k, n = cases.LONG[shape]
    assert _tiles(ask, [(rows, 0, n, k, gated, F32) for gated in (0, 1)]) == [cases.TILE_ROWS[shape]] * 2
    # (24 steps' scales lie in LDS)
    assert all((k + 255) // 256 > 24 for k in (k, cases.GROUPED_LONG[shape][2]))


def test_other_sizes_take_tiles(ask):
    rows, k, n = cases.FAR["rows"]
    experts, entries, k2, n2 = cases.FAR["entries"]
    experts3, entries3, _, k3, n3 = cases.FAR["index"]
    experts4, entries4, k4, n4 = cases.HEAVY
    _tiles(ask, [(rows, 0, n, k, 0, BF16), (entries, experts, n2, k2, 0, BF16), (entries3, experts3, n3, k3, 0, BF16), (entries4, experts4, n4, k4, 0, F32)])
    for experts, choices, tokens, width, hidden in cases.EXPERTS_LAYERS:
        _tiles(ask, [(tokens * choices, experts, 2 * hidden, width, 1, MX4), (tokens * choices, experts, width, hidden, 0, F32)])
    for rows, width, hidden in cases.FEEDFORWARD:
        _tiles(ask, [(rows, 0, 2 * hidden, width, 1, MX4), (rows, 0, width, hidden, 0, BF16)])
