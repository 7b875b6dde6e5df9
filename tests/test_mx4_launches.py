"""What products in MX4 launch: every tile once, in launches that the GPU takes."""
import pytest

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
