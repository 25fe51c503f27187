"""What the operators' checks of memory refuse and let through, without a GPU: on
addresses that count as device memory, where nothing can be launched."""
import pytest

torch = pytest.importorskip("torch")

import fake_device  # noqa: E402
from paper_2607_18957_amd import ii, ops  # noqa: E402
from test_decoder_ops_abi import ADAPT  # noqa: E402

AT = 1 << 40
LET_THROUGH = "II_EHIP"     # nothing can be launched


@pytest.fixture(scope="module")
def call(tmp_path_factory):
    fake = fake_device.build(str(tmp_path_factory.mktemp("fake")))

    def run(*calls):
        return [ii.ERRNAMES[rc] for rc in fake_device.codes(fake, calls)]
    return run


def _adapt(**change):
    return "ii_adapt", [ops._ADAPT.pack(*{**ADAPT, **change}.values())]


@pytest.mark.parametrize("work", [dict(), dict(work=1 << 50, work_bytes=1 << 20)])
def test_adapt_x_is_not_the_output(call, work):
    """x is read by every workgroup that shares its row's columns: base may be out
    itself, x may not, also where base is."""
    square = dict(n=64, k=64, b_stride=64 * 8, out=AT, out_stride=64, base_stride=64, **work)
    apart = {**square, "x": 1 << 47}
    assert call(_adapt(**square), _adapt(**square, x=AT), _adapt(**square, x=AT, base=AT),
                _adapt(**square, x=AT, base=AT, x_stride=128), _adapt(**square, x=AT, base=AT, x_stride=0),
                _adapt(**square, x=AT, base=AT, m=1),
                _adapt(**square, x=AT, base=AT, out_dtype=7, base_dtype=7)) == ["II_EOVERLAP"] * 7
    assert call(_adapt(**apart), _adapt(**apart, base=AT), _adapt(**apart, base=1 << 48),
                _adapt(**apart, base=apart["x"]), _adapt(**apart, base=AT, out_dtype=7, base_dtype=7)) == [LET_THROUGH] * 5
    # of base in place the strides and the types agree
    assert call(_adapt(**{**apart, "base_stride": 128}, base=AT), _adapt(**apart, base=AT, out_dtype=7),
                _adapt(**apart, base=AT, base_dtype=7)) == ["II_EOVERLAP"] * 3


@pytest.mark.parametrize("what", ["adapters", "scales", "ranks", "a", "b"])
def test_adapt_other_inputs_are_not_the_output(call, what):
    at = dict(out=AT, base=AT, base_stride=32, x=1 << 47)
    assert call(_adapt(**at), _adapt(**{**at, what: AT})) == [LET_THROUGH, "II_EOVERLAP"]
