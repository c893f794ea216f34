"""An output of the 8-bit path that overlaps an input, or another output, is refused before any device work: rows that are written would change
others before they are read."""
import pytest
import torch

from paper_2410_09615_b200 import binding as K, build

INVALID = K.SLIM_ERR_INVALID_ARG
B, D = 3, 144                                   # rows and columns: two groups of columns, one block of rows
SIZE = {"X": 2 * B * D, "residual": 2 * B * D, "gamma": 2 * D, "H": 2 * B * D, "Y": 2 * B * D, "codes": B * D, "scales": 4 * B * 2, "W": 2 * B * D}
AT = {name: 4096 * (i + 1) for i, name in enumerate(SIZE)}       # fake, aligned, never dereferenced addresses, apart from each other


@pytest.fixture(scope="module")
def lib():
    build.build()
    return K.lib()


def norm(lib, **at):
    a = AT | at
    return lib.slim_rmsnorm(a["X"], a["residual"], a["gamma"], 1e-5, B, D, a["H"], a["Y"], None)


def norm8(lib, **at):
    a = AT | at
    return lib.slim_rmsnorm_fp8(a["X"], a["residual"], a["gamma"], 1e-5, B, D, 0, a["H"], a["codes"], a["scales"], None)


def quant(lib, **at):
    a = AT | at
    return lib.slim_quant_fp8(a["X"], B, D, 0, a["codes"], a["scales"], None)


def pack(lib, **at):
    a = AT | at
    return lib.slim_pack_fp8(a["W"], 0, B, D, 0, a["codes"], a["scales"], None)


PAIRS = [(norm, "Y", o) for o in ("X", "residual", "gamma", "H")] + [(norm, "H", "gamma")] + \
        [(norm8, out, o) for out in ("codes", "scales") for o in ("X", "residual", "gamma", "H")] + [(norm8, "codes", "scales"), (norm8, "H", "gamma")] + \
        [(quant, "codes", "X"), (quant, "scales", "X"), (quant, "codes", "scales"), (pack, "codes", "W"), (pack, "scales", "W"), (pack, "codes", "scales")]


@pytest.mark.parametrize("call, out, other", PAIRS)
def test_outputs_that_overlap(lib, call, out, other):
    size = SIZE | ({"scales": 4 * 2} if call is pack else {})        # (a weight's rows share scales)
    last_in_out, last_in_other = (size[out] - 1) // 16 * 16, (size[other] - 1) // 16 * 16
    for at in (AT[other], AT[other] + last_in_other, AT[other] - last_in_out):
        assert call(lib, **{out: at}) == INVALID


@pytest.mark.parametrize("call", [norm, norm8])
@pytest.mark.parametrize("name", ["X", "residual"])
def test_the_sum_over_a_part_of_an_input(lib, call, name):
    """H may be an input itself, but no other rows of it."""
    for step in (16, -16, 2 * D, SIZE["X"] - 16):
        assert call(lib, H=AT[name] + step) == INVALID


@pytest.mark.parametrize("name", ["Xq", "Xs", "Wq", "Ws"])
def test_the_layer_into_an_operand(lib, name):
    a = {"Xq": 4096, "Xs": 8192, "Wq": 12288, "Ws": 16384}
    assert lib.slim_linear_fwd_fp8(a["Xq"], a["Xs"], 0, 1, a["Wq"], a["Ws"], 0, 16, 64, a[name], None, None) == INVALID


@pytest.mark.parametrize("call", [norm, norm8, quant, pack])
def test_neighbours_are_taken(lib, call):
    """Outputs right behind or ahead of an input, H in an input's place: what comes back is the missing device's error."""
    if torch.cuda.is_available():
        pytest.skip("fake addresses: there is a device that would follow them")
    source = "W" if call is pack else "X"
    for out in ("Y",) if call is norm else ("codes",):
        assert call(lib) in (K.SLIM_ERR_CUDA, K.SLIM_ERR_ARCH)
        assert call(lib, **{out: AT[source] + SIZE[source]}) != INVALID and call(lib, **{out: AT[source] - SIZE[out]}) != INVALID
    if call in (norm, norm8):
        for name in ("X", "residual"):
            assert call(lib, H=AT[name]) != INVALID and call(lib, residual=AT["X"], H=AT[name]) != INVALID
        assert call(lib, H=None) != INVALID and call(lib, residual=None, H=AT["X"]) != INVALID
