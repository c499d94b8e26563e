"""aoh_extend reads its inputs after it has begun to store rows, so that its output has to lie elsewhere; no GPU is needed."""
import pytest

from paper_2608_06849_amd import aoh as A
from tests.test_abi_extend import Call
from tests.test_abi_host import FAKE

APART = {name: FAKE + 0x100000 * i for i, name in enumerate(("q", "k", "v", "out"))}


def call(packed, **at):
    """The call's descriptors, their data at places of their own but for those given."""
    c = Call()
    for name, where in {**APART, **at}.items():
        getattr(c, ("p" if packed else "") + name).data = where
    return c


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_an_output_in_place_of_an_input_is_refused(name, packed):
    c = call(packed, out=APART[name])
    assert (c.packed if packed else c.dense)() == A.AOH_ERR_INVALID_ARG
    assert {"q": "q", "k": "k_new", "v": "v_new"}[name] in A.aoh_last_error() and "in place" in A.aoh_last_error()


@pytest.mark.parametrize("packed", [False, True])
def test_other_refusals_come_first(packed):
    c = call(packed, out=APART["q"])
    c.ws = None
    assert (c.packed if packed else c.dense)() == A.AOH_ERR_WORKSPACE
