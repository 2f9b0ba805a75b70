"""What calls of the 4-bit path and of the routers by scores launch, and that calls which are refused launch nothing
(launches_host.cpp: the library against a runtime that only takes notes)."""
import pytest

from mx4_launches import compile_program, kernels, run

OK, INVALID, UNSUPPORTED = 0, -1, -2
SOFTMAX, SIGMOID, NONE = 0, 1, -1


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return compile_program(tmp_path_factory.mktemp("host"))


# The router: 4 tokens of 256 threads with more than 16 groups, else 16; the combination: 256 threads a token. Of the rows'
# conversion no layer gets there on this card: 16 rows of 256 elements and 256 threads are 2^32 threads for 2^36 elements.
@pytest.mark.parametrize("call,tokens,experts", [
    (f"route {{}} {SIGMOID} 32 4", 2**26 - 4, 32), (f"route {{}} {SIGMOID} 1 1", 2**28 - 16, 32),
    (f"route {{}} {SOFTMAX} 16 4", 2**28 - 16, 32),
    (f"logits {{}} {SOFTMAX} 32 4", 2**26 - 4, 32), (f"logits {{}} {SIGMOID} 16 4", 2**28 - 16, 32), (f"logits {{}} {SOFTMAX} 1 1", 2**28 - 16, 8),
    (f"layer {{}} {SIGMOID} 32 4", 2**24 - 1, 32), (f"layer {{}} {NONE} 1 1", 2**24 - 1, 32), (f"layer {{}} {SOFTMAX} 1 1", 2**24 - 1, 8)])
def test_more_tokens_than_a_launch_holds(program, call, tokens, experts):
    """The most tokens are taken; of one more nothing is launched, also where only a later stage of the call could not be."""
    context = f"context {2**30} 512 128 {experts} 1"
    fits, refused, most = run(program, [context, call.format(tokens), call.format(tokens + 1), call.format(2**30)])[1:]
    assert fits[0] == OK and fits[1]
    assert all(l.grid * l.threads < 2**32 for l in fits[1])
    assert refused == (UNSUPPORTED, []) and most == (UNSUPPORTED, [])
