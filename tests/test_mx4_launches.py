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


def calls_of_every_kind():
    """Sizes on both sides of every choice that the calls make."""
    calls = ["context 64 512 128 8 1", "rows 5 64", "back 5 64"]
    for d, f in ((512, 128), (512, 1408), (2048, 768), (4096, 14336)):
        for E in (1, 8, 64):
            for T in (1, 40, 300, 1000, 3000, 9000, 30000):
                calls += [f"context {T} {d} {f} {E} 1", f"experts {T}"]
    for R in (1, 40, 300, 1000, 3000, 9000, 30000):
        calls.append(f"context {R} 512 128 256 1")
        for E in (1, 8, 40, 256):
            for N in (64, 80, 272, 2112, 4112, 8208, 16400):
                for K in (96, 256, 512, 544, 800, 2080, 9248):
                    calls += [f"product {R} {E} {N} {K} {fp32} {int(E > 1)}" for fp32 in (0, 1)]
    for E in (8, 15, 32, 34, 63, 64, 128, 130, 252, 255, 256):
        for groups in (1, 2, 3, 5, 8, 17, 32, 64):
            if E % groups == 0:
                for T in (5, 5000):
                    calls += [f"context {T} 512 128 {E} 1", f"route {T} {SIGMOID} {groups} 1", f"layer {T} {SOFTMAX} {groups} 1"]
    return calls


def test_every_kernel_is_launched_by_some_call(program):
    """The library holds no kernel of these paths that no call takes."""
    taken = set()
    for status, launches in run(program, calls_of_every_kind()):
        assert status == OK
        taken |= {l.kernel for l in launches}
    ours = {k for k in kernels(program) if any(name in k for name in ("mx4", "few_rows_kernel", "route_scored"))}
    assert len(ours) > 40 and not ours - taken, ours - taken
