"""What calls of the 4-bit path and of the routers by scores launch, and that calls which are refused launch nothing
(launches_host.cpp: the library against a runtime that only takes notes)."""
import re

import pytest

import mx4_large_sizes as S
from mx4_launches import compile_program, kernels, run
from mx4_sizes import PLAIN

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


# ---- what the sizes of the numerical tests stand for ----------------------------------------------------

def product_kernels(program, sizes, fp32):
    """The kernel of each product; groups by their rows."""
    calls = [call for counts, N, K in sizes
             for call in (f"context {sum(counts)} 512 128 {len(counts)} 1",
                          f"product {sum(counts)} {len(counts)} {N} {K} {int(fp32)} {int(len(counts) > 1)}")]
    return [launches[0].kernel for status, launches in run(program, calls)[1::2]]


def expert_kernels(program, sizes):
    """The kernels of each FFN: gate/up, down."""
    calls = [call for counts, f, d in sizes for call in (f"context {sum(counts)} {d} {f} {len(counts)} 1", f"experts {sum(counts)}")]
    return [tuple(l.kernel for l in launches) for status, launches in run(program, calls)[1::2]]


def tiles(counts, columns):
    return sum(-(-rows // 256) for rows in counts) * columns


LARGE_KERNEL = re.compile(r"large_kernel<.*>, (true|false), (true|false)>\(")


def persistent_and_odd(kernel):
    found = LARGE_KERNEL.search(kernel)
    return found and tuple(word == "true" for word in found.groups())


def test_every_product_kernel_is_compared_with_64_bits(program):
    plain = [((R // E,) * (E - 1) + (R - R // E * (E - 1),), N, K) for R, E, N, K in PLAIN] + S.PERSISTENT + S.LARGE
    tested = set(product_kernels(program, plain, False)) | set(product_kernels(program, plain, True))
    experts = S.GATEUP_PERSISTENT + S.GATEUP_LARGE + S.GATEUP_ENDS + S.GATEUP_OWN_KSTEPS
    tested |= {gateup for gateup, _ in expert_kernels(program, experts)}
    ours = {k for k in kernels(program) if "mx4::Operands" in k}
    assert len(ours) > 25 and not ours - tested, ours - tested


def test_sizes_of_persistent_workgroups(program):
    """More than two rounds, so that workgroups draw tiles; last rounds more and less than half full, the latter in halves."""
    for fp32 in (False, True):
        forms = [persistent_and_odd(k) for k in product_kernels(program, S.PERSISTENT, fp32)]
        assert all(f is not None and f[0] for f in forms)
        for groups in (1, 8, 12):
            assert {f[1] for f, (counts, _, _) in zip(forms, S.PERSISTENT) if len(counts) == groups} == {False, True}
        assert {(f[0], f[1]) for f in map(persistent_and_odd, product_kernels(program, S.LARGE, fp32))} == {(False, False), (False, True)}
    assert all(persistent_and_odd(gateup) == (True, False) for gateup, _ in expert_kernels(program, S.GATEUP_PERSISTENT))
    assert all(persistent_and_odd(gateup) == (False, False) for gateup, _ in expert_kernels(program, S.GATEUP_LARGE))
    plain = [tiles(counts, -(-N // 256)) for counts, N, _ in S.PERSISTENT]
    gateup = [tiles(counts, f // 128) for counts, f, _ in S.GATEUP_PERSISTENT]
    for totals in (plain, gateup):
        assert min(totals) > 512 and {0 < t % 256 <= 128 for t in totals} == {False, True}


def test_sizes_whose_rows_of_h_end_inside_a_run(program):
    gateup = [k[0] for k in expert_kernels(program, S.GATEUP_ENDS + S.GATEUP_LARGE + S.GATEUP_PERSISTENT[:3])]
    assert all(f % 256 == 128 for _, f, _ in S.GATEUP_ENDS + S.GATEUP_LARGE + S.GATEUP_PERSISTENT[:3])
    assert {persistent_and_odd(k) for k in gateup} == {None, (True, False), (False, False)}
    assert len(set(gateup)) >= 5


def test_sizes_of_ksteps_in_turn(program):
    """Every tile whose k-steps may begin anywhere."""
    for counts, _, K in S.OWN_KSTEPS + S.GATEUP_OWN_KSTEPS:
        assert K % 8192 == 0
    ring = {k for k in kernels(program) if "ring_kernel" in k}
    plain = {k for k in ring if re.search(r", true>\s*>\(", k)}                           # of fp32 outputs
    gateup = {k for k in ring if re.search(r", true, (true|false), false>\s*>\(", k)}     # DUAL
    assert set(product_kernels(program, S.OWN_KSTEPS, True)) >= plain - {k for k in plain if "128, 128, 2, 2, 2" in k}
    assert {k for k, _ in expert_kernels(program, S.GATEUP_OWN_KSTEPS)} >= gateup and len(gateup) == 4 and len(plain) == 7


def test_sizes_with_nan_take_ring_and_large_tiles(program):
    forms = {persistent_and_odd(k) for k in product_kernels(program, S.NAN, True)}
    assert forms == {None, (False, True), (True, False)}
