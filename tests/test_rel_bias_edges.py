"""The bucket borders of the relative position bias (CPU): where they lie, and
what the wrappers take as a sequence of them."""
import pytest

from paper_2506_20686_amd import binding as B


def test_last_border_is_far():
    # quotients and powers that floating point rounds up or down, at 100 exact widths
    for exact in range(1, 101):
        for far in list(range(exact + 1, exact + 60)) + [977 * exact // 31 + 60, 4001, 1 << 20]:
            for steps in (1, 2, 7):
                e = B.rel_bias_edges(exact, far, steps)
                assert e[-1] == far and e[0] == 1 - far, (exact, far, steps)
                assert all(a < b for a, b in zip(e, e[1:])) and len(e) <= 2 * (exact + steps)


@pytest.mark.parametrize("exact,far,steps", [(7, 29, 1), (7, 29, 2), (16, 512, 16), (3, 24, 3),
                                             (5, 405, 4), (49, 98, 3), (10, 100000, 4)])
def test_borders_are_the_powers_rounded_up(exact, far, steps):
    # border i is the least integer e >= exact (far / exact)^((i + 1) / steps), that is
    # e^steps >= exact^(steps - i - 1) far^(i + 1)
    up = [e for e in B.rel_bias_edges(exact, far, steps) if e > exact]
    want = set()
    for i in range(steps):
        e, least = exact, exact ** (steps - i - 1) * far ** (i + 1)
        while e ** steps < least:
            e += 1
        want.add(e)
    assert up == sorted(want)


@pytest.mark.parametrize("args", [(1,), (4,), (3, 17, 5), (16, 512, 16)])
def test_both_sides_alike(args):
    # 1 - exact .. exact - 1 have buckets of their own, and d and -d mirror each other
    edges = B.rel_bias_edges(*args)

    def bucket(d):
        return sum(e <= d for e in edges)

    own = [bucket(d) for d in range(1 - args[0], args[0])]
    every = [bucket(d) for d in range(-600, 601)]
    assert all(every.count(b) == 1 for b in own)
    assert all(bucket(d) + bucket(-d) == len(edges) for d in range(601))
    assert every[0] == 0 and every[-1] == len(edges)


@pytest.mark.parametrize("raw", [bytes(8), bytearray(16), b"\x00\x01\x02\x03"])
def test_raw_bytes_are_no_borders(raw):
    # their length counts bytes: the library would read four times what there is
    with pytest.raises(TypeError):
        B._edges_arr(raw)
    for call in (lambda: B.tri_rel_bias_fwd(B.F32, 1, 4, 4, raw, None, None, None, None, None, None),
                 lambda: B.tri_rel_bias_bwd(B.F32, 1, 4, 4, raw, None, None, None, None, None, 0,
                                            None)):
        with pytest.raises(TypeError):
            call()
