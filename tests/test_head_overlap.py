"""Outputs that share memory with what a call still reads are refused; outputs beside or between it are not (no GPU: tests/fake_hip.cpp)."""
import itertools

from test_launch_limits import _run

CROSS_ENTROPY = """
h = context()
def call(d, f, rows, classes, ld, fg, ldg):
    return lib.adapt_cross_entropy(h, at, f, rows, classes, ld, 2 * at, None, fg, b.Rng(1, 1, 1), at + d, ldg, None)
for d, wl, rows, classes, ld, wl_g, ldg in calls:
    print(call(d, b.Fmt(wl, 4), rows, classes, ld, b.Fmt(wl_g, 4), ldg))
print(len(fake.fake_launched().split()))
"""


def _bytes(wl):
    return 1 if 0 < wl <= 8 else 2 if 0 < wl <= 16 else 4


def _share(d, wl, rows, classes, ld, wl_g, ldg):
    """Whether any byte belongs to both, by looking at every row."""
    es, eg = _bytes(wl), _bytes(wl_g)
    x = {i * ld * es + k for i in range(rows) for k in range(classes * es)}
    return any(d + i * ldg * eg + k in x for i in range(rows) for k in range(classes * eg))


def _statuses(calls, tmp_path, source):
    out = [int(v) for v in _run(f"calls = {calls!r}\n" + source, tmp_path).split()]
    assert len(out) == len(calls) + 1
    return out[:-1], out[-1]


def test_gradients_in_the_place_of_the_logits_are_refused(tmp_path):
    calls = []
    for wl, wl_g in ((8, 8), (0, 8), (8, 16), (12, 12), (24, 16), (16, 32)):
        es, eg = _bytes(wl), _bytes(wl_g)
        for rows, classes in ((1, 5), (3, 7), (4, 300)):
            # in place, around the ends, and anywhere in rows far enough apart to hold both
            for ld, ldg in ((classes, classes), (classes + 4, classes + 2), (8 * classes, 8 * classes * es // eg)):
                if ldg < classes:
                    continue
                ends = (0, eg, -eg, (rows - 1) * ld * es + classes * es, -((rows - 1) * ldg * eg + classes * eg), classes * es + -(classes * es) % eg, 4 * classes * es // eg * eg)
                calls += [(d + off, wl, rows, classes, ld, wl_g, ldg) for d, off in itertools.product(ends, (0, eg, -eg)) if (d + off) % eg == 0]
    got, launches = _statuses(calls, tmp_path, CROSS_ENTROPY)
    shared = [_share(*c) for c in calls]
    assert any(shared) and not all(shared)
    for c, status, both in zip(calls, got, shared):
        d, wl, rows, classes, ld, wl_g, ldg = c
        if both:
            assert status == -1, c
        elif rows == 1 or ld * _bytes(wl) == ldg * _bytes(wl_g):
            assert status == 0, c                          # rows that lie between the other's rows are told apart
        else:
            first, last = 0, (rows - 1) * ld * _bytes(wl) + classes * _bytes(wl)
            apart = d >= last or d + (rows - 1) * ldg * _bytes(wl_g) + classes * _bytes(wl_g) <= first
            assert status == (0 if apart else -1), c
    assert launches == got.count(0)


DROPOUT = """
h = context()
for out, wl_x, wl_o, res, wl_res, n in calls:
    F = b.Fmt
    print(lib.adapt_dropout(h, at, F(wl_x, 4), n, 0.5, F(wl_o, 4), b.Rng(1, 1, 1), at + res if res is not None else None, F(wl_res, 4), at + out))
print(len(fake.fake_launched().split()))
"""


def test_dropout_in_place_is_taken_and_in_part_of_the_place_refused(tmp_path):
    """out may be x, or res, where the codes have one size (each is read before its successor is written); at any other distance
    codes would be overwritten before they are read."""
    def share(a, bytes_a, b, bytes_b):
        return a < b + bytes_b and b < a + bytes_a

    calls, want = [], []
    for wl_x, wl_o, wl_res in itertools.product((8, 16, 32), repeat=3):
        x, o, r = _bytes(wl_x), _bytes(wl_o), _bytes(wl_res)
        for n in (1, 100):
            for res in (None, 0, 4 * n, 1 << 20):
                for out in (0, o, -o, 4, -4, 4 * n, n * x // o * o, -n * o, 8 * n, (1 << 20) + o, 1 << 20):
                    calls.append((out, wl_x, wl_o, res, wl_res, n))
                    bad = share(0, n * x, out, n * o) and not (out == 0 and x == o)
                    if res is not None:
                        bad = bad or (share(res, n * r, out, n * o) and not (out == res and r == o))
                    want.append(-1 if bad else 0)
    got, launches = _statuses(calls, tmp_path, DROPOUT)
    assert got == want, next((c, g, w) for c, g, w in zip(calls, got, want) if g != w)
    assert 0 < launches == want.count(0) < len(want)
