"""Refusals and launches of dropout, log probabilities and cross entropy on a stand-in for the HIP runtime (tests/fake_hip.cpp: no
GPU, nothing is read)."""
from test_launch_limits import _run

REFUSALS = """
h = context()
F, R, N = b.Fmt, b.Rng, None
small = C.c_void_p()
assert lib.adapt_create(C.byref(small), None, 4096) == 0
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -5
def dropout(x=at, fx=F(8, 4), n=100, p=0.5, fo=F(8, 4), r=R(1, 1, 1), res=N, fres=F(8, 4), out=2 * at):
    return lib.adapt_dropout(h, x, fx, n, p, fo, r, res, fres, out)
def log_probs(logits=at, f=F(16, 8), rows=10, classes=1000, ld=1000, labels=2 * at, logp=3 * at, lse=4 * at, entropy=5 * at, topk=3, index=6 * at, top=7 * at, ctx=h):
    return lib.adapt_log_probs(ctx, logits, f, rows, classes, ld, labels, logp, lse, entropy, topk, index, top)
def cross_entropy(logits=at, f=F(16, 8), rows=10, classes=1000, ld=1000, labels=2 * at, weights=N, fg=F(16, 15), r=R(1, 1, 1), d=3 * at, ldg=1000, logp=4 * at, ctx=h):
    return lib.adapt_cross_entropy(ctx, logits, f, rows, classes, ld, labels, weights, fg, r, d, ldg, logp)
fake.fake_launched()
bad = [dropout(x=N), dropout(out=N), dropout(p=1.0), dropout(p=-0.01), dropout(p=float("nan")), dropout(p=65535.5 / 65536), dropout(n=(1 << 40) + 1),
       dropout(fx=F(1, 0)), dropout(fo=F(33, 0)), dropout(fo=F(8, 32)), dropout(r=R(2, 0, 0)), dropout(fx=F(16, 4), x=at + 1), dropout(res=at, fres=F(40, 0)),
       dropout(res=at + 1, fres=F(16, 2)),
       log_probs(logits=N), log_probs(labels=N), log_probs(classes=0), log_probs(ld=999), log_probs(classes=(1 << 30) + 1, ld=1 << 31), log_probs(rows=1 << 31),
       log_probs(rows=1 << 20, ld=1 << 21), log_probs(topk=-1), log_probs(topk=33), log_probs(classes=2, ld=2, topk=3), log_probs(index=N), log_probs(top=N),
       log_probs(logits=at + 1), log_probs(labels=2 * at + 4), log_probs(lse=at + 2), log_probs(f=F(1, 0)), log_probs(f=F(33, 0)), log_probs(f=F(8, 32)), log_probs(ctx=N),
       cross_entropy(logits=N), cross_entropy(labels=N), cross_entropy(d=N), cross_entropy(ldg=999), cross_entropy(ld=999), cross_entropy(classes=0), cross_entropy(rows=1 << 31),
       cross_entropy(fg=F(0, 0)), cross_entropy(fg=F(33, 0)), cross_entropy(r=R(7, 0, 0)), cross_entropy(weights=at + 2), cross_entropy(d=3 * at + 1), cross_entropy(ctx=N)]
assert bad == [EINVAL] * len(bad), bad
assert [dropout(fx=F(8, 0), fo=F(8, 16)), dropout(res=at, fres=F(8, 5))] == [EUNSUPPORTED] * 2
assert [log_probs(rows=1, classes=1 << 24, ld=1 << 24, topk=32, ctx=small), cross_entropy(rows=2, classes=1 << 24, ld=1 << 24, ldg=1 << 24, ctx=small)] == [EWORKSPACE] * 2
assert fake.fake_launched() == b""                # nothing was launched
assert [dropout(n=0, x=N, out=N), log_probs(rows=0, logits=N), cross_entropy(rows=0, d=N)] == [0, 0, 0]
assert fake.fake_launched() == b""
# what the queries say is enough
for rows, classes, topk in ((1, 1 << 24, 32), (60, 100003, 7), (64, 1 << 20, 0)):
    for call, f in ((b.CALL_LOG_PROBS, F(16, 8)), (b.CALL_CROSS_ENTROPY, F(8, 4))):
        q = b.WorkspaceQuery(call=call, n=rows, K=classes, count=topk, fa=f, fb=F(8, 7))
        need = lib.adapt_workspace_bytes(N, C.byref(q))
        assert need > 0
        c = C.c_void_p()
        assert lib.adapt_create(C.byref(c), N, need) == 0
        assert (log_probs(f=f, rows=rows, classes=classes, ld=classes, topk=topk, ctx=c) if call == b.CALL_LOG_PROBS else
                cross_entropy(f=f, rows=rows, classes=classes, ld=classes, ldg=classes, ctx=c)) == 0
for q in (b.WorkspaceQuery(call=b.CALL_LOG_PROBS, n=1, K=0, fa=F(8, 4)), b.WorkspaceQuery(call=b.CALL_LOG_PROBS, n=1, K=9, count=10, fa=F(8, 4)),
          b.WorkspaceQuery(call=b.CALL_CROSS_ENTROPY, n=1, K=9, fa=F(8, 4), fb=F(0, 0))):
    assert lib.adapt_workspace_bytes(N, C.byref(q)) == 0
fake.fake_launched()
# rows beyond what a launch takes go in slabs; few and long ones in chunks with a second launch
print(len([log_probs(rows=(1 << 23) + 1, classes=3, ld=3)] and fake.fake_launched().split()), len([cross_entropy(rows=(1 << 22) + 1, classes=300, ld=300, ldg=300)] and fake.fake_launched().split()),
      len([log_probs(rows=1, classes=1 << 20, ld=1 << 20)] and fake.fake_launched().split()), len([log_probs(rows=5000, classes=50000, ld=50000)] and fake.fake_launched().split()))
"""


def test_refusals_launch_nothing_and_large_calls_are_cut(tmp_path):
    out = _run(REFUSALS, tmp_path)
    assert [int(v) for v in out.split()] == [2, 3, 2, 1]
