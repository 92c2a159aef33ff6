"""Host threads that call the same kernels with different sizes at once: each gets what it gets alone, and no launch fails."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def work():
    """Calls that share kernels two by two and differ in the shared memory that they take."""
    import paper_2608_03676_b200 as P
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    wide, narrow = rand(40, 1024), rand(40, 768)
    many, few = rand(40000, 128).bfloat16(), rand(40000, 64).bfloat16()
    h, dy, w = rand(64, 192).bfloat16(), rand(64, 192).bfloat16(), torch.ones(192, dtype=torch.bfloat16, device="cuda")
    rstd = (h.float().square().mean(1) + 1e-6).rsqrt()
    grouped = dict(score="sigmoid", groups=8, groups_kept=4, group_top=2)
    return [(lambda: P.route(wide, 8, **grouped), lambda: P.route(narrow, 8, **grouped)),
            (lambda: P.route(many, 8), lambda: P.route(few, 8)),
            (lambda: P.rms_norm_backward(dy, h, w, rstd), lambda: P.rms_norm_backward(dy, h, w, rstd, want_dweight=False))]


@pytest.mark.parametrize("pair", range(3))
def test_two_host_threads(pair):
    calls = work()[pair]
    want = [f() for f in calls]
    torch.cuda.synchronize()
    start, failed = threading.Barrier(len(calls)), []

    def run(f, expected):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait(timeout=60)
                for _ in range(400):
                    got = f()
                torch.cuda.current_stream().synchronize()
                assert all(torch.equal(got[name], expected[name]) for name in expected)
        except BaseException as e:                 # (reported by the test's own thread)
            failed.append(e)

    threads = [threading.Thread(target=run, args=a) for a in zip(calls, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    assert not failed, failed
