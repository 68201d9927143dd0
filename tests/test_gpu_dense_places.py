"""Dense attention with a bias and its gradients where the queries begin at any place of grid rows of whole vectors.

On the key side a vector's rows are queries: one that begins off a multiple of 8 (bf16) or 4 (fp32) places crosses the end of a
grid row, where the place on the bias' plane jumps.
"""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_dense import check, make  # noqa: E402

pytestmark = pytest.mark.gpu

CASES = [
    dict(shape=(1, 1, 1, 8, 2, 8, 16), heads=1, first=4),
    dict(shape=(2, 2, 1, 16, 8, 8, 64), heads=2, first=5),
    dict(shape=(2, 2, 1, 20, 5, 16, 64), heads=2, first=[3, 37]),
    dict(shape=(2, 2, 1, 40, 6, 24, 32), heads=1, causal=True, first=13),
    dict(shape=(2, 2, 2, 8, 5, 8, 64), heads=1, first=5),
    dict(shape=(4, 2, 1, 30, 16, 24, 128), heads=2, causal=True, first=[1, 3, 5, 13]),
    dict(shape=(2, 1, 3, 24, 16, 24, 16), heads=2, first=[301, 12]),
    # several tiles of queries, of which some begin at a vector: runs and places, next to aligned slices of the same call
    dict(shape=(3, 3, 1, 200, 64, 64, 64), heads=3, first=[1, 64, 3891]),
    dict(shape=(4, 4, 5, 64, 64, 64, 32), heads=4, causal=True, first=[0, 3, 8, 2053]),
    dict(shape=(2, 2, 1, 100, 64, 64, 128), heads=1, first=13),
    # multiples of 4 that are none of 8
    dict(shape=(2, 2, 1, 70, 9, 12, 64), heads=2, causal=True, first=[4, 20]),
    # a grid of one row, which no vector leaves
    dict(shape=(2, 2, 1, 70, 1, 200, 64), heads=2, causal=True, first=[13, 129]),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", CASES, ids=lambda c: "x".join(map(str, c["shape"])))
def test_queries_at_any_place(scram, c, dtype):
    check(scram, c, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("first", [1, 3, 5, 13])
@pytest.mark.parametrize("H,W", [(8, 8), (16, 24), (64, 64)])
def test_runs_of_queries_that_cross_rows(scram, H, W, first, dtype):
    check(scram, dict(shape=(2, 2, 1, min(3 * W, H * W - first), H, W, 64), heads=2, first=first), dtype, seed=first)


# wide grids, whose part of the bias' plane fills what the staged rows leave of a block's shared memory: around the choice of one
# or two steps in flight, of how many queries a block holds, and the widest; heads of one slice of keys with a window each
WIDE = [
    dict(shape=(1, 1, 2, 1404, 2, 1404, 128), heads=1),
    dict(shape=(1, 1, 2, 1450, 2, 1450, 128), heads=1, causal=True),
    dict(shape=(300, 300, 1, 256, 2, 1450, 128), heads=2, first=1301),
    dict(shape=(1, 1, 2, 2950, 2, 2950, 128), heads=1),
    dict(shape=(2, 2, 1, 700, 2, 3400, 128), heads=1, first=[3000, 5]),
    dict(shape=(2, 2, 1, 1, 2, 3600, 128), heads=2, causal=True, first=[7199, 3600]),
    dict(shape=(1, 1, 1, 900, 2, 4993, 128), heads=1, causal=True, first=8001),
    dict(shape=(1, 1, 1, 900, 2, 4993, 16), heads=1, first=4500),
    dict(shape=(10, 1, 1, 1, 70, 70, 128), heads=10, causal=True, first=[4899, 0, 70, 69, 1, 2500, 2501, 3333, 4001, 8]),
    dict(shape=(20, 2, 1, 3, 70, 70, 128), heads=5, first=[4897, 0, 70, 69, 1, 2500, 2501, 3333, 4001, 8] * 2),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", WIDE, ids=lambda c: "x".join(map(str, c["shape"])))
def test_wide_grids(scram, c, dtype):
    check(scram, c, dtype)


def test_two_threads(scram):
    """Calls of one kernel with different needs of shared memory, issued by two threads at once on streams of their own."""
    import threading

    torch.cuda.synchronize()
    jobs = []
    for Wk in (1500, 4993):
        Q, K, V, dO, kw = make(dict(shape=(2, 2, 1, 300, 2, Wk, 128), heads=1, first=1000), "bf16")
        jobs.append(lambda Q=Q, K=K, V=V, dO=dO, kw=kw: [scram.dense_attend(Q, K, V, **kw), *scram.dense_attend_backward(Q, K, V, dO, **kw)])
    want = [job() for job in jobs]
    torch.cuda.synchronize()
    failed = []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(50):
                    got = jobs[i]()
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
        except BaseException as e:  # noqa: BLE001 (told by the test below)
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
