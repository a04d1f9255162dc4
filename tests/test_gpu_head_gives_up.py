"""A product of the head whose waits run out, in tiles that are split along their sums, and calls of another context behind
it on the stream, which take over its SMs and their shared memory."""
import pytest

from paper_2412_12487_gb300 import Echo, EchoError

from .test_gpu_head import BF16, F32, _case, _randint, _randn

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("skip", [1, 60, 100])  # a step of all products; the last of the logits'; one of dx alone
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_calls_behind_one_that_gives_up(monkeypatch, dtype, skip):
    n, h, v = 300, 4096, 9000
    x, w = _case(n, h, v, 0, dtype, 1)
    labels, dloss = _randint(0, v, (n,), 2), _randn((n,), 3)
    with Echo(0) as good:
        want = good.cross_entropy(x, w, labels)
        want += good.cross_entropy_grad(dloss, x, w, labels, want[1])
        monkeypatch.setenv("ECHO_TEST_SKIP_LEVEL", str(skip))
        monkeypatch.setenv("ECHO_TEST_WAIT_LIMIT_MS", "20")
        with Echo(0) as bad:
            calls = [lambda: bad.cross_entropy_grad(dloss, x, w, labels, want[1])]
            if skip < h // 64:
                calls.append(lambda: bad.cross_entropy(x, w, labels))
            for call in calls:
                call()
                got = good.cross_entropy(x, w, labels)
                got += good.cross_entropy_grad(dloss, x, w, labels, got[1])
                with pytest.raises(EchoError) as err:
                    bad.wait()
                assert err.value.code == 7
                bad.wait()
                torch.cuda.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, want))
        good.wait()
