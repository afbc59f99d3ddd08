"""What becomes of a bounded wait that runs out in a training operator: the call's status word has it, or the device's own."""
import ctypes as C

import pytest
import torch

from paper_2410_05589_b200 import binding as b

pytestmark = pytest.mark.gpu
OK, TIMEOUT = 0, -5


@pytest.fixture(scope="module")
def ps():
    import paper_2410_05589_b200 as ps
    assert torch.cuda.is_available()
    ps.train_poll()
    return ps


@pytest.mark.parametrize("loss", [0, 1])
def test_a_wait_that_runs_out_is_there_to_be_asked_for(ps, loss):
    lib = b.load_library()
    assert ps.train_poll() == OK
    assert lib.ps_debug_train_wait_expires(loss, 100000, None, b._stream()) == OK
    assert ps.train_poll() == TIMEOUT and ps.train_poll() == OK
    # calls with a word of their own report to it alone
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert lib.ps_debug_train_wait_expires(loss, 100000, C.c_void_p(status.data_ptr()), b._stream()) == OK
    assert ps.train_poll() == OK and status.item() == 2
    assert lib.ps_debug_train_wait_expires(loss, -1, None, None) == -1
    assert lib.ps_debug_train_wait_expires(loss, 4000000001, None, None) == -1


def test_replayed_waits_are_reported_too(ps):
    lib = b.load_library()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert lib.ps_debug_train_wait_expires(0, 1000, None, b._stream()) == OK
        assert ps.train_poll() == -1
    assert ps.train_poll() == OK
    for _ in range(2):
        g.replay()
        assert ps.train_poll() == TIMEOUT
    assert ps.train_poll() == OK


def test_calls_leave_the_word_alone_and_take_int32_status_alone(ps):
    x, w = torch.ones((300, 64), dtype=torch.bfloat16, device="cuda"), torch.ones((500, 64), dtype=torch.bfloat16, device="cuda")
    labels, up = torch.zeros(300, dtype=torch.int32, device="cuda"), torch.ones(300, device="cuda")
    q = torch.ones((20, 2, 64), dtype=torch.bfloat16, device="cuda")
    at = dict(n_ctx=[0], n_groups=[4], k_masks=4)
    r = ps.lm_loss(x, w, labels)
    ps.lm_loss_backward(x, w, labels, r["lse"], up)
    a = ps.group_attention(q, q, q, **at)
    ps.group_attention_backward(q, q, q, q, a["out"], a["lse"], **at)
    assert ps.train_poll() == OK
    for bad in (torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int32),
                torch.zeros(0, dtype=torch.int32, device="cuda")):
        for call in (lambda: ps.lm_loss(x, w, labels, status=bad), lambda: ps.lm_loss_backward(x, w, labels, r["lse"], up, status=bad),
                     lambda: ps.group_attention(q, q, q, status=bad, **at),
                     lambda: ps.group_attention_backward(q, q, q, q, a["out"], a["lse"], status=bad, **at)):
            with pytest.raises(ps.PsError):
                call()
