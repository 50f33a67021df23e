"""gs_clip_grads refuses an output that two gradients share, or that is another gradient's buffer (as a parameter listed twice makes it
in place): one would be read while the other is written.  No GPU: the calls return before the first CUDA call."""
import ctypes as C

import pytest

A = 1 << 20
BAD, CAPACITY = -1, -2


@pytest.fixture(scope="module")
def api():
    from paper_2609_05255_b200 import build
    build.build()
    from paper_2609_05255_b200 import api
    return api


def call(api, tensors, f=None):
    """Status of a call whose workspace is one byte short: the last check, so what is accepted gives CAPACITY."""
    ctx = C.create_string_buffer(1 << 16)
    arr = (api.GsGradTensor * len(tensors))()
    keep = []
    for s, (grad, out, count, more) in zip(arr, tensors):
        p = (C.c_void_p * max(1, len(more)))(*more)
        keep.append(p)
        s.grad, s.out, s.count, s.dtype, s.more_grads, s.num_more_grads = grad, out, count, 0, p, len(more)
    return (f or api._lib.gs_clip_grads)(ctx, arr, len(tensors), 1.0, A, A, api.gs_grad_workspace_bytes() - 1, None)


def test_outputs_of_their_own_are_accepted(api):
    at = lambda i: A + 4096 * i
    assert call(api, [(at(i), at(i), 10, []) for i in range(512)]) == CAPACITY                       # all in place
    assert call(api, [(at(i), at(1000 + i), 10, [at(2000 + i)]) for i in range(300)]) == CAPACITY
    assert call(api, [(at(1), at(2), 10, [at(2)])]) == CAPACITY                                      # over a further buffer of its own
    assert call(api, [(at(1), at(2), 10, []), (at(1), at(3), 10, [])]) == CAPACITY                   # one gradient read for two outputs
    assert call(api, [(at(1), at(1), 0, []), (at(1), at(1), 10, []), (None, None, 0, [])]) == CAPACITY   # empty ones write nothing


@pytest.mark.parametrize("before", [0, 1, 63, 64, 200, 510])
def test_an_output_that_is_anothers_is_refused(api, before):
    at = lambda i: A + 4096 * i
    others = [(at(i), at(i), 10, []) for i in range(10, 10 + before)]
    for pair in ([(at(1), at(1), 10, []), (at(1), at(1), 10, [])],                                   # the same one twice
                 [(at(1), at(3), 10, []), (at(2), at(3), 10, [])],
                 [(at(1), at(3), 10, []), (at(3), at(4), 10, [])],                                   # the other's gradient, after and before it
                 [(at(3), at(4), 10, []), (at(1), at(3), 10, [])],
                 [(at(1), at(3), 10, []), (at(2), at(4), 10, [at(5), at(3)])]):                      # ... and a further buffer of it
        assert call(api, others + pair) == BAD
        assert call(api, pair[:1] + others + pair[1:]) == BAD
        assert call(api, others + pair, api._lib.gs_grad_norm) == CAPACITY                           # which writes no outputs
