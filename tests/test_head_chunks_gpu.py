"""The gradient of a head's cross entropy adds its logits in the chunks of the forward pass, bf16 too: to the bound of such chunks, 44 blocks
of 16 indices at most, where test_head_gpu allows the bf16 gradient one running sum over the whole width."""
import pytest

import paper_1910_11971_gb300 as cci
import test_head_gpu as head

pytestmark = pytest.mark.gpu


# three chunks of eleven stages, the last width of them; eight chunks of eight; widths past whole chunks
@pytest.mark.parametrize("N,D,V", [(40, 1408, 700), (130, 2048, 513), (300, 2112, 1001), (64, 4096, 300), (257, 4104, 511)])
def test_the_gradients_logits_to_the_bound_of_chunks(monkeypatch, N, D, V):
    one = head.logit_error
    monkeypatch.setattr(head, "logit_error", lambda X, W, dtype, chunked: one(X, W, dtype, True))
    X, W, targets, dloss = head.inputs(N, D, V, "bf16", D)
    args = X.to("cuda:0"), W.to("cuda:0"), targets.to("cuda:0")
    loss, stats = cci.linear_cross_entropy(*args)
    head.check_forward(X, W, targets, loss, stats, "bf16")
    dX, dW = cci.linear_cross_entropy_backward(dloss.to("cuda:0"), *args, stats)
    head.check_backward(X, W, targets, stats, dloss, dX, dW, "bf16")
