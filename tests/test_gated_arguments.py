"""Which tensors the binding of the gated experts' gradient refuses, without a GPU."""
import pytest

from test_gated_abi import D, E, HID, R, OnGpu, call, library, tensors  # noqa: F401 (a fixture)


@pytest.mark.parametrize("n,shape", [("dW1", (E, D, 2 * HID)), ("dW1", (2 * HID, E, D)), ("dW1", (E, 2, HID, D)), ("dW1", (E * D, 2 * HID)), ("dW1", (E, HID, 2 * D)),
                                     ("dW2", (E, HID, D)), ("dW2", (D, E, HID)), ("dW2", (E * HID, D)), ("dW2", (1, E * D, HID))])
def test_a_gradient_of_weights_in_another_layout_is_refused(library, n, shape):  # noqa: F811
    """It has as many elements, and would be filled as if it were [E, 2 F, d] or [E, d, F]."""
    with pytest.raises(TypeError):
        call("scmoe_gated_ffn_backward", **{n: OnGpu(tensors()[n].reshape(shape))})
    assert library.called == []


@pytest.mark.parametrize("n", ["dW1", "dW2"])
def test_a_flat_gradient_of_weights_is_taken(library, n):  # noqa: F811
    """One element more or less is not, nor one with gaps."""
    flat = tensors()[n].reshape(-1)
    call("scmoe_gated_ffn_backward", **{n: OnGpu(flat)})
    assert [name for name, _ in library.called] == ["scmoe_gated_ffn_backward"]
    library.called.clear()
    for t in (flat[1:], flat.new_zeros(flat.numel() + 1), flat.new_zeros(2 * flat.numel())[::2]):
        with pytest.raises(TypeError):
            call("scmoe_gated_ffn_backward", **{n: OnGpu(t)})
    assert library.called == []


@pytest.mark.parametrize("n", ["dy_perm", "dx_perm", "x", "pre"])
def test_rows_of_a_gradient_that_do_not_fit_are_refused(library, n):  # noqa: F811
    """A row less, or some columns less or more."""
    t = tensors()[n]
    assert t.shape[0] == R
    for other in (t[1:], t[:, :-32].contiguous(), t[:, :-32], t.new_zeros(R, t.shape[1] + 32), t.reshape(-1)):
        with pytest.raises(TypeError):
            call("scmoe_gated_ffn_backward", **{n: OnGpu(other)})
    assert library.called == []
