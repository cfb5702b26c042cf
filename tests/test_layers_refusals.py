"""CPU-only checks of refusals that a caller in C can come by and Python's views cannot.  Addresses here are numbers that nothing dereferences."""
import pytest

from paper_2002_01119_amd import layers, psgd

F32, BF16 = layers.F32, layers.BF16


def refused(rc, code, text):
    assert rc == code, (rc, psgd.last_error())
    assert text in psgd.last_error(), psgd.last_error()


@pytest.mark.parametrize("given", [("dgain",), ("dbias",), ("dgain", "dbias")])
def test_one_view_for_the_gain_and_its_gradient(given):
    """The same struct, not one that is equal: the gain is read after its gradient may have been written."""
    lib, n, t, c = layers.load(), 2, 3, 8
    dy, x, dx = (layers.View((1 << 40) + (k << 30), t * c, c, F32) for k in range(3))
    gain = layers.View(1 << 50, c, 0, F32)
    outs = {name: gain if name in given else layers.View((1 << 51) + k * 4096, c, 0, F32) for k, name in enumerate(("dgain", "dbias"))}
    rc = lib.psgd_layer_norm_grad(dy, x, gain, 1 << 60, (1 << 60) + 4096, None, dx, outs["dgain"], outs["dbias"], n, t, c, 1 << 61, 1 << 20, None)
    refused(rc, psgd.EALIAS, "overlaps")


@pytest.mark.parametrize("n,t,i,o", [(4, 1 << 30, 1, 1 << 30), (1, 1 << 30, 1 << 30, 1), (512, 1, 1 << 20, 1 << 20), (512, (1 << 31) - 1, 8, 512)])
@pytest.mark.parametrize("act", [0, 1])
def test_products_whose_elements_no_address_reaches(n, t, i, o, act):
    """Inputs whose rows share one place can be of any size; dz of that size would be a workspace whose bytes overflow, to none at all for the first."""
    lib = layers.load()
    x, w, dy, z = (layers.View((1 << 40) + (k << 34), 0, 0, F32) for k in range(4))
    db = layers.View(1 << 50, o, 0, F32)
    refused(lib.psgd_linear_grad(dy, z, x, w, None, None, db, act, n, t, i, o, None, 0, None), psgd.EINVAL, "too large")
    y = layers.View(1 << 52, t * o, o, F32)
    refused(lib.psgd_linear(x, w, None, None, y, None, act, n, t, i, o, None, 0, None), psgd.EINVAL, "too large")
    assert lib.psgd_linear_workspace(x, w, n, t, i, o) == 0 and lib.psgd_linear_grad_workspace(dy, x, w, None, None, db, act, n, t, i, o) == 0


def test_calls_go_to_the_library_that_is_loaded():
    """A library built and loaded again is the one that psgd's errors and status are asked of; the layers' calls go there too."""
    torch = pytest.importorskip("torch")
    before = layers.load()
    after = psgd.load(reload=True)
    assert after is not before
    x = torch.zeros(1, 1, 4)
    with pytest.raises(ValueError, match="GPU"):
        layers.layer_norm(x, torch.zeros(1, 4), None, torch.zeros(1, 1, 4))
    assert layers._lib is after
