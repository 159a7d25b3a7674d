"""The layers' binding refuses tensors that are not on the handle's device, before
anything reaches the library.  Without a GPU: stand-ins for tensors of two
devices, and a handle that the library would refuse."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ifvs():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import ifvs as mod
    return mod


class Tensor:
    """What the binding asks of a tensor."""

    def __init__(self, at, *shape, dtype=torch.bfloat16):
        self.at, self.shape, self.dtype = at, shape, dtype
        self.device = torch.device("cuda", at) if at >= 0 else torch.device("cpu")

    def get_device(self):
        return self.at

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


def _calls(ifvs):
    """name, function, the tensors' (name, shape, type) in the order of the arguments, other arguments"""
    T, D, V, F, B, bf, i32, i64 = 6, 16, 9, 24, 2, torch.bfloat16, torch.int32, torch.int64
    td, d, bd = (T, D), (D,), (B, D)
    join = [("gate", bd, bf), ("w_post", d, bf), ("w_pre", d, bf), ("offsets", (B + 1,), i64)]
    ffn = [("x", td, bf), ("w_in", (2 * F, D), bf), ("w_out", (D, F), bf)]
    return [
        (ifvs.ifvs_embed, [("table", (V, D), bf), ("ids", (T,), i32), ("out", td, bf)]),
        (ifvs.ifvs_embed_grad, [("d_out", td, bf), ("ids", (T,), i32), ("d_table", (V, D), bf)]),
        (ifvs.ifvs_norm_join, [("x", td, bf), ("y", td, bf)] + join + [("x_out", td, bf), ("n_out", td, bf)]),
        (ifvs.ifvs_norm_join_grad, [("x_out", td, bf), ("y", td, bf)] + join + [
            ("d_x_out", td, bf), ("d_n", td, bf), ("dx", td, bf), ("dy", td, bf), ("d_gate", bd, bf), ("d_w_post", d, bf),
            ("d_w_pre", d, bf)]),
        (ifvs.ifvs_ffn, ffn + [("y", td, bf)]),
        (ifvs.ifvs_ffn_grad, ffn + [("dy", td, bf), ("dx", td, bf), ("d_w_in", (2 * F, D), bf), ("d_w_out", (D, F), bf)]),
    ]


def test_tensors_of_another_device_are_refused(ifvs):
    h = ifvs._LayersHandle()        # NULL: the library answers IFVS_ERR_ARG
    h.device = 1
    for f, tensors in _calls(ifvs):
        def call(elsewhere=(), at=1):
            kw = {n: Tensor(at if n not in elsewhere else 1 - at, *shape, dtype=dt) for n, shape, dt in tensors}
            return f(h, stream=1, **kw)

        with pytest.raises(ifvs.IfvsError):
            call()
        for n, _, _ in tensors:
            with pytest.raises(ValueError, match=n):
                call(elsewhere=(n,))
        with pytest.raises(ValueError):
            call(at=0)              # all on the other device
        with pytest.raises(ValueError):
            call(at=-1)             # host tensors
