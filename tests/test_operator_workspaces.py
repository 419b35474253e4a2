"""How much room the operators' calls ask for: needs the built library, no GPU."""
import pytest

import test_operator_arguments as A
from test_operator_arguments import Fake, binding, cross  # noqa: F401  (the binding is loaded by the fixture)


@pytest.mark.parametrize("B,Lq,H,Hkv,d,Lk", [(7, 200, 8, 8, 64, 3000), (3, 1, 8, 2, 128, 9000), (2, 40, 4, 4, 80, 5000), (64, 1, 32, 8, 128, 2048), (5, 700, 2, 1, 32, 400)])
@pytest.mark.parametrize("backward", [False, True])
def test_lengths_do_not_change_the_room(B, Lq, H, Hkv, d, Lk, backward):
    """The call looks at no pointer: asked before the lengths are set, it says enough for a call with them, and with all its other pointers null too."""
    import ctypes as C
    t = dict(q=Fake(B, Lq, H, d), k=Fake(B, Lk, Hkv, d), v=Fake(B, Lk, Hkv, d), o=Fake(B, Lq, H, d))
    without, given = cross(**t), cross(**t, kv_lens=Fake(B, dtype="torch.int32"))
    size = A.M.mmee_attn_workspace(without, backward)
    assert size == A.M.mmee_attn_workspace(given, backward)
    for name in ("q", "k", "v", "o"):
        setattr(without, name, None)
    assert size == A.M.mmee_attn_workspace(without, backward)
    assert A.M._lib.mmee_attn_workspace(None, 0, C.byref(C.c_uint64())) == A.M.EINVAL


def test_workspaces_that_are_refused():
    """Host memory, which no kernel may be given, and a view whose elements do not lie one behind the other: it is longer than it says."""
    from test_operator_arguments import block, refused, tree
    on_host = Fake(1 << 20, dtype="torch.uint8")
    on_host.is_cuda = False
    for call in (cross, tree, block):
        refused(lambda: call().use_workspace(on_host))
        refused(lambda: call().use_workspace(Fake(1 << 10, 1 << 10, dtype="torch.uint8", stride=(1 << 12, 4))))
        call().use_workspace(Fake(1 << 20, dtype="torch.uint8"))
