"""What the calls that norm, rotate and append refuse, before anything is launched: needs the built library, no GPU."""
import ctypes as C

import test_operator_arguments as A
from test_operator_arguments import Fake, binding, refused  # noqa: F401  (the binding is loaded by the fixture)

HALF, INT, BYTE, DOUBLE = "torch.float16", "torch.int32", "torch.uint8", "torch.float64"


def rotate(**over):
    t = {"q": Fake(9, 4, 64), "k": Fake(9, 2, 64), "q_out": Fake(9, 4, 64), "k_out": Fake(9, 2, 64), "freqs": Fake(16, dtype=DOUBLE), "positions": Fake(9, dtype=INT)}
    t |= {"q_weight": Fake(64), "k_weight": Fake(64)} | over
    return A.M.qk_rotate(**t)


def on_host(*shape, **kw):
    t = Fake(*shape, **kw)
    t.is_cuda = False
    return t


def test_rotation_refuses():
    M = A.M
    assert M.mmee_qk_rotate_workspace(rotate()) > 0 and M.mmee_qk_rotate_workspace(rotate(q_weight=None, k_weight=None)) == 0
    for over in (dict(q=on_host(9, 4, 64)), dict(q=Fake(9, 4, 64, dtype=HALF)), dict(q=Fake(9, 4, 64, dtype="torch.float32")), dict(k=Fake(8, 2, 64)), dict(k_out=Fake(9, 2, 32)),
                 dict(q=Fake(9, 256)), dict(q_weight=None), dict(k_weight=None), dict(q_weight=Fake(32)), dict(q_weight=Fake(64, dtype=HALF)), dict(positions=None), dict(positions=Fake(8, dtype=INT)),
                 dict(positions=Fake(9, dtype="torch.int64")), dict(positions=Fake(9, dtype=INT, stride=(2,))), dict(freqs=Fake(16, dtype="torch.float32")),
                 dict(freqs=Fake(33, dtype=DOUBLE)), dict(freqs=Fake(4, 4, dtype=DOUBLE)), dict(axis_of=Fake(16, dtype=INT)), dict(axis_of=Fake(15, dtype=BYTE)), dict(pairs="thirds"),
                 dict(freqs=None), dict(q=Fake(9, 4, 64, stride=(256, 1, 4)))):
        refused(lambda: rotate(**over))
    wide = lambda d: dict(q=Fake(9, 4, d), k=Fake(9, 2, d), q_out=Fake(9, 4, d), k_out=Fake(9, 2, d), q_weight=Fake(d), k_weight=Fake(d))  # noqa: E731
    for over in (wide(68), wide(264), dict(freqs=Fake(12, dtype=DOUBLE)), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-40),
                 dict(positions=Fake(5, 9, dtype=INT)), dict(q=Fake(9, 4, 64, stride=(260, 64, 1))), dict(k=Fake(9, 2, 64, stride=(-128, 64, 1))), dict(q_out=Fake(9, 4, 64, stride=(0, 64, 1))),
                 dict(k_out=Fake(9, 2, 64, stride=(128, 0, 1)))):
        refused(lambda: M.mmee_qk_rotate_workspace(rotate(**over)))
        refused(lambda: M.mmee_qk_rotate_forward(rotate(**over)))
    for name in ("q", "k", "q_out", "k_out"):
        H = 4 if name[0] == "q" else 2
        refused(lambda: M.mmee_qk_rotate_forward(rotate(**{name: Fake(9, H, 64, at=(1 << 20) + 8)})))
        refused(lambda: M.mmee_qk_rotate_forward(rotate(**{name: Fake(9, H, 64, at=0)})))
    refused(lambda: M.mmee_qk_rotate_forward(rotate(freqs=Fake(16, dtype=DOUBLE, at=(1 << 20) + 4))))
    refused(lambda: M.mmee_qk_rotate_forward(rotate(positions=Fake(9, dtype=INT, at=(1 << 20) + 2))))
    refused(lambda: M.mmee_qk_rotate_forward(rotate(k_weight=Fake(64, at=(1 << 20) + 2))))
    # in its input's place, but not as the input lies
    refused(lambda: M.mmee_qk_rotate_forward(rotate(q=Fake(9, 4, 64, at=1 << 24), q_out=Fake(9, 4, 64, at=1 << 24, stride=(512, 64, 1)))))
    for field, value in (("dtype", 2), ("pairs", 2), ("heads", 0), ("kv_heads", 0), ("head_dim", 0), ("rot_dim", 24), ("rot_dim", 80), ("axes", 0), ("axis_stride", -1), ("reserved", 1),
                         ("tokens", 1 << 29)):
        r = rotate()
        setattr(r, field, value)
        refused(lambda: M.mmee_qk_rotate_forward(r))
    assert M._lib.mmee_qk_rotate_forward(None) == M.EINVAL and M._lib.mmee_qk_rotate_workspace(C.byref(rotate()), None) == M.EINVAL


def test_rotation_backward_refuses():
    M = A.M
    grads = lambda **o: M.qk_rotate_grads(**{"dq_out": Fake(9, 4, 64), "dk_out": Fake(9, 2, 64), "dq": Fake(9, 4, 64), "dk": Fake(9, 2, 64), "dq_weight": Fake(64), "dk_weight": Fake(64)} | o)  # noqa: E731
    refused(lambda: M.mmee_qk_rotate_backward(rotate(), grads()), M.EWORKSPACE)
    r = rotate()
    size = M.mmee_qk_rotate_workspace(r)
    refused(lambda: M.mmee_qk_rotate_backward(rotate().use_workspace(Fake(size - 1, dtype=BYTE)), grads()), M.EWORKSPACE)
    r.use_workspace(Fake(size, dtype=BYTE))
    for over in (dict(dq=Fake(9, 2, 64)), dict(dk=Fake(9, 2, 64, dtype=HALF)), dict(dq_weight=Fake(32)), dict(dq=on_host(9, 4, 64))):
        refused(lambda: grads(**over))
    for over in (dict(dq_out=Fake(9, 2, 64), dq=Fake(9, 2, 64)), dict(dq_weight=None), dict(dk_weight=None), dict(dq=Fake(9, 4, 64, stride=(0, 64, 1))), dict(dk=Fake(9, 2, 64, at=0)),
                 dict(dk_out=Fake(9, 2, 64, at=(1 << 20) + 8)), dict(dq_weight=Fake(64, at=(1 << 20) + 2)),
                 dict(dq_out=Fake(9, 4, 64, at=1 << 24), dq=Fake(9, 4, 64, at=1 << 24, stride=(512, 64, 1)))):
        refused(lambda: M.mmee_qk_rotate_backward(r, grads(**over)))
    refused(lambda: M.mmee_qk_rotate_backward(rotate(q_weight=None, k_weight=None), grads()))
    refused(lambda: M.mmee_qk_rotate_backward(r, M.qk_rotate_grads(*(Fake(9, h, 64, dtype=HALF) for h in (4, 2, 4, 2)), Fake(64, dtype=HALF), Fake(64, dtype=HALF))))
    assert M._lib.mmee_qk_rotate_backward(C.byref(r), None) == M.EINVAL


def append(**over):
    t = {"k": Fake(12, 2, 64), "v": Fake(12, 2, 64), "k_pages": Fake(9, 16, 2, 64), "v_pages": Fake(9, 16, 2, 64), "page_table": Fake(3, 6, dtype=INT), "cache_lens": Fake(3, dtype=INT),
         "q": Fake(12, 4, 64), "q_out": Fake(12, 4, 64), "freqs": Fake(16, dtype=DOUBLE), "q_weight": Fake(64), "k_weight": Fake(64)}
    return A.M.cache_append(**t | over)


def test_append_refuses():
    M = A.M
    for over in (dict(q=None), dict(q_out=None), dict(v=Fake(11, 2, 64)), dict(v=Fake(12, 2, 64, dtype=HALF)), dict(k_pages=Fake(9, 16, 4, 64)), dict(v_pages=Fake(8, 16, 2, 64)), dict(v_pages=on_host(9, 16, 2, 64)),
                 dict(page_table=Fake(3, 6, dtype="torch.int64")), dict(page_table=Fake(18, dtype=INT)), dict(page_table=Fake(3, 6, dtype=INT, stride=(12, 2))), dict(cache_lens=Fake(4, dtype=INT)),
                 dict(starts=Fake(3, dtype=INT)), dict(starts=Fake(4, dtype="torch.int64")), dict(counts=Fake(4, dtype=INT)), dict(counts=Fake(3, dtype="torch.int64")), dict(q=Fake(12, 256)),
                 dict(k=Fake(12, 128)), dict(q_weight=None), dict(k_weight=None), dict(q=None, q_out=None), dict(freqs=None, positions=Fake(12, dtype=INT)), dict(pairs="")):
        refused(lambda: append(**over))
    odd = dict(k=Fake(13, 2, 64), v=Fake(13, 2, 64), q=Fake(13, 4, 64), q_out=Fake(13, 4, 64))
    for over in (odd, dict(k_pages=Fake(9, 24, 2, 64), v_pages=Fake(9, 24, 2, 64)), dict(axis_of=Fake(16, dtype=BYTE)), dict(eps=0.0), dict(q_out=Fake(12, 4, 64, stride=(0, 64, 1))),
                 dict(k_pages=Fake(9, 16, 2, 64, stride=(0, 128, 64, 1))), dict(v_pages=Fake(9, 16, 2, 64, stride=(2048, 0, 64, 1))), dict(v_pages=Fake(9, 16, 2, 64, stride=(2052, 128, 64, 1))),
                 dict(k=Fake(12, 2, 64, at=0)), dict(v=Fake(12, 2, 64, at=(1 << 20) + 8)), dict(v_pages=Fake(9, 16, 2, 64, at=0)), dict(cache_lens=Fake(3, dtype=INT, at=0)),
                 dict(page_table=Fake(3, 6, dtype=INT, at=0)), dict(starts=Fake(4, dtype=INT, at=(1 << 20) + 2)), dict(q=Fake(12, 4, 64, at=1 << 24), q_out=Fake(12, 4, 64, at=1 << 24, stride=(512, 64, 1)))):
        refused(lambda: M.mmee_cache_append_forward(append(**over)))
    for field, value in (("dtype", 2), ("seqs", 0), ("seqs", 5), ("kv_heads", 0), ("heads", 0), ("q", None), ("page_tokens", 0), ("page_tokens", 1 << 17), ("table_stride", -1), ("reserved", 1), ("axes", 2)):
        c = append()
        setattr(c, field, value)
        refused(lambda: M.mmee_cache_append_forward(c))
    assert M._lib.mmee_cache_append_forward(None) == M.EINVAL


def test_more_tokens_than_a_launch_holds():
    M = A.M
    r = rotate()
    r.tokens = 1 << 26
    refused(lambda: M.mmee_qk_rotate_forward(r))
    refused(lambda: M.mmee_qk_rotate_workspace(r))
    r.tokens = (1 << 26) - 4
    M.mmee_qk_rotate_workspace(r)
    c = append()
    c.tokens = 1 << 26
    refused(lambda: M.mmee_cache_append_forward(c))
