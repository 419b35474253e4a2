"""What the attention of packed prompts refuses, before anything is launched: needs the built library, no GPU."""
import ctypes as C

import test_operator_arguments as A
from test_operator_arguments import Fake, binding, refused  # noqa: F401  (the binding is loaded by the fixture)

HALF, INT, BYTE, FLOAT = "torch.float16", "torch.int32", "torch.uint8", "torch.float32"


def prompt(**over):
    t = {"q": Fake(50, 4, 64), "k": Fake(50, 2, 64), "v": Fake(50, 2, 64), "o": Fake(50, 4, 64), "q_starts": Fake(4, dtype=INT)}
    return A.M.prompt_attn(**t | over)


def test_refuses():
    M = A.M
    assert M.mmee_prompt_attn_workspace(prompt()) == 0 and M.mmee_prompt_attn_workspace(prompt(), True) > 0
    on_host = Fake(50, 4, 64)
    on_host.is_cuda = False
    for over in (dict(q=on_host), dict(q=Fake(50, 4, 64, dtype=FLOAT)), dict(v=Fake(50, 2, 64, dtype=HALF)), dict(v=Fake(49, 2, 64)), dict(o=Fake(50, 4, 32)), dict(q=Fake(50, 256)),
                 dict(q=Fake(50, 4, 64, stride=(256, 1, 4))), dict(q_starts=Fake(4, dtype="torch.int64")), dict(q_starts=Fake(1, dtype=INT)), dict(q_starts=Fake(2, 2, dtype=INT)),
                 dict(q_starts=Fake(4, dtype=INT, stride=(2,))), dict(kv_starts=Fake(5, dtype=INT)), dict(kv_starts=Fake(4, dtype=FLOAT)), dict(k=Fake(60, 2, 64), v=Fake(60, 2, 64)),
                 dict(lse=Fake(50, 4, dtype=FLOAT)), dict(lse=Fake(4, 50, dtype="torch.float64")), dict(lse=Fake(4, 50, dtype=FLOAT, stride=(1, 4)))):
        refused(lambda: prompt(**over))
    of = lambda d: dict(q=Fake(50, 4, d), k=Fake(50, 2, d), v=Fake(50, 2, d), o=Fake(50, 4, d))  # noqa: E731
    refused(lambda: prompt(**of(0)))
    for over in (of(68), of(136), dict(k=Fake(50, 3, 64), v=Fake(50, 3, 64)), dict(k=Fake(50, 2, 64, stride=(129, 64, 1))), dict(q=Fake(50, 4, 64, stride=(-256, 64, 1))),
                 dict(o=Fake(50, 4, 64, stride=(0, 64, 1))), dict(o=Fake(50, 4, 64, stride=(256, 0, 1))), dict(k=Fake(50, 2, 64, stride=(1 << 25, 64, 1))),
                 dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        refused(lambda: M.mmee_prompt_attn_workspace(prompt(**over)))
        refused(lambda: M.mmee_prompt_attn_forward(prompt(**over)))
    for over in (dict(q=Fake(50, 4, 64, at=(1 << 20) + 8)), dict(k=Fake(50, 2, 64, at=0)), dict(o=Fake(50, 4, 64, at=0)), dict(q_starts=Fake(4, dtype=INT, at=0)),
                 dict(q_starts=Fake(4, dtype=INT, at=(1 << 20) + 2)), dict(lse=Fake(4, 50, dtype=FLOAT, at=(1 << 20) + 2))):
        refused(lambda: M.mmee_prompt_attn_forward(prompt(**over)))
    for field, value in (("dtype", 2), ("seqs", 0), ("heads", 0), ("kv_heads", 0), ("head_dim", 0), ("kv_tokens", 49), ("q_tokens", 1 << 28), ("reserved", 1)):
        a = prompt()
        setattr(a, field, value)
        refused(lambda: M.mmee_prompt_attn_forward(a))
    assert M._lib.mmee_prompt_attn_forward(None) == M.EINVAL and M._lib.mmee_prompt_attn_workspace(C.byref(prompt()), 0, None) == M.EINVAL


def test_wants_its_workspace():
    M = A.M
    long = dict(q=Fake(2, 4, 64), k=Fake(9000, 1, 64), v=Fake(9000, 1, 64), o=Fake(2, 4, 64), q_starts=Fake(2, dtype=INT), kv_starts=Fake(2, dtype=INT))
    size = M.mmee_prompt_attn_workspace(prompt(**long))
    assert size > 0
    refused(lambda: M.mmee_prompt_attn_forward(prompt(**long)), M.EWORKSPACE)
    refused(lambda: M.mmee_prompt_attn_forward(prompt(**long).use_workspace(Fake(size - 1, dtype=BYTE))), M.EWORKSPACE)
    refused(lambda: M.mmee_prompt_attn_forward(prompt(**long).use_workspace(Fake(size, dtype=BYTE, at=(1 << 20) + 4))))


def test_backward_refuses():
    M = A.M
    grads = lambda **o: M.prompt_attn_grads(**{"do": Fake(50, 4, 64), "dq": Fake(50, 4, 64), "dk": Fake(50, 2, 64), "dv": Fake(50, 2, 64)} | o)  # noqa: E731
    lse = Fake(4, 50, dtype=FLOAT)
    a = prompt(lse=lse)
    a.use_workspace(Fake(M.mmee_prompt_attn_workspace(a, True), dtype=BYTE))
    refused(lambda: M.mmee_prompt_attn_backward(prompt(), grads()))                  # no lse
    refused(lambda: M.mmee_prompt_attn_backward(prompt(lse=lse), grads()), M.EWORKSPACE)
    refused(lambda: grads(do=Fake(50, 256)))
    for over in (dict(do=Fake(50, 2, 64), dq=Fake(50, 2, 64)), dict(dk=Fake(50, 4, 64), dv=Fake(50, 4, 64)), dict(dk=Fake(50, 2, 64, stride=(0, 64, 1))),
                 dict(dv=Fake(50, 2, 64, at=(1 << 20) + 2)), dict(dq=Fake(50, 4, 64, at=0)),
                 {n: Fake(50, h, 64, dtype=HALF) for n, h in (("do", 4), ("dq", 4), ("dk", 2), ("dv", 2))}):
        refused(lambda: M.mmee_prompt_attn_backward(a, grads(**over)))
    assert M._lib.mmee_prompt_attn_backward(C.byref(a), None) == M.EINVAL


def test_more_blocks_than_a_launch_holds():
    """Every sequence may begin a tile of its own, of every head."""
    M = A.M
    a = prompt()
    a.seqs = 1 << 24
    refused(lambda: M.mmee_prompt_attn_forward(a))
    refused(lambda: M.mmee_prompt_attn_workspace(a, True))
    a.seqs = (1 << 23) - 64
    M.mmee_prompt_attn_workspace(a, True)
