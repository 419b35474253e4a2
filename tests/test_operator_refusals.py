"""What the operators' calls refuse by the library's own error, besides test_operator_arguments.py: needs the built library, no GPU."""
import test_operator_arguments as A
from test_operator_arguments import Fake, binding, refused  # noqa: F401  (the binding is loaded by the fixture)


def test_head_size_of_zero():
    q, k = Fake(2, 5, 4, 0), Fake(2, 7, 2, 0)
    refused(lambda: A.M.attn(q, k, k, q))
    refused(lambda: A.M.attn(q, k, k, q, scale=1.0))
    pages = Fake(9, 16, 2, 0)
    refused(lambda: A.M.tree_attn(q, pages, pages, Fake(2, 6, dtype="torch.int32"), Fake(2, dtype="torch.int32"), Fake(2, 5, 1, dtype="torch.int64"), q))


def test_no_hidden_tensor():
    refused(lambda: A.M.ffn(Fake(9, 64), Fake(80, 64), Fake(80, 64), Fake(48, 80), Fake(9, 48), None))
