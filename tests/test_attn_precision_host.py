"""The bound on the steps' errors in the root mean square: it holds for the roundings that it is derived from, and not for coarser ones."""
import pytest

torch = pytest.importorskip("torch")

import attn_precision_reference as ref


def rounded(y, how):
    """Weights as the products take them."""
    if how == "one bf16":
        return y.to(torch.bfloat16).double()
    if how == "one fp16":
        return y.to(torch.float16).double()
    first = y.to(torch.bfloat16).double()
    return first + (y - first).to(torch.bfloat16).double()


@pytest.mark.parametrize("keys", [64, 400, 1500])
@pytest.mark.parametrize("how,weight", [("two bf16", ref.TWO_BF16), ("one fp16", ref.ONE_FP16), ("one bf16", ref.ONE_BF16)])
def test_the_bound_tells_one_number_of_a_weight_from_two(how, weight, keys):
    g = torch.Generator().manual_seed(keys)
    H, d = 64, 128
    q, k, v = (torch.randn(n, generator=g, dtype=torch.float64).to(torch.bfloat16) for n in ((H, d), (keys, 1, d), (keys, 1, d)))
    none = torch.zeros_like(k, dtype=torch.float64)
    out, squares = ref.attend(q, (none, k), (none, v))
    y = torch.softmax((q.double() @ k[:, 0].double().T) * d ** -0.5, -1)
    y = y / y.amax(-1, keepdim=True)
    got = ((rounded(y, how) @ v[:, 0].double()) / y.sum(-1, keepdim=True)).to(torch.bfloat16)
    error = ref.error(got, out)
    assert error <= ref.bound(out, squares, weight)
    assert (error <= ref.bound(out, squares, ref.TWO_BF16)) == (how != "one bf16")
    assert error >= 0.8 * ref.bound(out, squares, ref.TWO_BF16) / ref.MORE
