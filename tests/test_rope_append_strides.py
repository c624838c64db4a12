"""sv_rope_append: where there is one token, how far tokens are apart says nothing."""
import pytest
import torch


@pytest.mark.gpu
@pytest.mark.parametrize("n", [0, 1])
def test_one_token_of_a_tensor_with_any_stride(n):
    import paper_2512_21911_b200 as sv
    gen = torch.Generator(device="cuda").manual_seed(n)
    base = torch.empty((6, 1028), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    q, k, v = (base.as_strided((n, h, 128), (stride, 128, 1), at) for h, stride, at in ((4, 1028, 1028 * 2), (2, 3, 1028 * 4), (2, 259, 8)))
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    angle = torch.arange(64, device="cuda")[:, None] * 100.0 ** (-torch.arange(64, device="cuda") / 64)
    rope = torch.cat([angle.cos(), angle.sin()], 1)
    results = []
    for args in ((q, k, v), (q.contiguous(), k.contiguous(), v.contiguous())):
        pools = [torch.zeros((2, 2, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        out, lens = torch.zeros((n, 4, 128), dtype=torch.bfloat16, device="cuda"), ints(-1)
        sv.sv_rope_append(sv.make_geom(1, 4, 2, 128, 64, 2, 1), *pools, ints(1, 0).view(1, 2), ints(63), *args, ints(0, n), out, lens, rope=rope)
        results.append((*pools, out, lens))
    assert all(torch.equal(a, b) for a, b in zip(*results)) and int(results[0][3]) == 63 + n
    assert n == 0 or bool(results[0][0][1, :, 63].any())
