"""A token's value that is not finite, against a cache: its channels and no others, as in the forward."""
import pytest
import torch

import softmax_layer_reference as ref

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lasad():
    assert torch.cuda.is_available()
    from paper_2507_01652_amd import binding
    binding.load()
    return binding


# keys that are seen: one, fewer than a wavefront's rows, a step of a workgroup and more, several workgroups
@pytest.mark.parametrize("dtype,d,G,count", [(BF, 64, 1, 1), (BF, 64, 2, 5), (BF, 32, 1, 67), (BF, 128, 4, 131), (F, 64, 3, 40), (F, 32, 5, 300),
                                             (F, 128, 1, 77), (BF, 64, 1, 129), (BF, 64, 1, 256), (BF, 64, 2, 3001), (F, 64, 1, 2500)])
@pytest.mark.parametrize("value", [INF, -INF, NAN])
def test_a_value_that_is_not_finite(lasad, dtype, d, G, count, value):
    B, Hk, pos = 2, 2, count - 1
    q, k, v = ref.draw((B, Hk * G, d), dtype, 1).cuda(), ref.draw((B, count, Hk, d), dtype, 2).cuda(), ref.draw((B, count, Hk, d), dtype, 3).cuda()

    def step(v):
        caches = [x.transpose(1, 2).clone(memory_format=torch.contiguous_format) for x in (k, v)]
        for c in caches:
            c[:, :, pos] = NAN                              # (the call brings its own)
        return lasad.lasad_decode_step_window(q, *(x[:, pos].contiguous() for x in (k, v)), *caches, pos, count)
    clean = step(v)
    assert clean.isfinite().all()
    for j in {pos, pos // 2, 0}:
        bad = v.clone()
        bad[0, j, 0, 7] = value
        got = step(bad)
        whole = lasad.lasad_forward_window(q[:, None], k, bad, count, start_pos=pos)[:, 0]
        hit = torch.zeros_like(clean, dtype=torch.bool)
        hit[0, :G, 7] = True
        assert torch.equal(got[~hit], clean[~hit])
        assert torch.equal(got[hit].nan_to_num(9.0, 1.0, -1.0), torch.full_like(got[hit], value).nan_to_num(9.0, 1.0, -1.0))
        assert torch.equal(got[hit].isnan(), whole[hit].isnan()) and not whole[hit].isfinite().any()
