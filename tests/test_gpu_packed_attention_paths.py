"""Packed attention of prompt sizes, and what its calls leave alone."""
import pytest
import torch

from tests.test_gpu_packed_attention import check, make

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


# 640 blocks or more with at most 64 sequences (one wave group, tiles dealt by their work), key/value heads that
# divide among 8 XCDs, dK/dV in whole tiles of many rounds: the launches of prompts
@pytest.mark.parametrize("lens,H,G,hd", [([2048, 700, 1500, 900], 32, 8, 128), ([1300, 0, 1100], 32, 16, 64),
                                         ([1025, 1, 1200], 32, 8, 96)], ids=lambda x: str(x).replace(" ", ""))
def test_prompts(rq, ctx, lens, H, G, hd):
    print(f"[gpu-case] packed prompts {lens} {H}/{G} x {hd}", flush=True)
    check(rq, ctx, *make(lens, H, G, hd, 21))


def guarded(n_rows, shape, fill, behind=5):
    """(a view of n_rows rows of `shape`, the whole buffer): guard columns on both sides, guard rows around."""
    width = shape[0] * shape[1]
    buf = torch.full((n_rows + 2 * behind, width + 16), fill, dtype=BF16, device="cuda")
    return buf[behind:behind + n_rows, 8:8 + width].unflatten(1, shape), buf


@pytest.mark.parametrize("more", [0, 70], ids=["few", "many"])  # empty sequences behind
@pytest.mark.parametrize("offsets,rows", [([-5, 9999], (0, 64)), ([0, 40, 20, 64], (0, 64)), ([70, 90], (0, 0)),
                                          ([0, 2 ** 31 - 1], (0, 64)), ([-2 ** 31, 10], (0, 10)), ([30, 10, 40], (10, 40)),
                                          ([12, 50], (12, 50)), ([60, 20, 5], (0, 0))])
@pytest.mark.parametrize("T,H,G", [(64, 2, 1), (64, 16, 16), (640, 4, 1)])  # the last one: dK/dV in shares
def test_nothing_outside_the_cut_sequences_is_written(rq, ctx, offsets, rows, more, T, H, G):
    """Offsets outside the arrays or in a wrong order (given for 64 rows): results of no meaning, but only in rows of
    the sequences that cutting them leaves."""
    hd, n = 64, T // 64
    offsets, rows = [x * n if abs(x) < 1000 else x for x in offsets], [x * n for x in rows]
    cu = torch.tensor(offsets + [offsets[-1]] * more, dtype=torch.int64).to(torch.int32).cuda()
    q, k, v, do, _ = make([T], H, G, hd, 10)
    views = [guarded(T, (heads, hd), 7.0) for heads in (H, H, G, G)]
    out, dq, dk, dv = (x for x, _ in views)
    _, lse = rq.packed_attention(ctx, q, k, v, cu, out=out)
    # lse and O of rows outside are nobody's: the backward is given finite ones
    rq.packed_attention_backward(ctx, q, k, v, cu, torch.zeros_like(q), torch.zeros_like(lse), do, dq=dq, dk=dk, dv=dv)
    torch.cuda.synchronize()
    for name, (x, buf) in zip(("out", "dq", "dk", "dv"), views):
        kept = buf.clone()
        kept[5:5 + T, 8:-8][rows[0]:rows[1]] = 7.0
        assert (kept == 7).all(), name
        if offsets == sorted(offsets) and rows[1] < T:  # in order: everything inside is written
            assert (x[rows[0]:rows[1]] != 7).any(-1).all(), name


def test_bits_of_a_prompt_again(rq, ctx):
    q, k, v, do, cu = make([1500, 700, 300], 32, 8, 128, 22)
    runs = []
    for _ in range(2):
        o, lse = rq.packed_attention(ctx, q, k, v, cu)
        runs.append((o, lse, *rq.packed_attention_backward(ctx, q, k, v, cu, o, lse, do)))
    assert all(torch.equal(a, b) for a, b in zip(*runs))
