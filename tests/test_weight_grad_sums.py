"""Sums of the weight gradients from kept rows, db above all: a token that is missing, taken twice or left to another sum is
seen.  The shapes take every tile of either type in each of the ways in which its token sums are shared out:

  one      whole tiles only, the first column of tiles adds up db
  shared   whole tiles only, from 8192 tokens on: every column takes its part of the tokens
  slices   all tiles are cut along the tokens
  both     whole tiles and slices in one launch

u = 2^-24 is half a step of fp32, relative."""
import numpy as np
import pytest
import torch

from paper_2601_09026_amd import binding as mb

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
gpu = pytest.mark.gpu

SHAPES = [(F32, 100, 200, 17413), (F32, 8200, 130, 17413), (F32, 1000, 200, 4111), (F32, 333, 2060, 4000),   # 128 x 256
          (F32, 64, 200, 17413), (F32, 777, 200, 4111), (F32, 333, 4000, 2060),                             # 128 x 128
          (F32, 64, 24, 100), (F32, 333, 24, 24), (F32, 70001, 64, 40),                                     # 64 x 64
          (BF16, 64, 2060, 4000), (BF16, 8200, 130, 50257), (BF16, 3000, 130, 17413), (BF16, 333, 2047, 8200),   # 256 x 256
          (BF16, 64, 200, 17413), (BF16, 8200, 260, 17413), (BF16, 2000, 200, 4111), (BF16, 3000, 1000, 8200),   # 128 x 128
          (BF16, 64, 24, 100), (BF16, 8200, 24, 30000), (BF16, 500, 24, 24), (BF16, 70001, 64, 40)]              # 64 x 64


def say(*a):
    print("[case]", *a, flush=True)


def db_is_right(db, dy, scale=1.0):
    """None, or what is wrong with db = scale * the sum of dy's rows (float64 arrays).

    By element: a thread adds up to 4 values of a tile (3 u of their magnitudes) and carries the errors of its tiles' sums, of the
    threads' and of the slices' (2 u each and their second order); then the scale (u).  The largest bf16 tile's threads do
    not carry: u per tile of 64 tokens.  As a whole: that chain's partial sums grow like a random walk, which leaves
    sqrt(tiles / 2) u of the root of dy's squares; twice that."""
    ref, size = scale * dy.sum(0), abs(scale) * np.abs(dy).sum(0)
    tiles = -(-dy.shape[0] // 64)
    if not (np.abs(db - ref) <= (tiles + 14) * U * size).all():
        return "an element"
    if not np.linalg.norm(db - ref) <= U * (2 * np.sqrt(tiles) + 8) * abs(scale) * np.linalg.norm(dy):
        return "as a whole"
    return None


@pytest.mark.parametrize("rows,m", [(64, 24), (333, 24), (8200, 24), (70001, 64)])
def test_the_check_sees_one_token(rows, m):
    """The oracle with a token missing or taken twice, or one feature's value of a token missing: more than fp32 sums may differ by."""
    rng = np.random.default_rng(rows)
    dy = rng.standard_normal((rows, m)).astype(np.float32).astype(np.float64)
    exact = dy.sum(0).astype(np.float32).astype(np.float64)
    assert db_is_right(exact, dy) is None
    for t in (0, rows // 2, rows - 1):
        assert db_is_right(exact - dy[t], dy) and db_is_right(exact + dy[t], dy)
        one = exact.copy()
        one[3] -= dy[t, 3]
        assert abs(dy[t, 3]) < 0.05 or db_is_right(one, dy)


@gpu
@pytest.mark.parametrize("dtype,rows,m,k", SHAPES)
def test_db_within_its_own_chain(dtype, rows, m, k):
    say("db", dtype, rows, m, k)
    rng = np.random.default_rng(rows + m)
    dy = torch.from_numpy(rng.standard_normal((rows, m)).astype(np.float32)).to(dtype).cuda()
    x8 = mb.mgrit_q8_pack(torch.ones((rows, k), device="cuda"))
    for scale in (1.0, 0.375):
        _, db = mb.mgrit_q8_weight_grad(dy, x8, scale=scale)
        wrong = db_is_right(db.double().cpu().numpy(), dy.double().cpu().numpy(), scale)
        assert wrong is None, wrong


@gpu
@pytest.mark.parametrize("dtype,rows,m,k", SHAPES)
def test_whole_numbers_are_summed_exactly(dtype, rows, m, k):
    """Whole numbers whose sums stay below 2^24: every product and every sum is exact, in whatever order, so that dW and db have
    to be equal to the reference's.  An fp32 dy has as many bits as fit, all three of its parts where tokens are few."""
    say("whole numbers", dtype, rows, m, k)
    most = (1 << 24) // (2 * rows)
    most = min(most, 255) if dtype == BF16 else most
    assert most >= 100
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows + m)
    dy = torch.randint(-most, most + 1, (rows, m), generator=gen, device="cuda")
    x = torch.randint(-2, 3, (rows, k), generator=gen, device="cuda", dtype=torch.int8)
    dW, db = mb.mgrit_q8_weight_grad(dy.to(dtype), mb.mgrit_q8_pack(x.to(F32)))
    assert torch.equal(dy.to(dtype).double(), dy.double())
    assert torch.equal(db.double(), dy.double().sum(0))
    ref = dy.double().t().contiguous() @ x.double()
    assert torch.equal(dW.double(), ref)


# tokens, features, the value of all tokens but one, and what a thread's chain of tiles would lose of it without its carry
CARRIED = [(F32, 70001, 64, 40, 0.9375, 30), (F32, 400000, 300, 300, 0.4375, 30), (F32, 60000, 1100, 4200, 0.4375, 30),
           (F32, 100000, 300, 300, 0.4375, 14),
           (BF16, 200000, 64, 40, 0.4375, 30), (BF16, 400000, 300, 300, 0.21875, 30)]


@gpu
@pytest.mark.parametrize("dtype,rows,m,k,small,lost", CARRIED)
def test_what_is_small_beside_a_large_token_is_kept(dtype, rows, m, k, small, lost):
    """The first token is 2^24, every other one so small that a tile's sum of them is less than half a step of it: its
    thread's sum would stay where it is, and `lost` and more would be missing.  Carried sums err by 2 u of 2^24 each (a thread's,
    the threads', the slices'), which is 2, its first tile's plain one by less than 2, the result by a rounding, 1."""
    say("carried sums", dtype, rows, m, k)
    dy = torch.full((rows, m), small, dtype=dtype, device="cuda")
    dy[0] = 2.0 ** 24
    x8 = mb.mgrit_q8_pack(torch.ones((rows, k), device="cuda"))
    _, db = mb.mgrit_q8_weight_grad(dy, x8)
    ref = 2.0 ** 24 + small * (rows - 1)
    off = (db.double() - ref).abs().max().item()
    say("off by", off)
    assert off <= 9 < lost
