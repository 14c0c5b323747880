"""Runs of equal tokens around the borders of the chunks that lr_embed_grad sums (16 positions, 32 from 4096 tokens on), in every
width of load, written and accumulated, and rows of dout at any alignment.  Bound: L + 3 (accumulated: L + 4) roundings of a run's L rows."""
import pytest
import torch

from test_gpu_gate import DT, U, close, ctx, gen, grad_reference, rnd, strided   # noqa: F401 (ctx is a fixture)

pytestmark = pytest.mark.gpu


def check(ctx, ids, dout, V, scale=1.0):
    want, mag, count = grad_reference(ids, dout, V, scale)
    got = ctx.embed_grad(ids, dout, V, scale=scale)
    close(got, want, (count + 3) * U * mag)
    base = rnd(V, dout.shape[1], seed=9)
    want, mag, count = grad_reference(ids, dout, V, scale, base=base)
    into = base.clone()
    ctx.embed_grad(ids, dout, V, scale=scale, out=into, accumulate=True)
    close(into, want, (count + 4) * U * mag)
    return got


def tokens(lengths, total):
    lengths = list(lengths)
    lengths.append(total - sum(lengths))
    assert lengths[-1] > 0
    return torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), torch.tensor(lengths, device="cuda")), len(lengths) + 1


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [20, 24, 1024])
@pytest.mark.parametrize("R,T", [(16, 1000), (16, 4095), (32, 4096), (32, 5003)])
def test_runs_around_the_chunk_borders(ctx, R, T, n, dt):
    ids, V = tokens([1, R - 1, R, R + 1, 2 * R - 1, 2 * R, 2 * R + 1, 1, 3 * R, 1, 4 * R + 1, R - 2, 5 * R - 1], T)
    dout = rnd(T, n, seed=R, dtype=DT[dt])
    perm = torch.randperm(T, generator=gen(3), device="cuda")
    for order in (ids, ids.flip(0), ids[perm]):
        check(ctx, order.contiguous(), dout, V)


@pytest.mark.parametrize("R,T", [(16, 700), (32, 4200)])
@pytest.mark.parametrize("length", [1, 2, -1, 0, 1001, 1002, 2000, 2001, 2002, 3000, 3001])
def test_a_run_at_every_offset_in_its_chunk(ctx, R, T, length):
    # 1001: R + 1 and so on; single tokens before it move the run over all places of a chunk
    size = R + length if length < 1 else length if length < 1000 else length // 1000 * R + length % 1000
    for offset in range(R):
        ids, V = tokens([1] * (offset + 1) + [size, 1, size], T)
        check(ctx, ids, rnd(T, 8, seed=offset), V)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,n", [(63, 2, 130), (64, 300, 64), (1023, 3, 33), (1024, 40, 1000), (5000, 1, 40), (8192, 20, 24), (9001, 300, 520)])
@pytest.mark.parametrize("extra,shift", [(8, 3), (8, 0), (3, 1)])
def test_rows_of_any_alignment_give_every_row_of_the_gradient(ctx, dt, T, V, n, extra, shift):
    ids = torch.randint(0, V, (T,), generator=gen(T), device="cuda")
    dout = rnd(T, n, seed=n, dtype=DT[dt])
    got = check(ctx, ids, strided(dout, extra, shift), V, scale=1.3)
    close(got, ctx.embed_grad(ids, dout, V, scale=1.3), 0.0)            # the order of the sums does not depend on it
