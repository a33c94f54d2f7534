"""Activation checkpoints in 8 bits, bit by bit against their definition in 64 bits."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _activations import activations, expected_checkpoint, value  # noqa: E402
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from _train import DTYPES, generator  # noqa: E402

pytestmark = GPU_MARKS


def _check(x, out=None):
    import paper_2402_11857_amd as pkg

    saved = pkg.liec_checkpoint_save(x, out)
    q, s = expected_checkpoint(x)
    assert isinstance(saved, pkg.Checkpoint) and saved.values.dtype == torch.int8 and saved.exponents.dtype == torch.uint8
    assert torch.equal(saved.exponents, s), "exponents"
    assert torch.equal(saved.values, q), "values"
    want = value(saved)
    for dtype in DTYPES.values():
        got = pkg.liec_checkpoint_load(saved, dtype)
        assert got.shape == x.shape and got.dtype == dtype
        assert torch.allclose(got.double(), want.to(dtype).double(), rtol=0, atol=0, equal_nan=True), dtype
    for dtype in (torch.float32, torch.bfloat16):            # exact
        assert torch.equal(torch.nan_to_num(pkg.liec_checkpoint_load(saved, dtype).double()), torch.nan_to_num(want))
    return saved


COLUMNS = [1, 2, 7, 8, 9, 31, 32, 33, 40, 63, 64, 65, 100, 255, 256, 1000, 1001, 4096, 8160, 8192, 8193, 40_003]


@pytest.mark.parametrize("C", COLUMNS)
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_every_row_length(C, dtype):
    say(f"case checkpoint C={C} {dtype}")
    for shape in ((1, 1, C), (3, 5, C), (2, 67, C), (C,), (2, 3, 2, C)):
        x = activations(shape, dtype, seed=C)
        saved = _check(x)
        off = (value(saved) - x.double()).abs()
        largest = torch.nn.functional.pad(x.double().abs(), (0, -C % 32)).unflatten(-1, (-1, 32)).amax(-1)
        assert (off <= largest.repeat_interleave(32, -1)[..., :C] / 127.5 + 2.0 ** -127).all()        # half a step of at most largest / 63.75


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_values_of_every_size_and_kind(dtype):
    say(f"case checkpoint of special values {dtype}")
    t = DTYPES[dtype]
    info = torch.finfo(t)
    rows = [torch.zeros(64), torch.full((64,), info.max), torch.full((64,), -info.max), torch.full((64,), info.tiny), torch.full((64,), info.tiny * info.eps),
            torch.linspace(-127.5, 127.5, 64), torch.linspace(-127, 127, 64), torch.tensor([127.5] + [0.5] * 63), torch.tensor([127.0] + [0.5, 1.5, 2.5, -0.5, -1.5, -2.5] * 10 + [0.25] * 3),
            torch.tensor([1.0, -0.0] * 32)]
    for k in range(-130, 128, 7):                            # every range of exponents, and just under the next power of two
        rows.append((torch.linspace(-1, 1, 64).double() * 2.0 ** k).clamp(-info.max, info.max).float())
        rows.append(torch.full((64,), (1 - 2.0 ** -9) * 2.0 ** k if k < 127 else 1.0))
    x = torch.stack([r.float() for r in rows]).to(DEV).to(t)
    x = torch.where(torch.isinf(x), torch.full_like(x, info.max), x)
    _check(x)
    for bad in (math.inf, -math.inf, math.nan):
        y = activations((5, 100), dtype, seed=1)
        y[1, 40] = bad
        y[3, 99] = bad
        saved = _check(y)
        import paper_2402_11857_amd as pkg

        back = pkg.liec_checkpoint_load(saved)
        assert torch.isnan(back[1, 32:64]).all() and torch.isnan(back[3, 96:]).all()
        assert torch.isfinite(back).sum() == 500 - 32 - 4


def test_values_of_any_kind_load():
    """Integers and exponents that no save leaves are read by the definition."""
    import paper_2402_11857_amd as pkg

    say("case checkpoint, any bytes")
    q = torch.arange(-128, 128, device=DEV).to(torch.int8).repeat(256, 1)
    s = torch.arange(256, device=DEV)[:, None].repeat(1, 8).to(torch.uint8)
    got = pkg.liec_checkpoint_load(pkg.Checkpoint(q, s))
    want = q.double() * 2.0 ** (s.double().repeat_interleave(32, 1) - 127)
    want = torch.where(s.repeat_interleave(32, 1) == 0, torch.zeros_like(want), want)         # 2^-127 counts as zero
    fine = s.repeat_interleave(32, 1) != 255
    assert torch.equal(got[fine].double(), want[fine].float().double())
    assert torch.isnan(got[~fine]).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_strides_and_given_outputs(dtype):
    import paper_2402_11857_amd as pkg

    say(f"case checkpoint strides {dtype}")
    base = activations((4, 9, 300), dtype, seed=3)
    flat = base.reshape(-1)
    for x in (base[:, :, 5:105], base[:, 2:7, 1:34], base[1:2], base[:, ::2, 3:], base[::3, :, :65], flat[1:-299].reshape(-1, 300)[:, :77], flat[3:3 + 9 * 300].view(9, 300),
              base.transpose(0, 1)[:, :, :40], base[:1].expand(3, 9, 300), base.flip(0)[..., :33]):
        saved = _check(x)
        before = saved.values._version, saved.exponents._version
        saved.values.fill_(5)
        again = pkg.liec_checkpoint_save(x, out=saved)
        assert again.values is saved.values and saved.values._version > before[0] and saved.exponents._version > before[1]
        assert torch.equal(again.values, expected_checkpoint(x)[0])
        # values at any address
        room = torch.zeros(x.numel() + 64, dtype=torch.int8, device=DEV)
        odd = pkg.Checkpoint(room[3:3 + x.numel()].view(x.shape), torch.empty_like(saved.exponents))
        pkg.liec_checkpoint_save(x, out=odd)
        assert torch.equal(odd.values, saved.values) and not room[:3].any() and not room[3 + x.numel():].any()
        # into a wider tensor
        wide = torch.full((*x.shape[:-1], x.shape[-1] + 7), 9.0, dtype=x.dtype, device=DEV)
        got = pkg.liec_checkpoint_load(odd, out=wide[..., 2:-5])
        assert got.data_ptr() == wide[..., 2:-5].data_ptr()
        assert torch.equal(wide[..., 2:-5].double(), value(saved).to(x.dtype).double())
        assert (wide[..., :2] == 9).all() and (wide[..., -5:] == 9).all()
    assert torch.equal(pkg.liec_checkpoint_load(saved, out=torch.empty(x.shape, device=DEV)).double(), value(saved))


def test_nothing_to_save():
    import paper_2402_11857_amd as pkg

    say("case checkpoint of no rows")
    saved = pkg.liec_checkpoint_save(torch.empty(3, 0, 40, device=DEV))
    assert saved.values.shape == (3, 0, 40) and saved.exponents.shape == (3, 0, 2)
    assert pkg.liec_checkpoint_load(saved).shape == (3, 0, 40)


def test_refusals():
    import paper_2402_11857_amd as pkg

    say("case checkpoint refusals")
    x = torch.zeros(4, 5, 64, device=DEV)
    saved = pkg.liec_checkpoint_save(x)
    q, s = saved
    for error, call in ((TypeError, lambda: pkg.liec_checkpoint_save(x.double())), (TypeError, lambda: pkg.liec_checkpoint_save(x, out=q)),
                        (TypeError, lambda: pkg.liec_checkpoint_save(x, out=(q.float(), s))), (TypeError, lambda: pkg.liec_checkpoint_save(x, out=(q, s.to(torch.int8)))),
                        (ValueError, lambda: pkg.liec_checkpoint_save(x, out=(q[:3], s[:3]))), (ValueError, lambda: pkg.liec_checkpoint_save(x, out=(q, s[..., :1]))),
                        (ValueError, lambda: pkg.liec_checkpoint_save(x.transpose(1, 2))), (ValueError, lambda: pkg.liec_checkpoint_save(torch.zeros(3, 0, device=DEV))),
                        (TypeError, lambda: pkg.liec_checkpoint_load(saved, torch.float64)), (TypeError, lambda: pkg.liec_checkpoint_load(saved, None)),
                        (ValueError, lambda: pkg.liec_checkpoint_load(saved, out=x[:2])), (TypeError, lambda: pkg.liec_checkpoint_load((q.cpu(), s.cpu()))),
                        (ValueError, lambda: pkg.liec_checkpoint_load((q.transpose(0, 1), s.transpose(0, 1)))),
                        (pkg.LiecError, lambda: pkg.liec_checkpoint_load(saved, out=torch.zeros(1, 1, 64, device=DEV).expand(4, 5, 64))),
                        # what is written in the place of what is read
                        (pkg.LiecError, lambda: pkg.liec_checkpoint_load((q.reshape(-1)[:64].view(1, 64), s.view(-1)[:2].view(1, 2)), out=q.view(torch.float32).reshape(-1)[:64].view(1, 64)))):
        with pytest.raises(error):
            call()


def test_large_offsets():
    import paper_2402_11857_amd as pkg

    say("case checkpoint of 2^31 + 2^26 values")
    R, C = 34_000, 65_536 - 8
    x = torch.empty(R, C, dtype=torch.bfloat16, device=DEV).normal_(generator=generator(5))
    saved = pkg.liec_checkpoint_save(x)
    back = pkg.liec_checkpoint_load(saved, torch.bfloat16)
    for r in (0, 1, 17_000, 32_767, 32_768, 33_998, 33_999):
        q, s = expected_checkpoint(x[r])
        assert torch.equal(saved.values[r], q) and torch.equal(saved.exponents[r], s)
        assert torch.equal(back[r].double(), value((q, s)))
    assert float((back[::997].float() - x[::997].float()).abs().max()) <= float(x.abs().max()) / 127.5


def test_streams_and_graphs():
    import paper_2402_11857_amd as pkg

    say("case checkpoint on another stream and captured")
    x = activations((3, 70, 130), "bf16", seed=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        saved = pkg.liec_checkpoint_save(x)
        back = pkg.liec_checkpoint_load(saved)
    side.synchronize()
    assert torch.equal(back.double(), value(expected_checkpoint(x)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = pkg.liec_checkpoint_save(x)
        again = pkg.liec_checkpoint_load(kept, torch.bfloat16)
    for i in range(4):
        x.copy_(activations((3, 70, 130), "bf16", seed=20 + i))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(again.double(), value(expected_checkpoint(x)))
        assert torch.equal(pkg.liec_checkpoint_save(x).values, kept.values)


def test_results_carry_no_history():
    import paper_2402_11857_amd as pkg

    say("case checkpoint without history")
    x = torch.ones(2, 3, 16, device=DEV, requires_grad=True)
    saved = pkg.liec_checkpoint_save(x)
    assert not pkg.liec_checkpoint_load(saved).requires_grad
    with torch.inference_mode():
        inside = pkg.liec_checkpoint_save(torch.ones(2, 3, 16, device=DEV))
        pkg.liec_checkpoint_save(x, out=inside)
