"""What the binding of the candidate, distillation and preference calls refuses before anything reaches a device: tensors
of another type, too short for the batch, on another device.  A context that stands for CPU memory and a library that
only counts its calls take the GPU's place."""
import types

import pytest
import torch

from paper_2507_01663_b200 import binding as B

T, K, D, V, S = 5, 3, 16, 24, 4


class Library:
    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def entry(*args):
            self.calls += 1
            return 0
        return entry


@pytest.fixture()
def ctx():
    c = object.__new__(B.Context)
    c.lib, c.handle, c.device = Library(), None, -1           # the device number of CPU tensors
    yield c
    c.handle = None


BF, F, I = torch.bfloat16, torch.float32, torch.int32


def z(*shape, t=F):
    return torch.zeros(*shape, dtype=t)


def arguments():
    head = {"hidden": z(T, D, t=BF), "W": z(V, D, t=BF), "cand": z(T, K, t=I)}
    cu = torch.tensor([0, 2, 3, 3, T], dtype=I)
    return {
        "candidate_logprob": dict(head, cand_logp=z(T, K), entropy=z(T), lse=z(T)),
        "candidate_logprob_backward": dict(head, lse=z(T), dcand=z(T, K), d_hidden=z(T, D, t=BF), d_W=z(V, D)),
        "distill_loss": dict(cand_logp=z(T, K), teacher_logp=z(T, K), cu_seqlens=cu, out=z(24, t=torch.uint8), token_loss=z(T),
                             dcand=z(T, K)),
        "distill_update": dict(head, teacher_logp=z(T, K), cu_seqlens=cu, out=z(24, t=torch.uint8), cand_logp=z(T, K), lse=z(T),
                               d_hidden=z(T, D, t=BF), d_W=z(V, D, t=BF), entropy=z(T), token_loss=z(T), dcand=z(T, K)),
        "preference_loss": dict(logp=z(T), ref_logp=z(T), cu_seqlens=cu, out=z(32, t=torch.uint8), pair_loss=z(S // 2),
                                seq_score=z(S), dlogp=z(T)),
    }


def call(ctx, name, **kw):
    getattr(ctx, name)(**kw, stream=types.SimpleNamespace(cuda_stream=0))


NAMES = sorted(arguments())
PAIRS = [(n, a) for n in NAMES for a in arguments()[n]]
REQUIRED = ("hidden", "W", "cand", "cand_logp", "teacher_logp", "dcand", "lse", "d_hidden", "cu_seqlens", "out", "logp")


@pytest.mark.parametrize("name", NAMES)
def test_what_fits_is_passed_on(ctx, name):
    call(ctx, name, **arguments()[name])
    longer = {k: torch.cat([v, v]) if k not in ("W", "d_W", "cu_seqlens") else v for k, v in arguments()[name].items()}
    call(ctx, name, **longer, T=T)                            # rows behind the batch
    least = {k: v for k, v in arguments()[name].items() if k in REQUIRED}
    call(ctx, name, **(dict(least, ref_logp=None) if name == "preference_loss" else least))
    assert ctx.lib.calls == 3


@pytest.mark.parametrize("name,argument", PAIRS)
def test_another_type_is_refused(ctx, name, argument):
    """The type of half or twice the size, and one of the same size: ids for values and values for ids."""
    same_size = {F: I, I: F, BF: torch.float16, torch.uint8: None}
    for dtype in (torch.float64, torch.float16, same_size[arguments()[name][argument].dtype]):
        if dtype is None or argument == "out":
            continue
        kw = arguments()[name]
        kw[argument] = kw[argument].to(dtype)
        with pytest.raises(ValueError):
            call(ctx, name, **kw)
    assert ctx.lib.calls == 0


@pytest.mark.parametrize("name,argument", PAIRS)
def test_too_short_is_refused(ctx, name, argument):
    kw = arguments()[name]
    kw[argument] = kw[argument][:-1].contiguous()
    if argument == "W":
        kw["T"] = T
        kw["W"] = kw["W"][:, :-8].contiguous()                # rows shorter than the hidden ones
    with pytest.raises(ValueError):                           # the sizes are given: they would come from some of these
        call(ctx, name, **dict(kw, T=T, **({"B": S} if "cu_seqlens" in kw else {})))
    assert ctx.lib.calls == 0


@pytest.mark.parametrize("name,argument", [(n, a) for n, a in PAIRS if arguments()[n][a].dim() == 2])
def test_another_width_is_refused(ctx, name, argument):
    kw = arguments()[name]
    kw[argument] = torch.cat([kw[argument], kw[argument]], dim=1)
    with pytest.raises(ValueError):
        call(ctx, name, **kw)
    assert ctx.lib.calls == 0


@pytest.mark.parametrize("name,argument", PAIRS)
def test_strided_is_refused(ctx, name, argument):
    kw = arguments()[name]
    x = kw[argument]
    kw[argument] = torch.cat([x, x])[::2]
    with pytest.raises(ValueError):
        call(ctx, name, **kw)
    assert ctx.lib.calls == 0


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("device", [0, 1])
def test_tensors_of_another_device_are_refused(ctx, name, device):
    ctx.device = device
    with pytest.raises(ValueError):
        call(ctx, name, **arguments()[name])
    assert ctx.lib.calls == 0


@pytest.mark.parametrize("name", ["distill_loss", "distill_update", "preference_loss"])
def test_a_record_off_its_alignment_is_refused(ctx, name):
    kw = arguments()[name]
    kw["out"] = z(48, t=torch.uint8)[4:4 + kw["out"].numel()]
    assert kw["out"].data_ptr() % 8 == 4
    with pytest.raises(ValueError):
        call(ctx, name, **kw)
    assert ctx.lib.calls == 0
