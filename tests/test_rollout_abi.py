"""The rollout calls where there is no GPU: refusals of the library without a context, and of the binding before anything
reaches a device (a library that only counts its calls, and a context that stands for CPU memory)."""
import types

import pytest
import torch

from paper_2507_01663_b200 import binding as B

V, D, G, T, R, N = 24, 64, 32, 5, 3, 6        # N drafts


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
    c.lib, c.handle, c.device = Library(), None, -1
    yield c
    c.handle = None


BF, F, I, L = torch.bfloat16, torch.float32, torch.int32, torch.int64


def z(*shape, t=F):
    return torch.zeros(*shape, dtype=t)


def arguments():
    return {
        "quantize_head": dict(W=z(V, D, t=BF), codes=z(V, D // 8, t=I), scale=z(V, D // G, t=BF), values=z(V, D, t=BF), group=G),
        "quant_logits": dict(hidden=z(T, D, t=BF), codes=z(V, D // 8, t=I), scale=z(V, D // G, t=BF), logits=z(T, V), group=G, T=T),
        "draft_verify": dict(target_logits=z(N + R, V), draft_logits=z(N, V, t=BF), draft=z(N, t=I), cu_draft=z(R + 1, t=I), u_accept=z(N),
                             u_sample=z(R), token=z(N + R, t=I), n_emitted=z(R, t=I), logp=z(N + R), R=R, D=N),
        "block_slots": dict(length=z(R, t=I), grow=z(R, t=I), held=z(R, t=I), block_table=z(R, 4, t=I), free_blocks=z(9, t=I),
                            free_count=z(1, t=I), held_out=z(R, t=I), free_count_out=z(1, t=I), cu_new=z(R + 1, t=I), slot=z(20, t=L),
                            position=z(20, t=I), granted=z(R, t=I), block_size=16, R=R),
    }


def call(ctx, name, **kw):
    getattr(ctx, name)(**kw, stream=types.SimpleNamespace(cuda_stream=0))


PAIRS = [(n, a) for n, kw in arguments().items() for a, v in kw.items() if isinstance(v, torch.Tensor)]


@pytest.mark.parametrize("name", sorted(arguments()))
def test_what_fits_is_passed_on(ctx, name):
    call(ctx, name, **arguments()[name])
    optional = {"values", "logp", "position", "granted", "draft_logits"}
    call(ctx, name, **{k: None if k in optional else v for k, v in arguments()[name].items()})
    assert ctx.lib.calls == 2


@pytest.mark.parametrize("name,argument", PAIRS)
def test_another_type_is_refused(ctx, name, argument):
    either = argument in ("logits", "target_logits", "draft_logits")
    for dtype in (torch.float64, torch.float16, I, F, BF):
        kw = arguments()[name]
        if dtype == kw[argument].dtype or (either and dtype in (F, BF)):
            continue
        kw[argument] = kw[argument].to(dtype)
        with pytest.raises(ValueError):
            call(ctx, name, **kw)
    assert ctx.lib.calls == 0


@pytest.mark.parametrize("name,argument", [x for x in PAIRS if x[1] not in ("W", "free_blocks", "slot", "codes")])
def test_too_short_is_refused(ctx, name, argument):
    kw = arguments()[name]
    kw[argument] = kw[argument][:-1].contiguous()
    with pytest.raises(ValueError):
        call(ctx, name, **kw)
    assert ctx.lib.calls == 0


@pytest.mark.parametrize("name,argument", [x for x in PAIRS if arguments()[x[0]][x[1]].dim() == 2 and x[1] not in ("block_table", "target_logits")])
def test_another_width_is_refused(ctx, name, argument):
    kw = arguments()[name]
    kw[argument] = torch.cat([kw[argument], kw[argument]], dim=1)
    with pytest.raises(ValueError):
        call(ctx, name, **kw)
    assert ctx.lib.calls == 0


@pytest.mark.parametrize("name,argument", PAIRS)
def test_other_strides(ctx, name, argument):
    kw = arguments()[name]
    x = kw[argument]
    if x.dim() == 1:
        kw[argument] = torch.cat([x, x])[::2]
        if x.numel() == 1:
            return
        with pytest.raises(ValueError):
            call(ctx, name, **kw)
    else:
        kw[argument] = torch.cat([x, x], dim=1)[:, ::2]               # columns apart
        with pytest.raises(ValueError):
            call(ctx, name, **kw)
        kw[argument] = torch.cat([x, x], dim=1)[:, :x.shape[1]]       # rows apart
        if argument in ("logits", "target_logits", "draft_logits", "block_table"):
            call(ctx, name, **kw)
            return
        with pytest.raises(ValueError):
            call(ctx, name, **kw)
    assert ctx.lib.calls == 0


def test_rows_on_top_of_one_another_are_refused(ctx):
    for name, argument in (("quant_logits", "logits"), ("draft_verify", "target_logits"), ("block_slots", "block_table")):
        kw = arguments()[name]
        x = kw[argument]
        kw[argument] = x[:1].expand(x.shape)
        with pytest.raises(ValueError):
            call(ctx, name, **kw)
    assert ctx.lib.calls == 0


@pytest.mark.parametrize("name", sorted(arguments()))
@pytest.mark.parametrize("device", [0, 1])
def test_tensors_of_another_device_are_refused(ctx, name, device):
    ctx.device = device
    with pytest.raises(ValueError):
        call(ctx, name, **arguments()[name])
    assert ctx.lib.calls == 0


def test_group_sizes(ctx):
    kw = arguments()["quantize_head"]
    for group in (0, 16, 48, 256):
        with pytest.raises(ValueError):
            call(ctx, "quantize_head", **dict(kw, group=group))


def test_no_context_is_refused():
    from paper_2507_01663_b200 import build
    build.build()
    lib = B.load_library()
    assert lib.af_quantize_head(None, None, 1, 32, 32, None, None, None, None) == -1
    assert lib.af_quant_logits(None, None, None, None, 0, 32, 1, 32, None, 0, 1, None) == -1
    assert lib.af_draft_verify(None, None, 0, 1, None, 0, 1, None, None, None, None, 0, 0, 1, 0, 1.0, None, None, None, None) == -1
    assert lib.af_block_slots(None, None, None, None, 0, 1, None, 0, 0, None, 0, None, None, None, None, None, None, None, 0, None) == -1
    assert lib.af_reserve_rollout(None, 1, 1) == -1
