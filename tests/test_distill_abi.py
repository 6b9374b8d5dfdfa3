"""Struct layouts of the candidate, distillation and preference calls, and their refusals that need no GPU."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2507_01663_b200 import build as b
    b.build()
    from paper_2507_01663_b200 import binding
    return binding.load_library()


def test_struct_layouts_match_header():
    from paper_2507_01663_b200 import binding as B
    assert ctypes.sizeof(B.DistillParams) == 20 and B.DistillParams.temperature.offset == 12
    assert ctypes.sizeof(B.DistillOut) == 24 and B.DistillOut.n_tokens.offset == 16
    assert ctypes.sizeof(B.PreferenceParams) == 32 and B.PreferenceParams.beta.offset == 12
    assert ctypes.sizeof(B.PreferenceOut) == 32 and B.PreferenceOut.n_pairs.offset == 24


def test_no_context_is_refused(lib):
    from paper_2507_01663_b200 import binding as B
    dp, pp = B.DistillParams(0, 1, 0, 1.0, 1.0), B.PreferenceParams(0, 0, 0, 0.1, 0.0, 0.0, 0.0, 1.0)
    assert lib.af_candidate_logprob(None, None, None, None, 0, 1, 8, 8, None, None, None, None) == -1
    assert lib.af_candidate_logprob_backward(None, None, None, None, None, None, 0, 1, 8, 8, None, None, 0, 0, None) == -1
    assert lib.af_reserve_candidates(None, 1, 1, 8, 8, 0, 0) == -1
    assert lib.af_distill_loss(None, None, None, None, 0, 0, 1, ctypes.byref(dp), None, None, None, None) == -1
    assert lib.af_distill_update(None, None, None, None, None, None, 0, 0, 1, 8, 8, ctypes.byref(dp), None, None, None, None,
                                 None, None, None, None, 0, 0, None) == -1
    assert lib.af_preference_loss(None, None, None, None, 0, 0, ctypes.byref(pp), None, None, None, None, None) == -1
    assert lib.af_reserve_preference(None, 1, 2) == -1


def test_sequence_borders_are_int32():
    import torch
    from paper_2507_01663_b200 import binding as B
    cu = torch.zeros(4, dtype=torch.int32)
    assert B.Context._sequences(cu, None) == 3 and B.Context._sequences(cu, 2) == 2
    for bad, n in ((cu.long(), None), (cu.float(), None), (cu, 4)):
        with pytest.raises(ValueError):
            B.Context._sequences(bad, n)
