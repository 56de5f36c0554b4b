"""What the operators for learned inputs and large answers refuse, on the host, before a GPU is touched."""
import ctypes as C
import os

import pytest

INVALID, CAPACITY, UNSUPPORTED = -1, -3, -6
P = C.c_void_p(0x10000)          # an address that is never followed: every call here is refused first
ODD = C.c_void_p(0x10001)


@pytest.fixture(scope="module")
def lib():
    from paper_2311_13225_amd import binding as b
    if not os.path.exists(b.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return b.lib()


def swept(fn, good, cases):
    """Each case: {argument's place: value} put into `good`, and the status it has to give."""
    for change, status in cases:
        args = list(good)
        for at, v in change.items():
            args[at] = v
        assert fn(*args) == status, (fn.__name__, change, status)


def test_embed_refusals(lib):
    #       table dt rows dim stride scale ids n cap scale out dt stride stream
    good = [P, 0, 10, 8, 32, None, P, None, 4, 1.0, P, 0, 32, None]
    swept(lib.no_embed_fwd, good, [({0: None}, INVALID), ({6: None}, INVALID), ({10: None}, INVALID), ({1: 3}, INVALID), ({1: -1}, INVALID), ({11: 2}, INVALID),
                                   ({2: 0}, INVALID), ({3: 0}, INVALID), ({8: -1}, INVALID), ({4: 28}, INVALID), ({4: 33}, INVALID), ({12: 16}, INVALID),
                                   ({0: ODD}, INVALID), ({1: 1, 0: ODD}, INVALID), ({12: -32}, INVALID), ({3: (1 << 20) + 1, 4: 1 << 23, 12: 1 << 23}, UNSUPPORTED)])
    #       grad dt stride ids n cap scale acc table rows dim stride ws bytes stream
    good = [P, 0, 32, P, None, 4, 1.0, 0, P, 10, 8, 32, P, 1 << 30, None]
    swept(lib.no_embed_bwd, good, [({0: None}, INVALID), ({3: None}, INVALID), ({8: None}, INVALID), ({12: None}, INVALID), ({12: ODD}, INVALID), ({1: 2}, INVALID),
                                   ({5: -1}, INVALID), ({9: 0}, INVALID), ({9: 1 << 31}, INVALID), ({10: 0}, INVALID), ({2: 28}, INVALID), ({11: 28}, INVALID), ({8: ODD}, INVALID), ({13: 1}, CAPACITY),
                                   ({10: (1 << 20) + 1, 2: 1 << 23, 11: 1 << 23}, UNSUPPORTED)])
    assert lib.no_embed_ws_bytes(-1, 4) == 0 and lib.no_embed_ws_bytes(4, 0) == 0 and lib.no_embed_ws_bytes(4, (1 << 20) + 1) == 0 and lib.no_embed_ws_bytes(0, 1) > 0
    assert lib.no_embed_ws_bytes(2_000_000_000, 100_000) >= lib.no_embed_ws_bytes(1_000_000, 100_000)


def test_rmsnorm_refusals(lib):
    #       x dt stride res stride w eps n cap dim sum stride y dt stride scale rstd stream
    good = [P, 0, 32, None, 0, P, 1e-5, None, 4, 8, None, 0, P, 0, 32, None, None, None]
    swept(lib.no_rmsnorm_fwd, good, [({0: None}, INVALID), ({12: None}, INVALID), ({1: 2}, INVALID), ({13: 3}, INVALID), ({8: -1}, INVALID), ({9: 0}, INVALID),
                                     ({6: -1.0}, INVALID), ({6: float("nan")}, INVALID), ({2: 28}, INVALID), ({14: 28}, INVALID), ({3: P, 4: 28}, INVALID), ({10: P, 11: 30}, INVALID),
                                     ({13: 2, 14: 8}, INVALID), ({15: P}, INVALID), ({9: 65537, 2: 1 << 20, 14: 1 << 20}, UNSUPPORTED), ({0: ODD}, INVALID)])
    #       s dt stride w rstd gy stride gs stride n cap dim gx stride gw ws bytes stream
    good = [P, 0, 32, P, P, P, 32, None, 0, None, 4, 8, P, 32, P, P, 1 << 30, None]
    swept(lib.no_rmsnorm_bwd, good, [({0: None}, INVALID), ({4: None}, INVALID), ({5: None}, INVALID), ({12: None}, INVALID), ({15: None}, INVALID), ({16: 0}, CAPACITY), ({1: 2}, INVALID),
                                     ({6: 28}, INVALID), ({7: P, 8: 4}, INVALID), ({13: 31}, INVALID), ({11: 0}, INVALID), ({10: -2}, INVALID),
                                     ({11: 65537, 2: 1 << 20, 6: 1 << 20, 13: 1 << 20}, UNSUPPORTED), ({15: ODD}, INVALID)])
    assert lib.no_rmsnorm_ws_bytes(-1, 4) == 0 and lib.no_rmsnorm_ws_bytes(1, 65537) == 0 and lib.no_rmsnorm_ws_bytes(0, 1) > 0


def test_distill_refusals(lib):
    #       z dt stride n cap C ids logits k T w
    rows = [P, 0, 32, None, 4, 8, P, P, 2, 1.0, None]
    common = [({0: None}, INVALID), ({1: 2}, INVALID), ({2: 28}, INVALID), ({2: 33}, INVALID), ({4: -1}, INVALID), ({5: 0}, INVALID), ({5: (1 << 22) + 1, 2: 1 << 25}, UNSUPPORTED),
              ({6: None}, INVALID), ({7: None}, INVALID), ({8: 0}, INVALID), ({8: 257}, UNSUPPORTED), ({9: 0.0}, INVALID), ({9: -1.0}, INVALID),
              ({9: float("nan")}, INVALID), ({9: float("inf")}, INVALID), ({9: 1e-39}, INVALID), ({0: ODD}, INVALID)]
    swept(lib.no_distill_fwd, rows + [P, P, P, 1 << 30, None], common + [({11: None}, INVALID), ({12: None}, INVALID), ({13: None}, INVALID), ({14: 1}, CAPACITY)])
    swept(lib.no_distill_bwd, rows + [P, P, 32, None], common + [({11: None}, INVALID), ({12: None}, INVALID), ({13: 16}, INVALID)])
    swept(lib.no_distill_fwd_bwd, rows + [P, P, P, 32, P, 1 << 30, None], common + [({11: None}, INVALID), ({13: None}, INVALID), ({14: 16}, INVALID), ({15: None}, INVALID), ({15: ODD}, INVALID), ({16: 1}, CAPACITY)])
    assert lib.no_distill_ws_bytes(1, (1 << 22) + 1) == 0 and lib.no_distill_ws_bytes(-1, 3) == 0 and lib.no_distill_ws_bytes(0, 1) > 0


def test_logprobs_refusals(lib):
    #       z dt stride n cap C tokens T
    rows = [P, 0, 32, None, 4, 8, P, 1.0]
    common = [({0: None}, INVALID), ({1: 2}, INVALID), ({2: 28}, INVALID), ({4: -1}, INVALID), ({5: 0}, INVALID), ({5: (1 << 22) + 1, 2: 1 << 25}, UNSUPPORTED), ({6: None}, INVALID),
              ({7: 0.0}, INVALID), ({7: float("nan")}, INVALID), ({0: ODD}, INVALID)]
    swept(lib.no_logprobs_fwd, rows + [P, P, P, 2, P, P, P, 1 << 40, None],
          common + [({8: None}, INVALID), ({9: None}, INVALID), ({10: None}, INVALID), ({11: -1}, INVALID), ({11: 65}, UNSUPPORTED), ({12: None}, INVALID), ({13: None}, INVALID),
                    ({14: None}, INVALID), ({15: 1}, CAPACITY)])
    swept(lib.no_logprobs_bwd, rows + [P, P, P, P, P, 32, None], common + [({8: None}, INVALID), ({9: None}, INVALID), ({12: None}, INVALID), ({13: 30}, INVALID)])
    assert lib.no_logprobs_ws_bytes(1, 8, 65) == 0 and lib.no_logprobs_ws_bytes(0, 1, 0) > 0


def test_binding_refuses_other_types_and_shapes():
    """The binding's own checks come before the library is asked (tensors on the host are refused there)."""
    import torch
    from paper_2311_13225_amd import binding as b
    x = torch.zeros((3, 4))
    with pytest.raises(AssertionError):
        b.no_embed_fwd(x, torch.zeros(2, dtype=torch.int32), torch.zeros((2, 4)))
    with pytest.raises(AssertionError):
        b.no_rmsnorm_fwd(x, None, 1e-5, x)
    with pytest.raises(AssertionError):
        b.no_logprobs_bwd(x, torch.zeros(3, dtype=torch.int32), 1.0, x[:, 0], x[:, 0], None, None, x)
    with pytest.raises(AssertionError):
        b.no_distill_fwd(x, torch.zeros((3, 1), dtype=torch.int32), torch.zeros((3, 1)), 1.0, None, x[:, 0], x[:, 0], x)


def test_binding_finds_the_current_stream_with_public_names_alone(monkeypatch):
    """torch's shorter way to the stream's address is taken where it exists, and not needed."""
    from paper_2311_13225_amd import binding as b
    asked = []
    monkeypatch.setattr(b, "_stream", lambda stream=None: asked.append(stream) or 11)
    monkeypatch.setattr(b, "_raw_stream", None)
    assert b._stream_of(None) == 11 and b._stream_of("a stream") == 11 and asked == [None, "a stream"]
    monkeypatch.setattr(b, "_current_device", lambda: 5)
    monkeypatch.setattr(b, "_raw_stream", lambda device: 100 + device)
    assert b._stream_of(None) == 105 and b._stream_of("a stream") == 11
