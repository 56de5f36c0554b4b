"""What the operators of a dense block and of its update refuse, on the host, before a GPU is touched."""
import ctypes as C
import os

import pytest

from .test_operators_abi import CAPACITY, INVALID, ODD, UNSUPPORTED, P, swept


@pytest.fixture(scope="module")
def lib():
    from paper_2311_13225_amd import binding as b
    if not os.path.exists(b.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return b.lib()


def test_layernorm_refusals(lib):
    #       x dt stride res stride w b eps n cap dim sum stride y dt stride mean rstd stream
    good = [P, 0, 32, None, 0, P, P, 1e-5, None, 4, 8, None, 0, P, 0, 32, None, None, None]
    swept(lib.no_layernorm_fwd, good, [({0: None}, INVALID), ({13: None}, INVALID), ({1: 2}, INVALID), ({1: -1}, INVALID), ({14: 2}, INVALID), ({14: 3}, INVALID), ({9: -1}, INVALID),
                                       ({10: 0}, INVALID), ({7: -1.0}, INVALID), ({7: float("nan")}, INVALID), ({2: 28}, INVALID), ({2: 33}, INVALID), ({15: 28}, INVALID),
                                       ({3: P, 4: 28}, INVALID), ({11: P, 12: 30}, INVALID), ({10: 65537, 2: 1 << 20, 15: 1 << 20}, UNSUPPORTED), ({0: ODD}, INVALID), ({13: ODD}, INVALID),
                                       ({3: ODD, 4: 32}, INVALID)])
    #       s dt stride w mean rstd gy stride gs stride n cap dim gx stride gw gb ws bytes stream
    good = [P, 0, 32, P, P, P, P, 32, None, 0, None, 4, 8, P, 32, P, P, P, 1 << 30, None]
    swept(lib.no_layernorm_bwd, good, [({0: None}, INVALID), ({4: None}, INVALID), ({5: None}, INVALID), ({6: None}, INVALID), ({13: None}, INVALID), ({17: None}, INVALID), ({17: ODD}, INVALID),
                                       ({18: 0}, CAPACITY), ({1: 2}, INVALID), ({7: 28}, INVALID), ({8: P, 9: 4}, INVALID), ({14: 31}, INVALID), ({12: 0}, INVALID), ({11: -2}, INVALID),
                                       ({12: 65537, 2: 1 << 20, 7: 1 << 20, 14: 1 << 20}, UNSUPPORTED)])
    assert lib.no_layernorm_ws_bytes(-1, 4) == 0 and lib.no_layernorm_ws_bytes(1, 65537) == 0 and lib.no_layernorm_ws_bytes(1, 0) == 0 and lib.no_layernorm_ws_bytes(0, 1) > 0


def test_linear_refusals(lib):
    #       x dt stride w stride bias act res stride n cap d_in d_out z stride y stride ws bytes stream
    good = [P, 0, 32, P, 64, P, 1, None, 0, None, 4, 8, 16, None, 0, P, 64, P, 1 << 40, None]
    swept(lib.no_linear_fwd, good, [({0: None}, INVALID), ({3: None}, INVALID), ({15: None}, INVALID), ({17: None}, INVALID), ({17: ODD}, INVALID), ({18: 0}, CAPACITY), ({1: 2}, INVALID),
                                    ({1: -1}, INVALID), ({6: 4}, INVALID), ({6: -1}, INVALID), ({10: -1}, INVALID), ({11: 0}, INVALID), ({12: 0}, INVALID), ({2: 28}, INVALID), ({2: 34}, INVALID),
                                    ({4: 60}, INVALID), ({16: 60}, INVALID), ({7: P, 8: 60}, INVALID), ({13: P, 14: 60}, INVALID), ({0: ODD}, INVALID), ({3: ODD}, INVALID),
                                    ({11: (1 << 20) + 1, 2: 1 << 23}, UNSUPPORTED), ({12: (1 << 20) + 1, 4: 1 << 23, 16: 1 << 23}, UNSUPPORTED),
                                    ({10: (1 << 31) - 1023}, UNSUPPORTED)])
    #       x dt stride w stride act z stride gy stride n cap d_in d_out gx stride gw stride gb ws bytes stream
    good = [P, 0, 32, P, 64, 2, P, 64, P, 64, None, 4, 8, 16, P, 32, P, 64, P, P, 1 << 40, None]
    swept(lib.no_linear_bwd, good, [({0: None}, INVALID), ({3: None}, INVALID), ({6: None}, INVALID), ({8: None}, INVALID), ({19: None}, INVALID), ({19: ODD}, INVALID), ({20: 0}, CAPACITY),
                                    ({1: 2}, INVALID), ({5: 4}, INVALID), ({11: -1}, INVALID), ({12: 0}, INVALID), ({13: 0}, INVALID), ({2: 28}, INVALID), ({4: 60}, INVALID), ({7: 60}, INVALID),
                                    ({9: 60}, INVALID), ({15: 28}, INVALID), ({17: 60}, INVALID), ({14: ODD}, INVALID), ({12: (1 << 20) + 1, 2: 1 << 23, 15: 1 << 23}, UNSUPPORTED)])
    for bad in ((2, 4, 8, 8), (0, -1, 8, 8), (0, 4, 0, 8), (0, 4, 8, 0), (0, 4, (1 << 20) + 1, 8), (1, 4, 8, (1 << 20) + 1), (1, (1 << 31) - 1, 8, 8)):
        assert lib.no_linear_ws_bytes(*bad) == 0, bad
    assert lib.no_linear_ws_bytes(0, 0, 1, 1) > 0
    # (a size that does not fit 32 bits anywhere on its way)
    assert lib.no_linear_ws_bytes(1, 2_000_000_000, 4096, 4096) > 2_000_000_000 * 4096 * 4


def test_orthogonalise_refusals(lib):
    #       x dt stride matrix n rows cols steps out dt stride matrix ws bytes stream
    good = [P, 0, 32, 256, 2, 8, 8, 5, P, 0, 32, 256, P, 1 << 40, None]
    swept(lib.no_orthogonalise, good, [({0: None}, INVALID), ({8: None}, INVALID), ({12: None}, INVALID), ({12: ODD}, INVALID), ({13: 0}, CAPACITY), ({1: 2}, INVALID), ({9: 2}, INVALID),
                                       ({4: -1}, INVALID), ({5: 0}, INVALID), ({6: 0}, INVALID), ({7: 0}, INVALID), ({7: 101}, INVALID), ({2: 28}, INVALID), ({2: 33}, INVALID), ({3: 252}, INVALID),
                                       ({3: 0}, INVALID), ({11: 252}, INVALID), ({11: 257}, INVALID), ({10: 28}, INVALID), ({0: ODD}, INVALID), ({5: 32769, 3: 1 << 30, 11: 1 << 30}, UNSUPPORTED),
                                       ({6: 32769, 2: 1 << 20, 10: 1 << 20, 3: 1 << 30, 11: 1 << 30}, UNSUPPORTED), ({4: 65536}, UNSUPPORTED)])
    #       w stride matrix m stride matrix g dt stride matrix n rows cols lr beta nesterov steps decay scale ws bytes stream
    good = [P, 32, 256, P, 32, 256, P, 1, 16, 128, 2, 8, 8, 0.1, 0.9, 1, 5, 0.0, 1.0, P, 1 << 40, None]
    swept(lib.no_muon_step, good, [({0: None}, INVALID), ({3: None}, INVALID), ({6: None}, INVALID), ({19: None}, INVALID), ({20: 0}, CAPACITY), ({7: 2}, INVALID), ({1: 28}, INVALID), ({4: 28}, INVALID),
                                   ({8: 14}, INVALID), ({2: 250}, INVALID), ({5: 0}, INVALID), ({9: 126}, INVALID), ({10: -1}, INVALID), ({11: 0}, INVALID), ({12: 0}, INVALID), ({16: 0}, INVALID),
                                   ({11: 32769, 2: 1 << 30, 5: 1 << 30, 9: 1 << 30}, UNSUPPORTED)])
    for bad in ((-1, 4, 4), (1, 0, 4), (1, 4, 0), (1, 32769, 4), (65536, 4, 4)):
        assert lib.no_orthogonalise_ws_bytes(*bad) == 0, bad
    assert lib.no_orthogonalise_ws_bytes(0, 1, 1) > 0 and lib.no_orthogonalise_ws_bytes(4, 32768, 32768) > 4 * 32768 * 32768 * 8


def test_binding_refuses_other_types_and_shapes():
    """The binding's own checks come before the library is asked (tensors on the host are refused there)."""
    import torch
    from paper_2311_13225_amd import binding as b
    x = torch.zeros((3, 4))
    with pytest.raises(AssertionError):
        b.no_layernorm_fwd(x, None, None, 1e-5, x)
    with pytest.raises(AssertionError):
        b.no_linear_fwd(x, torch.zeros((4, 5)), None, 0, torch.zeros((3, 5)), x)
    with pytest.raises(AssertionError):
        b.no_linear_bwd(x, torch.zeros((4, 5)), 0, None, torch.zeros((3, 5)), x, None, None, x)
    with pytest.raises(AssertionError):
        b.no_orthogonalise(x, x, x)
    with pytest.raises(AssertionError):
        b.no_muon_step(x, x, x, 0.1, 0.9, x)
    assert C.sizeof(C.c_void_p) == 8
