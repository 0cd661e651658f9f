"""The operators' calls marshalled in C against the binding's general path, over the forms that arguments come in: the same values reach
the library, the same exceptions come back.  The library is a stub that records its arguments' addresses and numbers."""
import ctypes as C

import numpy as np
import pytest
import torch

import test_binding_calls as calls
from paper_2502_11058_amd import binding as B

# entry point -> letters of its arguments: d a description, h a description of heads, p a tensor, i a 64-bit integer, s the stream
ENTRIES = {"ddp_norm_backward_workspace": "d", "ddp_attention_forward_workspace": "dhhh", "ddp_attention_backward_workspace": "dhhhh",
           "ddp_cross_entropy_forward_workspace": "dpp", "ddp_cross_entropy_backward_workspace": "dpp", "ddp_norm_forward": "dpppppps", "ddp_norm_backward": "dpppppppppis",
           "ddp_rotary": "dpppppps", "ddp_attention_forward": "dhhhpphppis", "ddp_attention_backward": "dhhhhhppphhhpis", "ddp_cross_entropy_forward": "dppppppis",
           "ddp_cross_entropy_backward": "dppppppppis"}
DESCRIPTIONS = {"norm": B.ddp_norm, "rotary": B.ddp_rotary_shape, "attention": B.ddp_attention, "cross": B.ddp_head}


def _stub():
    src = calls._stub()
    for name, sig in ENTRIES.items():
        args = ", ".join(f"{'long' if k == 'i' else 'void *'} a{j}" for j, k in enumerate(sig))
        body = "".join(f" rec[{j + 1}] = (long)a{j};" for j in range(len(sig)))
        src = src.replace(f"int {name}(void) {{ return 0; }}\n", f"long {name}({args}) {{{body} return status; }}\n")
    return src


@pytest.fixture
def stub(tmp_path, monkeypatch):
    source = _stub()
    monkeypatch.setattr(calls, "_stub", lambda: source)
    with calls._stubbed(tmp_path, monkeypatch) as l:
        yield l


def _usual(name):
    """Arguments as operators.py passes them."""
    heads, t = B.ddp_heads(4096, 1, 2, 3), torch.zeros(8)
    of = {"d": DESCRIPTIONS[name.split("_")[1]](), "h": heads, "p": t, "i": 1024, "s": None}
    return [of[k] for k in ENTRIES[name]]


@pytest.mark.parametrize("name", sorted(ENTRIES))
def test_same_as_the_general_path(stub, monkeypatch, name):
    call, sig = getattr(B, name), ENTRIES[name]

    class Own(B.ddp_heads):
        pass

    other = {"d": [None, B.ddp_heads(), 7, torch.zeros(2), C.create_string_buffer(128)], "h": [None, Own(64, 1, 2, 3), B.ddp_head(), 7, torch.zeros(2)],
             "p": [None, 0, 4096, True, torch.zeros(0), np.zeros(4), "x", 1.5, 2 ** 70], "i": [0, -1, 2 ** 40, 2 ** 63, True, np.int64(3), 1.0, None],
             "s": [0, 5, calls._Stream(), True, 1.5, "x", np.int64(3)]}
    forms = [_usual(name)]
    for j, k in enumerate(sig):
        for x in other[k]:
            forms.append(_usual(name))
            forms[-1][j] = x
    for args in forms:
        fast, general = calls._both(stub, monkeypatch, lambda: call(*args))
        assert fast == general, (name, args)
    taken = getattr(B._calls, {"norm_backward_workspace": "norm_space", "attention_forward_workspace": "attention_forward_space", "attention_backward_workspace": "attention_backward_space",
                               "cross_entropy_forward_workspace": "entropy_forward_space", "cross_entropy_backward_workspace": "entropy_backward_space"}
                    .get(name[4:], name[4:].replace("cross_entropy", "entropy")))
    assert taken(*forms[0]) == 0                                    # (the comparison would not see a fall back to the general path)
    C.c_int.in_dll(stub, "status").value = -3 if "workspace" in name else 3
    fast, general = calls._both(stub, monkeypatch, lambda: call(*forms[0]))
    assert fast == general and fast[0] == ("DdpError", 3)
