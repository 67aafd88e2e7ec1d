"""dsde_kv_map_next on the host: it refuses what dsde_kv_map refuses, with last_err or without."""
import ctypes

import pytest
import torch

from test_kv_host import FAKE, MAP, ODD, calls, dsde, rc, refused  # noqa: F401 (dsde is a fixture)


def after(last_err, **over):
    args = {}
    for k, v in dict(MAP, **over).items():
        args[k] = v
        if k == "accepted":
            args["last_err"] = last_err
    return args


@pytest.mark.parametrize("last_err", [None, FAKE])
def test_refusals(dsde, last_err):  # noqa: F811
    bad = [dict(B=0), dict(B=(1 << 20) + 1), dict(page_size=24), dict(pages=0), dict(pages=1 << 27), dict(width=0),
           dict(width=(1 << 26) + 1), dict(rows=-1), dict(rows=1 << 31), dict(ws=ODD)]
    bad += [{k: None} for k, v in MAP.items() if isinstance(v, ctypes.c_void_p)]
    for over in bad:
        assert rc(dsde, "dsde_kv_map_next", after(last_err, **over)) == 1, over
    assert rc(dsde, "dsde_kv_map_next", after(last_err, ws_bytes=64)) == 2


def test_binding_takes_it(dsde):  # noqa: F811
    i32 = dict(dtype=torch.int32)
    with pytest.raises(dsde.DsdeError, match="sl must be a GPU tensor"):
        dsde.kv_map(torch.zeros(3, **i32), torch.zeros(3, **i32), dsde.new_kv_pool(3, 4, 12, device="cpu"), 16, 5,
                    accepted=torch.zeros(3, **i32), last_err=torch.zeros(3, **i32))
