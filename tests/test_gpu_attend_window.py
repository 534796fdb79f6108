"""Attention with a sliding window and first tokens that stay visible
(bkv_attend_window) against the 64-bit reference: windows and sinks about the
groups' borders, types, head layouts, ragged and empty rows, what lies behind a
sequence and outside of every window, streams and graphs."""
import pytest
import torch

import attend_ref
import paper_2609_04971_amd as bkv
from attend_more import call, make, reference, run_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,G", [(1, 1), (1, 4), (3, 7), (9, 4), (40, 3)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 0), (32, 4), (33, 31), (64, 64), (65, 33), (127, 1), (300, 129), (700, 5), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("N", [1, 33, 129, 700])
def test_windows(dtype, T, G, window, sinks, N):
    run_case(2, 2, G, 64 if N == 129 else 128, T, N, N + N % 3, dtype, False, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,N", [(1, 5000), (4, 4097), (130, 130), (300, 1111), (257, 256), (1000, 3001)])
@pytest.mark.parametrize("window,sinks", [(64, 4), (100, 0), (1030, 77)])
def test_every_row_of_v_counts(dtype, D, T, N, window, sinks):
    run_case(1, 2, 4, D, T, N, N + 5, dtype, False, window=window, sinks=sinks, spread=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 4, 50])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 3), (64, 0), (200, 100)])
def test_ragged_lengths_and_rows_that_see_nothing(dtype, T, window, sinks):
    run_case(8, 2, 4, 64, T, 500, 517, dtype, False, lens=[-7, 0, 1, 3, 33, 499, 500, 2 ** 31 - 1], window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kw", [
    dict(B=3, Hkv=1, G=71, D=64, T=1, N=1234, cap=1234, lens=[1234, 0, 777], window=500, sinks=9),    # one kv-head for all
    dict(B=2, Hkv=1, G=128, D=128, T=1, N=2500, cap=2501, window=999, sinks=65),
    dict(B=3, Hkv=2, G=6, D=64, T=33, N=2100, cap=2100, lens=[2100, 40, 1999], window=333, sinks=4),
    dict(B=2, Hkv=3, G=1, D=128, T=200, N=3100, cap=3100, lens=[199, 3100], window=77, sinks=300),
    dict(B=9, Hkv=5, G=3, D=64, T=11, N=333, cap=340, lens=[333, 1, 0, 64, 65, 128, 5, 11, 12], window=17, sinks=2),
    dict(B=1, Hkv=2, G=2, D=128, T=2000, N=2000, cap=2000, window=256, sinks=4),                     # a prompt
    dict(B=300, Hkv=2, G=2, D=64, T=1, N=650, cap=651, window=65, sinks=1),
    dict(B=1, Hkv=1, G=4, D=128, T=1, N=40000, cap=40000, window=30000, sinks=1000),                 # split
    dict(B=1, Hkv=1, G=40, D=128, T=3, N=40000, cap=40000, window=30000, sinks=1000),
    dict(B=4, Hkv=2, G=1, D=64, T=128, N=9000, cap=9001, lens=[9000, 127, 128, 4500], window=4000, sinks=4),
])
def test_head_layouts_and_ragged_batches(dtype, kw):
    run_case(dtype=dtype, mx=False, **kw)
    run_case(dtype=dtype, mx=False, spread=True, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 7, 200])
def test_what_no_window_reaches_changes_nothing(dtype, T):
    """NaN between the first tokens and the windows, past the groups that a window's ends lie in: bits stay."""
    N, window, sinks = 2000, 300, 20
    d = bkv.dims(B=2, Hq=8, Hkv=2, D=128, N=N, W=0, C=0, budget=1, dtype=dtype)
    x = make(2, 2, 4, 128, T, N, N, dtype, 7, False)
    want = call(d, x, T, window=window, sinks=sinks)
    for k in "KV":
        x[k][:, :, 64:(N - T + 1 - window) // 64 * 64] = float("nan")
    got = call(d, x, T, window=window, sinks=sinks)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 5, 100])
def test_a_window_over_everything_is_causal_attention(dtype, T):
    N = 900
    d = bkv.dims(B=2, Hq=8, Hkv=2, D=128, N=N, W=0, C=0, budget=1, dtype=dtype)
    x = make(2, 2, 4, 128, T, N, N, dtype, 8, False, lens=[900, 333])
    ref = reference(x["q"], x["K"], x["V"], N, True, x["lens"])
    ref["mass"] = None
    for window, sinks in ((N, 0), (1, N), (450, 450), (2 ** 31 - 1, 0)):
        out, lse, _ = call(d, x, T, window=window, sinks=sinks)
        attend_ref.check(ref, out, lse, None, None, N)


@pytest.mark.parametrize("T", [1, 40])
def test_side_stream_and_captured_graph(T):
    N = 1600
    d = bkv.dims(B=4, Hq=8, Hkv=2, D=128, N=N, W=0, C=0, budget=1)
    x = make(4, 2, 4, 128, T, N, N, "bf16", 9, False, lens=[N, N, 700, 3])
    kw = {"window": 400, "sinks": 4}
    want = call(d, x, T, **kw)
    ws = bkv.attend_workspace(d, T)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = call(d, x, T, ws=ws, **kw)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    out, lse = torch.empty_like(x["q"]), torch.empty_like(want[1])
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            bkv.attend_window(d, x["q"], x["K"], x["V"], out, ws, 400, sinks=4, lens=x["lens"], lse=lse)
        graphs.append(g)
    for i in range(4):
        x["q"].mul_(0.9)
        x["lens"].copy_(torch.tensor([N - i, 300 * i, 2 * i, 900], dtype=torch.int32))  # the lengths move on
        x["K"].nan_to_num_(0.5), x["V"].nan_to_num_(0.5)
        out.fill_(float("nan"))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = (out.clone(), lse.clone())
        want = call(d, x, T, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), f"replay {i}"


def test_one_workspace_serves_every_window():
    d = bkv.dims(B=1, Hq=8, Hkv=2, D=128, N=9000, W=0, C=0, budget=1)
    for T in (1, 60):
        ws = bkv.attend_workspace(d, T)
        x = make(1, 2, 4, 128, T, 9000, 9000, "bf16", 4, False)
        for window, sinks in ((1, 0), (200, 4), (3000, 70), (8999, 1), (9000, 0), (10 ** 6, 10 ** 6)):
            ws.fill_(0xff)
            out, lse, _ = call(d, x, T, ws=ws, window=window, sinks=sinks)
            attend_ref.check(reference(x["q"], x["K"], x["V"], 9000, True, None, 0.0, window, sinks), out, lse, None, None, 9000)


def test_window_behind_2_32_bytes():
    # 17 M tokens of one head, 4.3 GB of keys; the window lies past 2^32 bytes, the sinks before
    N, D = (1 << 24) + 77, 128
    d = bkv.dims(B=1, Hq=2, Hkv=1, D=D, N=N, W=0, C=0, budget=1)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = {k: torch.zeros(1, 1, N, D, dtype=torch.bfloat16, device="cuda") for k in "KV"}
    for k in "KV":
        x[k][:, :, :200].normal_(generator=g), x[k][:, :, -2000:].normal_(generator=g)
    for T in (1, 40):
        x["q"], x["lens"] = torch.randn(1, 2, T, D, generator=g, device="cuda").bfloat16(), None
        out, lse, _ = call(d, x, T, window=1500, sinks=100)
        near = {k: torch.cat([x[k][:, :, :100], x[k][:, :, -1600:]], 2) for k in "KV"}
        attend_ref.check(reference(x["q"], near["K"], near["V"], 1700, True, None, 0.0, 1500, 100), out, lse, None, None, N)


def test_refusals_of_the_binding():
    d = bkv.dims(B=2, Hq=4, Hkv=2, D=128, N=32, N_cap=40, W=0, C=0, budget=1)
    x = make(2, 2, 2, 128, 1, 32, 40, "bf16", 1, False)
    ws, out = bkv.attend_workspace(d, 1), torch.empty_like(x["q"])
    for window, sinks in ((0, 0), (-1, 0), (5, -1)):
        with pytest.raises(bkv.BkvError) as e:
            bkv.attend_window(d, x["q"], x["K"], x["V"], out, ws, window, sinks=sinks)
        assert e.value.status == bkv.ERR_SHAPE
    for kw in (dict(K=x["K"].float()), dict(V=x["V"][:, :, :39]), dict(q=x["q"][:1]), dict(out=out.float())):
        a = dict(q=x["q"], K=x["K"], V=x["V"], out=out) | kw
        with pytest.raises(ValueError):
            bkv.attend_window(d, a["q"], a["K"], a["V"], a["out"], ws, 5)
