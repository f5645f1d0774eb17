"""Every form of the 4-bit product (64, 128 or 192 output channels per tile, and pairs of thread blocks) with every activation, with and
without a bias: the call's own plan says which form runs.  Tolerances as in test_gpu_mxfp4.py."""
import pytest
import torch

from paper_2411_00288_b200 import api
from tests.test_gpu_mxfp4 import DEV, _check_layer, _layer, _randn

pytestmark = pytest.mark.gpu

# (rows, C_in, C_out) whose form is the same with any activation and from 66 to 74 pairs of blocks on the device: ragged tiles of rows and of
# channels, last stages of all three widths of codes, odd numbers of row tiles (half a pair)
FORMS = {
    (64, False): [(129, 4072, 200), (3000, 1096, 136)],
    (128, False): [(2049, 1096, 520), (20_000, 256, 200)],
    (192, False): [(50_177, 96, 392), (30_001, 328, 1536)],
    (192, True): [(16_385, 4072, 576), (6000, 4096, 1536), (20_000, 4040, 952)],
}
CASES = [(form, *shape) for form, shapes in FORMS.items() for shape in shapes]
IDS = [f"{c}{'_pairs' if p else ''}-{r}x{i}-{o}" for (c, p), r, i, o in CASES]


def _expect(form, rows, cin, cout, act="none", bias=True):
    plan = api.ssconv_plan_mxfp4(api.make_desc(rows, 1, 1, cin, cout, 1, 1, bias=bias, relu=act == "relu", gelu=act == "gelu"))
    assert (plan["columns"], plan["pair"]) == form


@pytest.mark.parametrize("bias", [True, False], ids=["bias", "no_bias"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("form,rows,cin,cout", CASES, ids=IDS)
def test_layers_of_every_form(form, rows, cin, cout, act, bias):
    _expect(form, rows, cin, cout, act, bias)
    _check_layer(rows, cin, cout, act, bias=bias, seed=rows)


@pytest.mark.parametrize("form,rows,cin,cout", CASES, ids=IDS)
def test_sums_that_fit_come_out_exactly_in_every_form(form, rows, cin, cout):
    _expect(form, rows, cin, cout)
    buf = torch.full((rows * cout + 65_536,), 7.0, dtype=torch.bfloat16, device=DEV)
    out, want, _ = _layer(rows, cin, cout, exact=True, seed=cout, y=buf[:rows * cout].view(rows, 1, 1, cout))
    assert torch.equal(out, want.float().bfloat16()) and (buf[rows * cout:] == 7.0).all()


@pytest.mark.parametrize("form,rows,cin,cout", [CASES[i] for i in (0, 2, 4, 6)], ids=[IDS[i] for i in (0, 2, 4, 6)])
def test_nan_reaches_its_row_and_channel_alone_in_every_form(form, rows, cin, cout):
    _expect(form, rows, cin, cout, bias=False)
    x, w = _randn(1, rows, cin).bfloat16(), _randn(2, cout, cin).bfloat16()
    rows_hit, channels_hit = [0, 127, rows - 1], [3, cout - 1]
    x[rows_hit, cin - 1], w[channels_hit, 40] = float("nan"), float("inf")
    desc = api.make_desc(rows, 1, 1, cin, cout, 1, 1, bias=False)
    y = api.ssconv_forward_dense_mxfp4(desc, *api.ssconv_quantize_mxfp4(x), *api.ssconv_quantize_mxfp4(w)).view(rows, cout)
    bad = torch.zeros(rows, cout, dtype=torch.bool, device=DEV)
    bad[rows_hit], bad[:, channels_hit] = True, True
    assert torch.equal(y.isnan(), bad)


def test_captured_pairs_of_blocks():
    rows, cin, cout = 6000, 4096, 1536
    _expect((192, True), rows, cin, cout, "relu")
    x, w, b = _randn(1, rows, cin).bfloat16(), _randn(2, cout, cin).bfloat16(), _randn(3, cout)
    desc = api.make_desc(rows, 1, 1, cin, cout, 1, 1, bias=True, relu=True)
    wq = api.ssconv_quantize_mxfp4(w)
    want = api.ssconv_forward_dense_mxfp4(desc, *api.ssconv_quantize_mxfp4(x), *wq, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = api.ssconv_forward_dense_mxfp4(desc, *api.ssconv_quantize_mxfp4(x), *wq, b)
    x.copy_(x.flip(0))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y.flip(0), want)
