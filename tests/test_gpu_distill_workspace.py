"""The distillation loss with as much scratch as makes it fastest, with less, and with none: rows are split over workgroups, over
fewer, or not at all, and the results are the formulas' each time.  Nothing behind the scratch is written."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_1811_06965_amd import gp  # noqa: E402
from tests.test_gpu_distill import check, formulas, make  # noqa: E402


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab,top", [(2, 140001, 40), (5, 600011, 40), (90, 262144, 7)])
def test_any_scratch(dtype, rest, rows, vocab, top):
    _, z, ids, t = make(rows, vocab, top, dtype)
    ref = formulas(z, ids, t, 0.5, 0.0, rest, torch.ones(rows, device="cuda"))
    kind = gp.GP_BF16 if dtype == "bf16" else gp.GP_F32
    need = gp.gp_distill_workspace(kind, rows, vocab)
    splits = need // (8 * rows)
    assert splits > 3 and need == splits * 8 * rows
    ws = torch.empty(need + 64, dtype=torch.uint8, device="cuda")
    used = {}
    for size in (need, need - 1, need // 2 + 3, 3 * 8 * rows, 2 * 8 * rows, 2 * 8 * rows - 1, 8 * rows, 8, 0, None):
        ws.fill_(0xa5)
        loss, lse, far = torch.full((3, rows), -7.0, device="cuda").unbind(0)
        gp.gp_distill(kind, z.data_ptr(), rows, vocab, z.stride(0), ids.data_ptr(), t.data_ptr(), top, 0.5, 0.0, rest, loss.data_ptr(),
                      lse.data_ptr(), far.data_ptr() if rest else None, None if size is None else ws.data_ptr(), size or 0,
                      torch.cuda.current_stream().cuda_stream)
        check("loss", loss, ref)
        check("lse", lse, ref)
        if rest:
            check("rest_lse", far, ref)
        written = int((ws != 0xa5).nonzero().max()) + 1 if (ws != 0xa5).any() else 0
        assert written <= (size or 0)
        used[size] = written > 0
    assert used[need] and used[2 * 8 * rows] and not (used[2 * 8 * rows - 1] or used[8 * rows] or used[0] or used[None])


@pytest.mark.parametrize("dtype,rows,vocab,top,rest,split", [
    ("bf16", 1, 131072, 32, True, True), ("bf16", 96, 131072, 32, True, True), ("bf16", 1, 131072, 128, True, False),
    ("f32", 32, 80000, 32, True, True), ("f32", 64, 65536, 32, True, False), ("f32", 64, 65536, 32, False, True),
    ("f32", 96, 65536, 32, False, False), ("f32", 1, 262144, 128, True, True), ("f32", 1, 65536, 128, True, False)])
def test_split_where_that_is_faster(dtype, rows, vocab, top, rest, split):
    """Rows are split where their chunks cost more than what joining them does: its figures stand beside the rule."""
    _, z, ids, t = make(rows, vocab, top, dtype, ragged=False)
    kind = gp.GP_BF16 if dtype == "bf16" else gp.GP_F32
    need = gp.gp_distill_workspace(kind, rows, vocab)
    ws = torch.full((need,), 0xa5, dtype=torch.uint8, device="cuda")
    out = torch.empty(3, rows, device="cuda")
    gp.gp_distill(kind, z.data_ptr(), rows, vocab, vocab, ids.data_ptr(), t.data_ptr(), top, 1.0, 0.0, rest, out[0].data_ptr(),
                  out[1].data_ptr(), out[2].data_ptr(), ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    assert need > 0 and bool((ws != 0xa5).any()) == split
