"""Tiles that are written in parts and joined within the call: whatever the workspace held before."""
import pytest

from test_gpu_paged import _case, _check, cg, i32, torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,rep,lens,new", [
    (128, 1, [9000], [1]), (128, 3, [5000], [1]), (64, 7, [4000, 3, 6100], [1, 1, 1]), (256, 2, [3000], [2]),
    (128, 4, [2500, 7000], [4, 1]),
])
def test_parts_whatever_the_workspace_held(d, rep, lens, new):
    """One or a few rows of a tile's sixteen, long histories cut into many parts; a workspace full of NaN or
    of another call's parts before each call. Every call gives the same bits."""
    cases = [_case("bf16", d, 2, rep, 16, lens, new, seed=s) for s in (31, 32)]
    state, first = [], []
    for c in cases:
        pages = cg.Pages(n_pages=c["pool"].shape[1], page=16, H=2, d=d, n_req=len(lens), max_pages=c["table"].shape[1])
        q = c["q"].cuda()
        state.append([pages, cg.PagedAttention(rep, max(new), d ** -0.5), q, c["pool"].cuda(), i32(c["table"]), i32(c["lens"]), i32(c["cu"]),
                      torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")])
    ws = torch.empty(cg.paged_attention_workspace_bytes(*state[0][:2], state[0][2].shape[0]), dtype=torch.uint8, device="cuda")
    for k in range(200):
        s = state[k % 2]
        if k % 3 == 0:
            ws.fill_(255)                       # NaN as numbers
        s[7].fill_(float("nan"))
        cg.paged_attention(*s, ws)
        if k < 2:
            first.append((s[7].clone(), s[8].clone()))
            _check(cases[k], *first[k])
        assert torch.equal(s[7], first[k % 2][0]) and torch.equal(s[8], first[k % 2][1])
    assert cg.get_status() == 0
