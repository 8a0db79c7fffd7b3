"""Reading back 4-bit caches whose dense rows are few megabytes, just below and above the size from which they pass the
caches by, and many: every row against the definition, read again by what follows on the stream."""
import pytest
import torch

from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
@pytest.mark.parametrize("rows,H_kv,D", [(700, 4, 128), (24575, 4, 128), (24577, 4, 128), (12289, 4, 128), (60001, 8, 64)])
def test_every_row_is_what_the_pages_hold(dtype, rows, H_kv, D):
    page, pad = 64, 5
    P = -(-rows // page)
    g = torch.Generator(device="cuda").manual_seed(rows)
    pages = [torch.randint(0, 256, (P, H_kv, page, D // 2), dtype=torch.uint8, device="cuda", generator=g) for _ in "kv"]
    scales = [torch.randint(100, 150, (P, H_kv, page, D // 32), dtype=torch.uint8, device="cuda", generator=g) for _ in "kv"]
    order = torch.randperm(P, device="cuda", generator=g).to(torch.int32)
    out = [torch.full((rows + pad, H_kv, D), 9.0, dtype=dtype, device="cuda") for _ in "kv"]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    pdec.paged_kv_read(*pages, order[None].contiguous(), i32([rows]), i32([0, rows]), k_out=out[0], v_out=out[1],
                       k_scales=scales[0], v_scales=scales[1])
    again = [x * 1 for x in out]
    mags = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    for x, y, p, s in zip(out, again, pages, scales):
        code = torch.stack((p & 15, p >> 4), -1).flatten(-2).long()
        v = torch.where(code > 7, -1.0, 1.0).double() * mags[code & 7]
        v = v * torch.exp2(s.double() - 127).repeat_interleave(32, -1)
        want = v[order.long()].transpose(1, 2).reshape(P * page, H_kv, D)[:rows]
        assert torch.equal(x[:rows].double(), want) and (x[rows:] == 9).all() and torch.equal(x, y)
