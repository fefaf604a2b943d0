"""Results of a backward pass that would lie over what another of its results still reads."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2003_10579_b200 import binding
    return binding


def test_results_over_kept_values(B):
    """The buffers of a Checkpoint count as the tensor that they stand for: db and dx are written before dw reads the kept values, db before dx takes the
    slopes from them.  dw, written last, may lie over them."""
    M, N, K = 64, 40, 96
    q = B.Checkpoint.empty(M, K, "cpu")
    apart = B.Checkpoint.empty(M, K, "cpu")
    dy, w = torch.zeros(M, N, dtype=torch.bfloat16), torch.zeros(N, K, dtype=torch.bfloat16)
    over = q.codes[:M // 2 * K].view(torch.bfloat16).view(M // 4, K)
    scales = q.scales[:4 * K // 32 * 4].view(torch.float32)
    beside = apart.codes[:M // 2 * K].view(torch.bfloat16).view(M // 4, K)

    def check(need, grad=False, **out):
        B._results_apart(need, dy, q, w, None, grad, *(out.get(k) for k in ("dx", "dw", "db")))

    for need, out in (("xw", dict(dx=over)), ("wb", dict(db=over[0])), ("wb", dict(db=scales)), ("xwb", dict(dx=scales))):
        with pytest.raises(ValueError):
            check(need, **out)
        with pytest.raises(ValueError):
            check(need, True, **out)
    with pytest.raises(ValueError):
        check("xb", True, db=over[0])                       # the slopes of dx
    check("xb", False, db=over[0])
    check("x", False, dx=over)                              # nobody else reads it
    check("xwb", True, dw=over)
    check("xwb", True, dx=beside, dw=over, db=apart.codes[-K * 4:].view(torch.float32))
    with pytest.raises(ValueError):
        check("xw", dx=beside, dw=beside)


@pytest.mark.gpu
def test_the_backward_pass_refuses_them(B):
    M, N, K = 64, 40, 96
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, dy, w = (torch.randn(*s, generator=gen, device="cuda").bfloat16() for s in ((M, K), (M, N), (N, K)))
    room = torch.zeros(2 * M * K, dtype=torch.uint8, device="cuda")
    kept = B.checkpoint(x)
    room[:M * K].copy_(kept.codes)
    q = B.Checkpoint(room[:M * K], kept.scales, M, K)
    want = B.linear_backward(dy, q, w)
    with pytest.raises(ValueError):
        B.linear_backward(dy, q, w, out=(room.view(torch.bfloat16).view(M, K), None, None))
    with pytest.raises(ValueError):
        B.linear_backward(dy, q, w, need="wb", out=(None, None, room[:4 * N].view(torch.float32)))
    for a, b in zip(B.linear_backward(dy, q, w), want):
        assert torch.equal(a, b)
