"""Tokens and targets that are no entry of the vocabulary: the caller of any operator that reads them can learn of it, and the agent's job stops."""
import pytest

pytestmark = pytest.mark.gpu

BAD = (40, -2, 1 << 40, -(1 << 50))


def test_they_are_reported_where_a_status_is_given():
    import torch
    import paper_2008_12260_amd as px
    for N in (0, 5, 700, 3000):
        for D in (16, 13):
            hidden, weight = torch.randn((N, D), device="cuda"), torch.randn((40, D), device="cuda")
            lse = torch.zeros(N, device="cuda")
            tokens = torch.randint(-1, 40, (N,), device="cuda")
            status = torch.zeros((), dtype=torch.int32, device="cuda")
            calls = (lambda t, s: px.token_loss(hidden, weight, t, status=s), lambda t, s: px.token_loss_grad(hidden, weight, t, lse, status=s),
                     lambda t, s: px.embed_grad(t, hidden, 40, status=s), lambda t, s: px.embed(t, weight, status=s))
            for call in calls:
                call(tokens, status)
                assert int(status) == 0
                for bad in BAD if N else ():
                    off = tokens.clone()
                    off[N // 2] = bad
                    status.zero_()
                    call(off, status)
                    assert int(status) == px.PX_ST_BAD_TOKEN
                    call(tokens, status)                     # added to what it holds
                    assert int(status) == px.PX_ST_BAD_TOKEN
                status.fill_(1)
                call(tokens, status)
                assert int(status) == 1
                status.zero_()


def test_in_a_callers_workspace_on_another_stream_and_in_a_graph():
    import torch
    import paper_2008_12260_amd as px
    hidden, weight = torch.randn((60, 24), device="cuda").bfloat16(), torch.randn((40, 24), device="cuda").bfloat16()
    tokens = torch.randint(0, 40, (60,), device="cuda")
    tokens[3] = 41
    workspace = torch.empty((1 << 20,), dtype=torch.float32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    px.token_loss(hidden, weight, tokens, workspace=workspace, stream=other, status=status)
    other.synchronize()
    assert int(status) == px.PX_ST_BAD_TOKEN
    px.embed_grad(tokens, hidden, 40, status=status)
    status.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        px.token_loss(hidden, weight, tokens, status=status)
        px.embed_grad(tokens, hidden, 40, status=status)
    for value, want in ((0, 0), (40, px.PX_ST_BAD_TOKEN), (39, 0), (-7, px.PX_ST_BAD_TOKEN)):
        status.zero_()
        tokens[3] = value
        graph.replay()
        torch.cuda.synchronize()
        assert int(status) == want


def test_wrong_statuses_are_refused():
    import torch
    import paper_2008_12260_amd as px
    hidden, weight, tokens = torch.randn((5, 16), device="cuda"), torch.randn((40, 16), device="cuda"), torch.zeros(5, dtype=torch.int64, device="cuda")
    for status in (torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int32)):
        for call in (lambda: px.token_loss(hidden, weight, tokens, status=status), lambda: px.token_loss_grad(hidden, weight, tokens, hidden[:, 0].contiguous(), status=status),
                     lambda: px.embed_grad(tokens, hidden, 40, status=status), lambda: px.embed(tokens, weight, status=status)):
            with pytest.raises(ValueError):
                call()


def test_the_agents_job_stops_at_them():
    from paper_2008_12260_amd.agent import Job
    job = Job(V=300, D=32, length=8, seed=2)
    whole = job.examples

    def strayed(m):
        tokens = whole(m)
        tokens[0, at] = 300
        return tokens
    for at in (0, 8):                                        # a token looked up, and one that is a target alone
        job.examples = strayed
        with pytest.raises(ValueError):
            job.iteration(4, 1)
        job.examples = whole
        job.iteration(4, 1)
