"""Helpers for the tests of the experts' operators: choices of experts and, from the definition, the order of the rows that they make."""
import torch


def choices(tokens, experts, chosen, seed, how="some"):
    """[tokens, chosen], different experts for each token, int32 on the host.  `how`: "some" are more popular; "even"; "one": all tokens at the first ones; "first" tokens
    alone have any (a padded batch); "holes": each choice may be missing; "none"."""
    g = torch.Generator().manual_seed(seed)
    popular = torch.randn(experts, generator=g) * {"even": 0.0}.get(how, 1.0)
    if how == "one":
        popular = -100.0 * torch.arange(experts)
    u = torch.rand(tokens, experts, generator=g).clamp(1e-7, 1 - 1e-7)
    index = (popular - torch.log(-torch.log(u))).argsort(dim=1, descending=True)[:, :chosen]
    if how == "first":
        index[(tokens + 1) // 2:] = -1
    elif how == "holes":
        index[torch.rand(index.shape, generator=g) < 0.3] = -1
    elif how == "none":
        index[:] = -1
    return index.int().contiguous()


def tables(index, experts):
    """slots, source and offsets of the definition, int32 on the host: one choice after the other."""
    tokens, chosen = index.shape
    rows = [[] for _ in range(experts)]
    flat = index.flatten().tolist()
    for i, e in enumerate(flat):
        if 0 <= e < experts:
            rows[e].append(i)
    slots, source, offsets = [-1] * len(flat), [-1] * len(flat), [0]
    for e in range(experts):
        offsets.append(offsets[e] + len(rows[e]))
    order = [i for r in rows for i in r]
    for row, i in enumerate(order):
        slots[i], source[row] = row, i // chosen
    ints = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return ints(slots).view(tokens, chosen), ints(source), ints(offsets)


def plan_on_device(experts_module, index, experts):
    """The plan of the definition in device memory, and its groups: (expert, first row, end)."""
    slots, source, offsets = tables(index, experts)
    plan = experts_module.Plan(index.cuda(), slots.cuda(), source.cuda(), offsets.cuda())
    o = offsets.tolist()
    return plan, [(e, o[e], o[e + 1]) for e in range(experts)], source
