"""Bags whose rows attend to one another, trained and served.

Users' histories are ragged bags of items of one embedding table. Training:
every item's row is looked up (a bag per token), q, k and v are made of it,
the rows of a history attend to the earlier ones with a learned distance bias,
and the result predicts the next item's class. The gradients go back through
the attention into the distance bias (a small embedding table of its own,
updated by tc_sparse_update) and, cast and coalesced, into the item table.

Serving: the keys and values of the histories are kept in a paged 8-bit cache;
each new item appends one row and attends to the whole history by it.

    python examples/sequence_bags.py [--steps 40] [--users 512]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2010_13100_amd import tc  # noqa: E402

ITEMS, CLASSES = 2000, 16
HEADS, KV_HEADS, DIM = 4, 2, 16
WIDTH = HEADS * DIM
QKV = WIDTH + 2 * KV_HEADS * DIM
BUCKETS, REACH, MAX_LEN = 16, 64, 96


def histories(users, gen):
    """Ragged histories: lengths 1 .. MAX_LEN, every item's class one more
    than the last one's. Returns items, next items' classes, offsets, lengths."""
    lens = (40 + 12 * torch.randn(users, generator=gen)).round().long().clamp(1, MAX_LEN)
    offsets = torch.zeros(users + 1, dtype=torch.int32)
    offsets[1:] = lens.cumsum(0)
    user = torch.repeat_interleave(torch.arange(users), lens)
    step = torch.arange(int(offsets[-1])) - offsets[:-1].long()[user]
    first = torch.randint(CLASSES, (users,), generator=gen)
    cls = (first[user] + step) % CLASSES
    items = torch.randint(ITEMS // CLASSES, cls.shape, generator=gen) * CLASSES + cls
    return items.int(), (cls + 1) % CLASSES, offsets, lens.int()


class Model:
    def __init__(self, device, gen):
        def weights(*shape):
            return (torch.randn(shape, generator=gen) * shape[0] ** -0.5).to(device)

        self.device = device
        self.items = torch.randn((ITEMS, WIDTH), generator=gen).to(device)
        self.qkv = weights(WIDTH, QKV)
        self.head = weights(WIDTH, CLASSES)
        self.bias = torch.zeros((BUCKETS, HEADS), device=device)
        self.bias_state = torch.zeros_like(self.bias)
        self.bias_rows = torch.arange(BUCKETS, dtype=torch.int32, device=device)
        self.bias_count = torch.full((1,), BUCKETS, dtype=torch.int32, device=device)
        self.bucket_of = tc.relative_buckets(BUCKETS, REACH).to(device)

    def rows(self, x):
        """q, k and v of looked-up rows: strided views of one product."""
        t = x @ self.qkv
        return tuple(part.unflatten(1, (-1, DIM)) for part in
                     t.split([WIDTH, KV_HEADS * DIM, KV_HEADS * DIM], dim=1))

    def attention(self, **sizes):
        return tc.BagAttention(num_heads=HEADS, num_kv_heads=KV_HEADS, head_dim=DIM, causal=True,
                               dtype=torch.float32, bias_table=self.bias,
                               bucket_of=self.bucket_of, device=self.device, **sizes)


def train(model, users, steps, gen, lr=0.1):
    """Mean loss of every step."""
    dev, losses = model.device, []
    table_offset = torch.tensor([0, ITEMS], device=dev)
    item_state = torch.zeros_like(model.items)
    for _ in range(steps):
        items, target, offsets, lens = histories(users, gen)
        n = items.numel()
        items, target, offsets = items.to(dev), target.to(dev), offsets.to(dev)
        one_row_bags = torch.arange(n + 1, dtype=torch.int32, device=dev)
        emb = tc.EmbeddingTrainer(total_rows=ITEMS, dim=WIDTH, num_tables=1, bags_per_table=n,
                                  max_pairs=n, optimizer="adagrad", lr=lr, table=model.items)
        emb.A = item_state
        att = model.attention(num_seqs=users, max_q=int(lens.max()), total_q=n, total_k=n,
                              train=True)
        emb.forward_cast(table_offset, items, one_row_bags, n)
        q, k, v = model.rows(emb.out)
        out = att.forward(q, k, v, offsets)

        y = out.flatten(1).requires_grad_()
        head = model.head.requires_grad_()
        loss = torch.nn.functional.cross_entropy(y @ head, target, reduction="sum") / users
        grad_y, grad_head = torch.autograd.grad(loss, (y, head))

        att.backward(q, k, v, grad_y.view_as(out), offsets)
        grad_qkv = torch.cat([att.dq.flatten(1), att.dk.flatten(1), att.dv.flatten(1)], dim=1)
        emb.backward_update(grad_qkv @ model.qkv.T)
        tc.tc_sparse_update(model.bias, model.bias_state, model.bias_rows, att.grad_bias,
                            model.bias_count, BUCKETS, tc.TC_OPT_ADAGRAD, lr, 1e-8, 0.0)
        with torch.no_grad():
            model.qkv -= lr / 10 * (emb.out.T @ grad_qkv)
            model.head -= lr / 10 * grad_head
        model.head = head.detach()
        losses.append(float(loss.detach()) * users / n)
    return losses


def serve(model, users, new_items, gen, page_size=16):
    """Prefills a cache with the histories, then adds `new_items` items to each
    user's one at a time. Returns the outputs' largest difference from the
    attention over the whole histories with the cache's contents for keys and
    values, and the largest value."""
    dev = model.device
    items, _, offsets, lens = histories(users, gen)
    offsets, lens = offsets.to(dev), lens.to(dev)
    x = model.items[items.long().to(dev)]
    pages = (MAX_LEN + new_items + page_size - 1) // page_size
    table = torch.randperm(users * pages, generator=gen).int().view(users, pages).to(dev)
    cache = tc.PagedCache.empty(users * pages, page_size, KV_HEADS, DIM, device=dev)
    one_each = torch.arange(users + 1, dtype=torch.int32, device=dev)
    bound = int(lens.max()) + new_items

    q, k, v = model.rows(x)
    prefill = model.attention(num_seqs=users, max_q=MAX_LEN, max_k=bound, total_q=x.shape[0],
                              paged=True)
    decode = model.attention(num_seqs=users, max_q=1, max_k=bound, paged=True)
    cache.write(k, v, offsets, table, lens)
    outs, qs = [prefill.forward_paged(q, cache, offsets, table, lens)], [q]
    for _ in range(new_items):
        q, k, v = model.rows(model.items[torch.randint(ITEMS, (users,), generator=gen).to(dev)])
        lens = lens + 1
        cache.write(k, v, one_each, table, lens)
        outs.append(decode.forward_paged(q, cache, one_each, table, lens).clone())
        qs.append(q)

    # the same rows at once: queries in order of user and position, keys read back
    user = torch.repeat_interleave(torch.arange(users, device=dev), offsets.diff().long())
    order = torch.cat([user] + [torch.arange(users, device=dev)] * new_items).argsort(stable=True)
    got, queries = torch.cat(outs)[order], torch.cat(qs)[order].contiguous()
    offsets = torch.nn.functional.pad(lens.cumsum(0), (1, 0)).int()
    k = torch.empty((got.shape[0], KV_HEADS, DIM), device=dev)
    v = torch.empty_like(k)
    cache.read(k, v, offsets, table, lens)
    whole = model.attention(num_seqs=users, max_q=bound, total_q=k.shape[0], total_k=k.shape[0])
    want = whole.forward(queries, k, v, offsets)
    return float((got - want).abs().max()), float(v.abs().max())


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--users", type=int, default=512)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--new-items", type=int, default=8)
    args = ap.parse_args()
    gen = torch.Generator().manual_seed(1)
    model = Model("cuda", gen)
    losses = train(model, args.users, args.steps, gen)
    print(f"loss per item: {losses[0]:.3f} at first, {losses[-1]:.3f} after {args.steps} steps")
    diff, size = serve(model, args.users, args.new_items, gen)
    print(f"served from the 8-bit cache: within {diff:.1e} of one pass (values up to {size:.1f})")


if __name__ == "__main__":
    main()
