"""Embeddings of a block-model graph, and a classifier of the nodes' blocks on them.

The graph is the tiny workload's (10,000 nodes in 10 blocks).  The embeddings are
trained in one of two ways on the same co-occurrence triples:

  sampled  skip-gram negative sampling with sparse SGD (Trainer);
  exact    the softmax over all nodes that negative sampling stands in for: the
           source rows pass layer norm and a softmax head whose classes are the
           nodes (SoftmaxHead), and AdamW updates rows and head alike.

Then a second SoftmaxHead learns the blocks of half of the nodes from their rows
and is tested on the other half, as the paper's downstream classifier (Sec. 4.2).

    python examples/classify_blocks.py --objective exact --epochs 2
"""
import argparse
import os
import sys

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def blocks_of(workload):
    """The block of every (relabelled) node: equal blocks of consecutive ids."""
    from synth import relabel
    n = workload.cfg.num_nodes
    node = np.arange(n)
    block = np.empty(n, np.int64)
    block[relabel(node, n, workload.perm)] = node * workload.cfg.blocks // n
    return block


def train_sampled(workload, epochs, log):
    """Rows of the source table after skip-gram negative sampling, as the workload
    sets it."""
    import torch

    import paper_2307_14490_amd as P
    cfg, batch = workload.cfg, workload.cfg.batch
    src, dst, cc = (torch.from_numpy(a).cuda() for a in workload.epoch())
    trainer = P.Trainer(cfg.num_nodes, cfg.dim, cfg.num_neg, batch)
    first = 0
    for epoch in range(epochs):
        for a in range(0, src.numel(), batch):
            b = slice(a, a + batch)
            loss = trainer.step(src[b], dst[b], cc[b], first, cfg.lr)
            first += src[b].numel()
        log(f"epoch {epoch}: loss {loss.item() / src[b].numel():.4f} a triple in its last batch")
    if trainer.check() != 0:
        raise RuntimeError("device reported an error")
    return trainer.S


def train_exact(workload, epochs, batch, log, lr=1e-2, states="f32"):
    """Rows trained on the exact softmax over all nodes."""
    import torch

    import paper_2307_14490_amd as P
    cfg = workload.cfg
    src, dst, cc = (torch.from_numpy(a).cuda() for a in workload.epoch())
    weights = cc.float()
    rows = torch.randn((cfg.num_nodes, cfg.dim), device="cuda",
                       generator=torch.Generator(device="cuda").manual_seed(0)) * 0.1
    head = P.SoftmaxHead(cfg.num_nodes, cfg.dim, batch, lr=lr, weight_decay=0.0, states=states)
    opt = P.AdamW([rows], lr=lr, weight_decay=0.0, states=states)
    for epoch in range(epochs):
        for a in range(0, src.numel(), batch):
            b = slice(a, a + batch)
            loss, dx = head.step(rows[src[b]], dst[b], weights[b])
            opt.step([torch.zeros_like(rows).index_add_(0, src[b], dx)])
        log(f"epoch {epoch}: loss {loss.item():.4f} a triple in its last batch")
    head.check()
    opt.check()
    return rows


def classify(rows, block, classes, log, steps=200, norm="layer", max_norm=None):
    """Test accuracy of a softmax head on the rows of half of the nodes: how often the
    most likely block is the node's."""
    import torch

    import paper_2307_14490_amd as P
    label = torch.from_numpy(block.astype(np.int32)).cuda()
    half = torch.randperm(len(block), generator=torch.Generator().manual_seed(1)).cuda()
    train, test = half[: len(block) // 2], half[len(block) // 2:]
    head = P.SoftmaxHead(classes, rows.shape[1], len(block), lr=1e-2, norm=norm,
                         max_norm=max_norm, top=1)
    x, y = rows[train].contiguous(), label[train]
    for step in range(steps):
        loss, _ = head.step(x, y, want_dx=False)
    log(f"classifier: loss {loss.item():.4f} a node after {steps} steps")
    head.check()
    answers = head.answers(rows[test].contiguous(), label[test])
    log(f"classifier: log probability {answers.logp.mean().item():.4f} of a node's block, entropy "
        f"{answers.entropy.mean().item():.4f}")
    return (answers.ids[:, 0] == label[test]).float().mean().item()


def main(argv=None, log=print):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--objective", choices=("sampled", "exact"), default="exact")
    ap.add_argument("--epochs", type=int, default=2)
    ap.add_argument("--batch", type=int, default=8192)
    ap.add_argument("--states", choices=("f32", "q8"), default="f32",
                    help="moments of AdamW in 32 or in 8 bits")
    ap.add_argument("--norm", choices=("layer", "rms"), default="layer",
                    help="the classifier's norm")
    ap.add_argument("--clip", type=float, default=None,
                    help="largest norm of the classifier's gradients")
    a = ap.parse_args(argv)
    from synth import make_workload
    workload = make_workload("tiny", 0)
    if a.objective == "exact":
        rows = train_exact(workload, a.epochs, a.batch, log, states=a.states)
    else:
        rows = train_sampled(workload, a.epochs, log)
    accuracy = classify(rows, blocks_of(workload), workload.cfg.blocks, log, norm=a.norm,
                        max_norm=a.clip)
    log(f"{a.objective}: {100 * accuracy:.1f}% of the other half's blocks found "
        f"({100 / workload.cfg.blocks:.0f}% by chance)")
    return accuracy


if __name__ == "__main__":
    main()
